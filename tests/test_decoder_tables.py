"""The fused decoder's rotation tables go where its parameters go (no GPU needed)."""
import torch

from paper_2106_06899_gb300 import decoder
from paper_2106_06899_gb300 import topk as T


def test_tables_follow_the_decoder():
    m = decoder.Decoder(1, 64, 1, 64, topk=8, fused=True, max_positions=16, device="cpu")
    want = T.rope_tables(16, 64, device="cpu")
    assert all(torch.equal(a, b) for a, b in zip(m.tables, want))
    m.to("meta")
    assert m.norm.weight.device.type == "meta" and all(t.device.type == "meta" for t in m.tables)
    m.to_empty(device="cpu")
    assert all(torch.equal(a, b) for a, b in zip(m.tables, want))
    torch.nn.Sequential(m).to(torch.float16).bfloat16()  # the angles stay in 32 bits
    assert all(t.dtype == torch.float32 and torch.equal(t, b) for t, b in zip(m.tables, want))
    assert not any("table" in n or "cos" in n or "sin" in n for n in m.state_dict())
    assert decoder.Decoder(1, 64, 1, 64, topk=8, device="cpu").to("meta").tables is None
