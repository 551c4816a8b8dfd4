"""An optimizer's step on the decoder with token ids moves its parameters against their gradients."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from paper_2106_06899_gb300.decoder import Decoder
from paper_2106_06899_gb300.optim import AdamW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("topk", [None, 64])
def test_a_step_goes_against_the_gradient(topk):
    torch.manual_seed(0)
    m = Decoder(2, 256, 4, 512, topk=topk, fused=True, max_positions=128, vocab=1000)
    opt = AdamW(m.parameters(), lr=1e-3, weight_decay=0.0, masters=True)
    ids = torch.randint(0, 1000, (2, 128), device="cuda")
    (-m.logprobs(m(ids)[:, :-1], ids[:, 1:]).logp.mean()).backward()
    before = {n: p.detach().clone() for n, p in m.named_parameters()}
    opt.step()
    T.topk_check()
    for n, p in m.named_parameters():
        moved = p.detach().float() - before[n].float()
        assert bool((moved * p.grad.float() <= 0).all()), n
        # the first step is lr of each element, but for gradients near the step's epsilon of 1e-8: it shows in bf16 elements below 1/2
        clear = (p.grad.float().abs() > 1e-6) & (before[n].float().abs() < 0.5)
        assert bool((moved[clear] != 0).all()), n
    assert int(((m.embedding.detach() != before["embedding"]).any(1)).sum()) == 1000  # the output projection reaches every token
