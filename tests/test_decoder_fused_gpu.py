"""The fused decoder (library linear layers, norms and rotation, AdamW) as a model is trained and served.

References are the same decoder in fp32 PyTorch operations.  bf16 activations and weights alone move a two-layer
network's gradients by several per cent (see test_decoder_gpu.py), so the fused decoder and a bf16
PyTorch one are both held against fp32, and the fused one must be about as close (within a factor of two).
"""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from paper_2106_06899_gb300.decoder import Decoder
from paper_2106_06899_gb300.optim import AdamW

pytestmark = pytest.mark.gpu


def _rel(a, b):
    return ((a.float() - b.float()).norm() / b.float().norm()).item()


def _plain(model, x, dtype):
    """The fused decoder's function in PyTorch operations, with its parameters cast to dtype."""
    P = {n: p.detach().to(dtype).requires_grad_() for n, p in model.named_parameters()}
    cos, sin = (t.to(torch.float32) for t in model.tables)
    B, L, D = x.shape
    x = x.to(dtype)
    ln = torch.nn.functional.layer_norm
    for i, layer in enumerate(model.layers):
        p = {n[len(f"layers.{i}."):]: v for n, v in P.items() if n.startswith(f"layers.{i}.")}
        h, d = layer.h, layer.dh
        qkv = (ln(x, (D,), p["ln1.weight"], p["ln1.bias"]) @ p["qkv.weight"].t()).view(B, L, 3 * h, d)
        q, k, v = qkv.split(h, 2)

        def turn(t, w):
            n = t.float() * torch.rsqrt(t.float().square().mean(-1, keepdim=True) + 1e-6) * w.float()
            a, b = n.chunk(2, -1)
            c, s = cos[:L, None], sin[:L, None]
            return torch.cat((a * c - b * s, b * c + a * s), -1)

        q, k = (turn(q, p["q_norm"]) * d ** -0.5).to(dtype), turn(k, p["k_norm"]).to(dtype)
        score = (q.transpose(1, 2).float() @ k.transpose(1, 2).float().transpose(-1, -2)).masked_fill(
            torch.ones(L, L, dtype=torch.bool, device=x.device).triu(1), float("-inf"))
        a = (score.softmax(-1).to(dtype) @ v.transpose(1, 2)).transpose(1, 2).reshape(B, L, D)
        x = x + a @ p["proj.weight"].t()
        x = x + torch.relu(ln(x, (D,), p["ln2.weight"], p["ln2.bias"]) @ p["w1"].t()) @ p["w2"].t()
    return ln(x, (D,), P["norm.weight"], P["norm.bias"]), P


@pytest.mark.parametrize("topk", [None, 256])
def test_fused_decoder_against_plain_operations(topk):
    torch.manual_seed(0)
    B, L, D, H, F, layers = 2, 256, 256, 4, 520, 2
    m = Decoder(layers, D, H, F, topk=topk, fused=True, max_positions=L)
    with torch.no_grad():
        for layer in m.layers:
            layer.q_norm.uniform_(0.5, 1.5)
            layer.k_norm.uniform_(0.5, 1.5)
    x = torch.randn(B, L, D, device="cuda", dtype=torch.bfloat16)
    g = torch.randn(B, L, D, device="cuda", dtype=torch.bfloat16)
    y = m(x)
    (y.float() * g.float()).sum().backward()
    T.topk_check()
    outs = {}
    for dtype in (torch.float32, torch.bfloat16):
        yp, P = _plain(m, x, dtype)
        (yp.float() * g.float()).sum().backward()
        outs[dtype] = (yp, P)
    (yr, ref), (yb, half) = outs[torch.float32], outs[torch.bfloat16]
    assert _rel(y, yr) <= max(2 * _rel(yb, yr), 1e-2)
    for n, p in m.named_parameters():
        e, plain = _rel(p.grad, ref[n].grad), _rel(half[n].grad, ref[n].grad)
        assert e <= max(2 * plain, 3e-2), (n, e, plain)


def _train(bits, masters, steps=60):
    torch.manual_seed(1)
    B, L, D, H, F, layers = 2, 512, 256, 4, 512, 2
    m = Decoder(layers, D, H, F, topk=64, fused=True, max_positions=L)
    opt = AdamW(m.parameters(), lr=2e-3, weight_decay=0.0, state_bits=bits, masters=masters, seed=3)
    g = torch.Generator("cuda").manual_seed(5)
    x = torch.randn(B, L, D, device="cuda", generator=g).bfloat16()
    want = torch.roll(x, 1, 1).float()  # the token before
    losses = []
    for _ in range(steps):
        opt.zero_grad()
        loss = (m(x).float() - want)[:, 1:].square().mean()
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    T.topk_check()
    return [float(v) for v in losses]


def test_training_falls_and_8_bit_moments_follow_32():
    full, eight, plain = _train(32, True), _train(8, True), _train(8, None)
    assert full[-1] < 0.8 * full[0]
    # the losses' fall with 8-bit moments, and with bf16 parameters alone, is the 32-bit run's to a fifth
    for other in (eight, plain):
        assert abs((other[0] - other[-1]) / (full[0] - full[-1]) - 1) <= 0.2, (full[-1], other[-1])


@pytest.mark.parametrize("topk", [None, 64])
def test_steps_give_what_the_whole_sequence_gives(topk):
    # the same bf16 operations a token at a time; kernels differ in their order of addition, so an output can be
    # off by some roundings (2^-8 each): 3e-2 of the output in the 2-norm for two layers
    torch.manual_seed(2)
    B, L, D, H, F, layers, cap = 3, 40, 256, 4, 512, 2, 64
    m = Decoder(layers, D, H, F, topk=topk, fused=True, max_positions=cap)
    x = torch.randn(B, L, D, device="cuda", dtype=torch.bfloat16)
    with torch.no_grad():
        whole = m(x)
    caches = m.new_cache(B, cap)
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    for t in range(L):
        y = m.step(x[:, t].contiguous(), caches, start)
        assert _rel(y, whole[:, t]) <= 3e-2, t
        start += 1
    T.topk_check()


def test_fused_decoder_with_topk_ffn_trains():
    torch.manual_seed(4)
    m = Decoder(2, 256, 4, 2048, topk=32, ffn_topk=128, fused=True, max_positions=300)
    x = torch.randn(1, 300, 256, device="cuda", dtype=torch.bfloat16)
    m(x).float().square().mean().backward()
    for n, p in m.named_parameters():
        assert p.grad is not None and torch.isfinite(p.grad.float()).all(), n


def test_refusals():
    with pytest.raises(ValueError):
        Decoder(1, 256, 4, 512, dtype=torch.float32, fused=True)
    m = Decoder(1, 256, 4, 512)
    with pytest.raises(ValueError):
        m.step(torch.zeros(1, 256, device="cuda", dtype=torch.bfloat16), [], torch.zeros(1, dtype=torch.int32, device="cuda"))
