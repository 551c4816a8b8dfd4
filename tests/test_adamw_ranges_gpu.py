"""AdamW with 8-bit moments where magnitudes in one block of 256 lie far apart: the update stays bounded.

For any gradients m^2 <= v (1 - beta1)^2 / (1 - beta2) sum_k (beta1^2 / beta2)^k (Cauchy-Schwarz over the sums
that m and v are), so |m| <= 7.28 sqrt(v) with betas 0.9 and 0.999, and the bias corrections' quotient is at most 1: no
step of the formula in exact arithmetic is longer than 7.28 lr.  In 8 bits the worst place is at the smallest codes: a
root of almost two codes cut to one (half of it), and m one code longer, which is max|m| / max root <= 7.28 of the root's
code: (2 + 1) 7.28 = 21.9 lr.
"""
import pytest
import torch

from paper_2106_06899_gb300 import optim
from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
LONGEST = 21.9


def _gradients(kind, size, n, g):
    x = torch.randn(n, device="cuda", generator=g)
    if kind == "sparse":  # one element in a hundred has a gradient, as the rows of an embedding
        x = x * (torch.rand(n, device="cuda", generator=g) < 0.01)
    x *= size
    x.view(-1, 256)[:, 17] = torch.randn(n // 256, device="cuda", generator=g)  # one large element in each block
    return x


@pytest.mark.parametrize("kind,size", [("dense", 1e-4), ("dense", 1e-5), ("dense", 1e-6), ("sparse", 1e-2), ("sparse", 1e-4)])
@pytest.mark.parametrize("pdt,masters", [(torch.float32, None), (torch.bfloat16, True)])
def test_steps_of_8_bit_moments_stay_bounded(kind, size, pdt, masters):
    n, lr = 1 << 14, 1.0
    g = torch.Generator("cuda").manual_seed(3)
    p = torch.zeros(n, dtype=pdt, device="cuda")
    opt = optim.AdamW([p], lr=lr, betas=(0.9, 0.999), weight_decay=0.0, state_bits=8, seed=5, masters=masters)
    held = opt.masters[0] if masters else p
    longest = torch.zeros((), device="cuda")
    for _ in range(400):
        before = held.clone()
        opt.step([_gradients(kind, size, n, g).to(pdt)])
        longest = torch.maximum(longest, (held - before).abs().max())
    T.topk_check()
    assert float(longest) <= LONGEST * lr, float(longest)


def test_a_positive_root_keeps_a_code():
    # roots over 2^30 in a block: those below the smallest code are held as it, a zero as zero
    g = torch.zeros(512, device="cuda")
    g[1:256] = 2.0 ** torch.linspace(-30, 0, 255, device="cuda")
    opt = optim.AdamW([torch.zeros(512, device="cuda")], state_bits=8)
    opt.step([g])
    code = opt.state["exp_avg_root"].float()
    assert float(code[0]) == 0 and float(code[256:].max()) == 0
    assert bool((code[1:256] >= 2.0 ** -9).all())
