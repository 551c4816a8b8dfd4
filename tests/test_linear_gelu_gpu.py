"""GELU and its slope over all bf16 numbers of magnitude 2^-12 to 12, each by itself.

Phi is formed in fp32 with the hardware's 2^x (to 2^-22) and 1/x (to 2^-23).  The fit's own error is 7.5e-8, the roundings of
five products at values up to 1/2 and the two instructions' errors come to 6e-7 at most (evaluated over the range with
the instructions' errors at their bounds), for Phi and for the slope Phi + z pdf.  Below zero the fit's relative
error grows, to 1e-3 at -4.5, 3.7e-3 at -6 and 3.2e-2 at -12.
"""
import math

import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
F64, BF = torch.float64, torch.bfloat16
ABSOLUTE = 6.2e-7


def _values():
    patterns = torch.arange(0x3980, 0x4141, dtype=torch.int32, device="cuda")  # 2^-12 to 12
    z = (patterns << 16).view(torch.float32)
    z = torch.cat((z, -z, torch.zeros(8, device="cuda"))).to(BF)
    return z[: z.numel() // 8 * 8]


def _phi(z):
    return 0.5 * torch.erfc(-z / math.sqrt(2))


@pytest.mark.parametrize("M", [1, 130])  # the kernel for few tokens, and tiles
def test_forward(M):
    z = _values()
    w = torch.zeros(z.numel(), 8, device="cuda", dtype=BF)
    w[:, 0] = z
    x = torch.zeros(M, 8, device="cuda", dtype=BF)
    x[:, 0] = 1
    y, kept = T.linear(x, w, act="gelu", return_preact=True)
    T.topk_check()
    assert torch.equal(kept[0], z) and torch.equal(kept[-1], z)
    zz = z.to(F64)
    want = zz * _phi(zz)
    # y is the rounding of a value that near (rounding keeps the order)
    lo, hi = ((want + d * ABSOLUTE * zz.abs()).to(BF) for d in (-1, 1))
    assert bool(((lo <= y) & (y <= hi)).all())
    # the tail by its relative error
    tail = zz < -1
    zz, want = zz[tail], want[tail]
    relative = torch.where(zz >= -4.5, 1e-3, torch.where(zz >= -6, 3.7e-3, 3.2e-2))
    most, least = ((want * (1 + d * relative)).to(BF) for d in (-1, 1))  # want is below zero
    assert bool(((least <= y[:, tail]) & (y[:, tail] <= most)).all())


def test_slope():
    z = _values()
    dy = torch.ones(1, z.numel(), device="cuda", dtype=BF)
    x, w = torch.zeros(1, 8, device="cuda", dtype=BF), torch.zeros(z.numel(), 8, device="cuda", dtype=BF)
    _, _, db = T.linear_bwd(dy, x, w, z[None].contiguous(), "gelu", bias=True, grad_dtype=torch.float32)
    T.topk_check()
    zz = z.to(F64)
    want = _phi(zz) + zz * torch.exp(-zz * zz / 2) / math.sqrt(2 * math.pi)
    # db is the slope itself here: 6.2e-7, and a rounding of a sum of up to 1.13
    assert bool(((db.to(F64) - want).abs() <= ABSOLUTE + 2.0 ** -23).all()), float((db.to(F64) - want).abs().max())
