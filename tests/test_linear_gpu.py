"""The linear layer with bias, activation and residual, forward and backward, against 64 bits.

Tolerances.  A bf16 result is within half a place of the fp32 one: 2^-8 of its magnitude.  The fp32 sum
of K products, sixteen to a tensor-core step, is off by at most (K / 16 + 32) 2^-23 of the sum of
their magnitudes; the activations have slopes below 1.2, and their own arithmetic (erff, __expf: up to 14 units
for arguments below 10) stays within 2^-19 of |z|.  The backward pass rounds dz to bf16 before the two products:
2^-8 of the sum of the products' magnitudes, elementwise, and 2^-8 / sqrt(3) of the result in
the 2-norm, as the result's own rounding (the two are independent: 3.2e-3 together, held to 4e-3).
"""
import math

import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
F64, BF = torch.float64, torch.bfloat16


def _act(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp_min(0), "gelu": lambda: 0.5 * z * torch.erfc(-z / math.sqrt(2)),
            "silu": lambda: z * torch.sigmoid(z)}[act]()


def _slope(z, act):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).to(F64),
            "gelu": lambda: 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
            "silu": lambda: s * (1 + z * (1 - s))}[act]()


def _rand(g, *shape, scale=1.0):
    return (scale * torch.randn(*shape, generator=g)).to(BF).cuda()


def _forward(M, K, N, act, bias, res, keep, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, w = _rand(g, M, K), _rand(g, N, K, scale=K ** -0.5)
    b, r = (_rand(g, N) if bias else None), (_rand(g, M, N) if res else None)
    got = T.linear(x, w, b, act, r, return_preact=keep)
    T.topk_check()
    y, z = got if keep else (got, None)
    rz = x.to(F64) @ w.to(F64).t() + (0 if b is None else b.to(F64))
    mag = (K / 16 + 32) * 2.0 ** -23 * (x.abs().to(F64) @ w.abs().to(F64).t() + (0 if b is None else b.abs().to(F64)))
    if keep:
        err = (z.to(F64) - rz).abs()
        assert bool((err <= 2.0 ** -8 * rz.abs() + mag + 1e-30).all()), float((err / (2.0 ** -8 * rz.abs() + mag)).max())
    want = _act(rz, act) + (0 if r is None else r.to(F64))
    tol = 2.0 ** -8 * want.abs() + 1.2 * mag + 2.0 ** -19 * (rz.abs() + (0 if r is None else r.abs().to(F64))) + 1e-30
    err = (y.to(F64) - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())
    return x, w, b, r, y


@pytest.mark.parametrize("M,K,N", [
    (1, 8, 8), (1, 1024, 4096), (2, 264, 40), (3, 768, 2304), (4, 4096, 1000), (7, 2056, 136), (8, 768, 768), (13, 520, 3000), (16, 8192, 256),
    (17, 768, 768), (33, 64, 8), (64, 4096, 512), (100, 1032, 2064), (127, 16, 24), (128, 128, 128), (129, 72, 264), (257, 2048, 520),
    (640, 640, 2560), (1000, 8, 1000), (2049, 1000, 136), (5000, 768, 768),
])
@pytest.mark.parametrize("act,bias,res,keep", [("none", False, False, False), ("relu", True, False, True), ("gelu", True, True, True), ("silu", False, True, False)])
def test_forward(M, K, N, act, bias, res, keep):
    _forward(M, K, N, act, bias, res, keep, seed=M + N)


def test_forward_many_tiles():
    # several units for each CTA, both accumulators reused, ragged in both directions
    _forward(16 * 1024 + 5, 512, 1096, "silu", True, True, True)


@pytest.mark.parametrize("M,K,N", [(1, 8, 8), (5, 768, 256), (100, 1032, 2064), (129, 72, 264), (1000, 8, 1000), (2049, 1000, 136), (513, 2048, 520),
                                   (9000, 256, 128), (40, 4096, 64), (4097, 640, 2560)])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_backward(M, K, N, act, grad):
    g = torch.Generator().manual_seed(M + K)
    x, w, dy = _rand(g, M, K), _rand(g, N, K, scale=K ** -0.5), _rand(g, M, N)
    z = None if act == "none" else _rand(g, M, N)
    dx, dw, db = T.linear_bwd(dy, x, w, z, act, bias=True, grad_dtype=grad)
    again = T.linear_bwd(dy, x, w, z, act, bias=True, grad_dtype=grad)
    T.topk_check()
    assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), again))  # a fixed order of addition
    zz = torch.zeros(M, N, dtype=F64, device="cuda") if z is None else z.to(F64)
    dz = dy.to(F64) * _slope(zz, act)
    zm = dy.abs().to(F64) * _slope(zz, act).abs() + 2.0 ** -12 * dy.abs().to(F64) * (1 + zz.abs())
    half = 2.0 ** -8
    for got, want, mag, n in ((dx, dz @ w.to(F64), zm @ w.abs().to(F64), N), (dw, dz.t() @ x.to(F64), zm.t() @ x.abs().to(F64), M)):
        tol = (half * want.abs() if got.dtype == BF else 0) + ((half if act != "none" else 0) + (n / 16 + 32) * 2.0 ** -23) * mag + 1e-30
        err = (got.to(F64) - want).abs()
        assert bool((err <= tol).all()), float((err / tol).max())
        if want.numel() > 1000:
            assert float(err.norm() / want.norm()) <= 4e-3
    tol = (half * dz.sum(0).abs() if grad == BF else 0) + (M / 256 + 40) * 2.0 ** -24 * zm.sum(0) + 2.0 ** -19 * (dy.abs().to(F64) * (1 + zz.abs())).sum(0)
    err = (db.to(F64) - dz.sum(0)).abs()
    assert bool((err <= tol + 1e-30).all()), float((err / tol).max())
    only = T.linear_bwd(dy, x, w, z, act, need_dx=False, grad_dtype=grad)
    assert only[0] is None and only[2] is None and torch.equal(only[1], dw)
    only = T.linear_bwd(dy, x, w, z, act, bias=True, need_dw=False, grad_dtype=grad)
    assert torch.equal(only[0], dx) and only[1] is None and torch.equal(only[2], db)


@pytest.mark.parametrize("act", ["gelu", "silu", "none"])
def test_gradient_against_differences(act):
    # central differences of the kernel's forward pass along a random direction of x and of w.  With a step of
    # size h in 2-norm units of the input, y's roundings (2^-8 / sqrt(3) of each value) enter the
    # directional slope as noise: the loss is a sum of n outputs against dy of order 1
    M, K, N = 256, 128, 192
    g = torch.Generator().manual_seed(3)
    x, w, dy = _rand(g, M, K), _rand(g, N, K, scale=K ** -0.5), _rand(g, M, N)
    _, z = T.linear(x, w, act=act, return_preact=True)
    dx, dw, _ = T.linear_bwd(dy, x, w, z if act != "none" else None, act)
    for which, grad in ((0, dx), (1, dw)):
        base = (x, w)[which]
        u = torch.randn(base.shape, generator=g).cuda() * float(base.float().std())
        h = 0.125
        hi, lo = (base.float() + h * u).to(BF), (base.float() - h * u).to(BF)
        step = hi.to(F64) - lo.to(F64)  # the difference as it is after rounding
        a, b = (T.linear(*((t, w) if which == 0 else (x, t)), act=act).to(F64) for t in (hi, lo))
        slope = float(((a - b) * dy.to(F64)).sum())
        want = float((grad.to(F64) * step).sum())
        noise = 2.0 ** -8 / math.sqrt(3) * float(((a.square() + b.square()) * dy.to(F64).square()).sum().sqrt())
        size = float((grad.to(F64).abs() * step.abs()).square().sum().sqrt())
        # six deviations of the rounding noise, the gradient's own rounding, and h^2 / 6 of a third
        # derivative of order 1 (2.6e-3 of the slope's size)
        assert abs(slope - want) <= 6 * noise + 0.02 * size, (slope, want, noise, size)


def test_residual_in_place_and_strides():
    g = torch.Generator().manual_seed(1)
    for M in (5, 700):
        x, w, r = _rand(g, M, 256), _rand(g, 520, 256, scale=1 / 16), _rand(g, M, 520)
        want = T.linear(x, w, residual=r)
        y = r.clone()
        T.topk_linear_fwd(x, w, y, residual=y)
        assert torch.equal(y, want)
    with pytest.raises(ValueError):
        T.linear(x.t(), w)
    with pytest.raises(ValueError):
        T.linear(x, w, residual=r[:, ::2])


def test_streams():
    g = torch.Generator().manual_seed(2)
    x, w = _rand(g, 300, 4096), _rand(g, 264, 4096, scale=1 / 64)
    want = T.linear(x, w, act="gelu")
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = T.linear(x, w, act="gelu")
    st.synchronize()
    T.topk_check()
    assert torch.equal(got, want)


@pytest.mark.parametrize("M", [3, 40, 300])
def test_nonfinite_values_stay_in_their_rows(M):
    # a NaN token and an infinite weight row touch only their own outputs; ragged tiles around them stay clean
    g = torch.Generator().manual_seed(4)
    K, N = 200, 72
    x, w = _rand(g, M, K), _rand(g, N, K)
    x[1, 5] = float("nan")
    w[70, 199] = float("inf")
    x[:, 199] = 1.0
    y = T.linear(x, w, act="relu")
    bad = ~torch.isfinite(y)
    assert bad[1].all() and bad[:, 70].all() and torch.isnan(y[1]).all()
    bad[1] = False
    bad[:, 70] = False
    assert not bad.any()


def test_replays_in_a_graph():
    g = torch.Generator().manual_seed(6)
    x, w, b = _rand(g, 64, 512), _rand(g, 256, 512, scale=0.05), _rand(g, 256)
    y = torch.empty(64, 256, dtype=BF, device="cuda")
    T.topk_linear_fwd(x, w, y, b, act="silu")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.topk_linear_fwd(x, w, y, b, act="silu")
    x.copy_(_rand(g, 64, 512))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, T.linear(x, w, b, "silu"))
