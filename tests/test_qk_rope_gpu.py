"""Query/key norm with the position rotation (forward, cache-writing form, backward) against the
formulas in 64 bits.

Tolerances.  The kernels hold sums in fp32 and round a result once.  A bf16 result is within half a
unit in the last place, at most 2^-8 of its magnitude; the fp32 arithmetic before it (a sum of d
squares in a tree, a reciprocal root of 2 units, and about ten products and sums) stays below
2^-19 = 32 x 2^-24 of the magnitudes that are added, which the reference computes from absolute values.
"""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
F64 = torch.float64
ARITH = 2.0 ** -19


def _inputs(B, L, Hq, Hkv, d, dtype, seed=0, weights=True):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn(B, L, Hq + 2 * Hkv, d, generator=g).to(dtype).cuda()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(dtype).cuda() if weights else None for _ in range(2)]
    return qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:], w[0], w[1]


def _angles(cos, sin, positions, sections, B, L, sign=1.0):
    """cos, sin fp64 [B, L, 1, half]."""
    half = cos.shape[1]
    if positions is None:
        positions = torch.arange(L, device="cuda", dtype=torch.int32).expand(len(sections), B, L)
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    p = torch.stack([positions[a].long() for a in axis], -1) if half else torch.zeros(B, L, 0, dtype=torch.long, device="cuda")
    i = torch.arange(half, device="cuda")
    return cos.to(F64)[p, i][:, :, None], sign * sin.to(F64)[p, i][:, :, None]


def _rotate(n, c, s, interleaved):
    half = c.shape[-1]
    out = n.clone()
    i = torch.arange(half, device=n.device)
    ia, ib = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    out[..., ia] = n[..., ia] * c - n[..., ib] * s
    out[..., ib] = n[..., ib] * c + n[..., ia] * s
    return out


def _rotate_abs(n, c, s, interleaved):
    return _rotate(n.abs(), c.abs(), s.abs(), interleaved).abs().maximum(_rotate(n.abs(), c.abs(), -s.abs(), interleaved).abs())


def _ref_fwd(x, w, cs, eps, scale, interleaved, normalize):
    x = x.to(F64)
    n = x
    if normalize:
        n = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * (1 if w is None else w.to(F64))
    return (_rotate(n, *cs, interleaved) * scale).transpose(1, 2), (_rotate_abs(n, *cs, interleaved) * scale).abs().transpose(1, 2)


def _check(got, ref, mag):
    tol = (2.0 ** -8 * ref.abs() if got.dtype == torch.bfloat16 else 0) + ARITH * mag + 1e-30
    bad = (got.to(F64) - ref).abs() / tol
    assert torch.isfinite(got).all() and bad.max() <= 1, float(bad.max())


CASES = [
    # B, L, Hq, Hkv, d, rot, sections, interleaved, normalize, weights, dtype
    (1, 1, 1, 1, 64, 64, None, False, True, True, torch.bfloat16),
    (2, 77, 12, 12, 64, 64, None, False, True, True, torch.bfloat16),
    (1, 333, 8, 2, 128, 128, (16, 24, 24), False, True, True, torch.bfloat16),
    (3, 19, 5, 1, 128, 64, (7, 25), True, True, False, torch.float32),   # sections cut inside a lane's four pairs
    (2, 41, 3, 3, 96, 96, (13, 11, 24), False, True, True, torch.bfloat16),  # d not a power of two
    (1, 65, 7, 3, 256, 40, (20,), False, True, True, torch.float32),
    (1, 9, 4, 4, 16, 0, (0,), False, True, True, torch.bfloat16),       # norm alone
    (2, 30, 6, 6, 32, 32, None, True, False, False, torch.bfloat16),    # rotation alone
    (1, 2048, 33, 1, 8, 8, (1, 1, 1, 1), False, True, True, torch.float32),
    (1, 5000, 4, 4, 80, 80, None, True, True, True, torch.bfloat16),
]


def _positions(sections, B, L, rows, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, rows, (len(sections), B, L), generator=g, dtype=torch.int32).cuda()


def _setup(case, seed):
    B, L, Hq, Hkv, d, rot, sections, interleaved, normalize, weights, dtype = case
    q, k, v, qw, kw = _inputs(B, L, Hq, Hkv, d, dtype, seed, weights)
    rows = 2 * L + 7
    cos, sin = T.rope_tables(rows, rot)
    sec = sections or (rot // 2,)
    pos = None if sections is None else _positions(sec, B, L, rows, seed + 1)
    opts = dict(positions=pos, q_weight=qw, k_weight=kw, eps=1e-5, q_scale=d ** -0.5, sections=sections, interleaved=interleaved,
                normalize=normalize)
    return q, k, v, cos, sin, opts, _angles(cos, sin, pos, sec, B, L)


@pytest.mark.parametrize("case", CASES, ids=str)
def test_forward(case):
    q, k, v, cos, sin, o, cs = _setup(case, 1)
    qo, ko, vo = T.qk_norm_rope(q, k, v, cos, sin, **o)
    T.topk_check()
    _check(qo, *_ref_fwd(q, o["q_weight"], cs, 1e-5, o["q_scale"], o["interleaved"], o["normalize"]))
    _check(ko, *_ref_fwd(k, o["k_weight"], cs, 1e-5, 1.0, o["interleaved"], o["normalize"]))
    assert torch.equal(vo, v.transpose(1, 2))
    qo2, ko2, none = T.qk_norm_rope(q, k, None, cos, sin, **o)
    assert none is None and torch.equal(qo2, qo) and torch.equal(ko2, ko)


def _ref_bwd(dy, x, w, cs, eps, scale, interleaved, normalize):
    """dx, its magnitude, dw, its magnitude."""
    c, s = cs
    dy = dy.to(F64).transpose(1, 2) * scale
    g, gm = _rotate(dy, c, -s, interleaved), _rotate_abs(dy, c, s, interleaved)
    if not normalize:
        return g, gm, None, None
    x, w = x.to(F64), (torch.ones(x.shape[-1], dtype=F64, device="cuda") if w is None else w.to(F64))
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    u = g * w
    dx = r * u - x * r ** 3 * (u * x).mean(-1, keepdim=True)
    mag = r * gm * w.abs() + x.abs() * r ** 3 * (gm * w.abs() * x.abs()).mean(-1, keepdim=True)
    return dx, mag, (g * x * r).sum((0, 1, 2)), (gm * x.abs() * r).sum((0, 1, 2))


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("case", CASES, ids=str)
def test_backward(case, grad):
    B, L, Hq, Hkv, d = case[:5]
    if case[-1] == torch.float32 and grad == torch.bfloat16:
        pytest.skip("fp32 inputs take fp32 gradients")
    q, k, v, cos, sin, o, cs = _setup(case, 2)
    g = torch.Generator().manual_seed(5)
    dq, dk, dv = (torch.randn(B, h, L, d, generator=g).to(grad).cuda() for h in (Hq, Hkv, Hkv))
    packed, dqw, dkw = T.qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, **o)
    again = T.qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, **o)
    T.topk_check()
    for got, dy, x, w, scale, dw, dw2 in ((packed[:, :, :Hq], dq, q, o["q_weight"], o["q_scale"], dqw, again[1]),
                                          (packed[:, :, Hq:Hq + Hkv], dk, k, o["k_weight"], 1.0, dkw, again[2])):
        dx, mag, rw, rwm = _ref_bwd(dy, x, w, cs, 1e-5, scale, o["interleaved"], o["normalize"])
        _check(got, dx, mag)
        if o["normalize"]:
            # at most one addition for each (token, head) of a warp's share, 2^-24 each; the cases' shares are
            # below 400 additions
            assert ((dw.to(F64) - rw).abs() <= 400 * 2.0 ** -24 * rwm + 1e-30).all()
            assert torch.equal(dw, dw2)  # a fixed order of addition
        else:
            assert dw is None
    assert torch.equal(packed[:, :, Hq + Hkv:], dv.transpose(1, 2).to(q.dtype))
    assert torch.equal(packed, again[0])
    pair = T.qk_norm_rope_bwd(dq, dk, None, q, k, cos, sin, **o)[0]
    assert torch.equal(pair, packed[:, :, :Hq + Hkv])


def test_gradient_against_differences():
    # along random directions, central differences of the kernel's own fp32 forward pass: their error is
    # h^2 / 6 of the third derivative (h = 1e-2 on values of order 1: 1e-4 of the slope) and the outputs'
    # rounding, 2^-23 sqrt(n) / h, against slopes of order sqrt(n)
    B, L, Hq, Hkv, d = 2, 50, 4, 2, 64
    q, k, v, qw, kw = _inputs(B, L, Hq, Hkv, d, torch.float32, 9)
    cos, sin = T.rope_tables(64, 48)
    o = dict(q_weight=qw, k_weight=kw, q_scale=0.3)
    g = torch.Generator().manual_seed(3)
    dq, dk, dv = (torch.randn(B, h, L, d, generator=g).cuda() for h in (Hq, Hkv, Hkv))
    packed, dqw, dkw = T.qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, **o)

    def loss(q, k, qw, kw):
        a, b, _ = T.qk_norm_rope(q, k, v, cos, sin, q_weight=qw, k_weight=kw, q_scale=0.3)
        return float((a.double() * dq.double()).sum() + (b.double() * dk.double()).sum())

    h = 1e-2
    for which, grad in ((0, packed[:, :, :Hq]), (1, packed[:, :, Hq:Hq + Hkv]), (2, dqw), (3, dkw)):
        args = [q, k, qw, kw]
        u = torch.randn(args[which].shape, generator=g).cuda()
        hi, lo = ([x + sign * h * u if i == which else x for i, x in enumerate(args)] for sign in (1, -1))
        slope = (loss(*hi) - loss(*lo)) / (2 * h)
        want = float((grad.double() * u.double()).sum())
        scale = float(grad.double().norm())
        assert abs(slope - want) <= 2e-3 * scale, (which, slope, want, scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_weight_gradients_without_eps(dtype):
    # head counts that leave lanes without a row, eps = 0: the missing rows, zeros, must not reach the sums
    B, L, Hq, Hkv, d = 2, 45, 5, 3, 64
    q, k, v, qw, kw = _inputs(B, L, Hq, Hkv, d, dtype, 21)
    cos, sin = T.rope_tables(64, d)
    g = torch.Generator().manual_seed(22)
    dq, dk, dv = (torch.randn(B, h, L, d, generator=g).cuda() for h in (Hq, Hkv, Hkv))
    packed, dqw, dkw = T.qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, q_weight=qw, k_weight=kw, eps=0.0)
    T.topk_check()
    cs = _angles(cos, sin, None, (d // 2,), B, L)
    for got, dy, x, w, dw in ((packed[:, :, :Hq], dq, q, qw, dqw), (packed[:, :, Hq:Hq + Hkv], dk, k, kw, dkw)):
        dx, mag, rw, rwm = _ref_bwd(dy, x, w, cs, 0.0, 1.0, False, True)
        _check(got, dx, mag)
        assert ((dw.to(F64) - rw).abs() <= 400 * 2.0 ** -24 * rwm + 1e-30).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cache_rows(dtype):
    B, L, Hq, Hkv, d, cap = 3, 5, 8, 4, 64, 100
    q, k, v, qw, kw = _inputs(B, L, Hq, Hkv, d, dtype, 4)
    cos, sin = T.rope_tables(cap, d)
    start = torch.tensor([0, 17, 95], dtype=torch.int32, device="cuda")
    pos = (start[:, None] + torch.arange(L, device="cuda", dtype=torch.int32))[None].contiguous()
    kc, vc = (torch.full((B, Hkv, cap, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    qo, k2, v2 = T.qk_norm_rope(q, k, v, cos, sin, cache=(kc, vc), cache_start=start, positions=pos, q_weight=qw, k_weight=kw)
    T.topk_check()
    assert k2 is kc and v2 is vc
    qr, kr, vr = T.qk_norm_rope(q, k, v, cos, sin, positions=pos, q_weight=qw, k_weight=kw)
    assert torch.equal(qo, qr)
    for b in range(B):
        s = int(start[b])
        assert torch.equal(kc[b, :, s:s + L], kr[b]) and torch.equal(vc[b, :, s:s + L], vr[b])
        rest = torch.ones(cap, dtype=torch.bool, device="cuda")
        rest[s:s + L] = False
        assert (kc[b][:, rest] == 7).all() and (vc[b][:, rest] == 7).all()


def test_rows_and_positions_out_of_range_are_reported():
    # row 100 of a 100-row cache and row -1 are not written; a position beyond the tables takes the last row
    B, L, H, d, cap = 2, 2, 2, 64, 100
    q, k, v, _, _ = _inputs(B, L, H, H, d, torch.bfloat16, 6)
    cos, sin = T.rope_tables(10, d)
    kc, vc = (torch.full((B, H, cap, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    start = torch.tensor([99, -1], dtype=torch.int32, device="cuda")
    T.qk_norm_rope(q, k, v, cos, sin, cache=(kc, vc), cache_start=start)
    with pytest.raises(T.TopkError) as e:
        T.topk_check()
    assert e.value.code == -8
    assert (kc[0, :, :99] == 7).all() and (kc[1, :, 1:] == 7).all()
    assert torch.equal(vc[0, :, 99], v[0, 0]) and torch.equal(vc[1, :, 0], v[1, 1])
    far = torch.tensor([[[3, 10], [-4, 9]]], dtype=torch.int32, device="cuda")
    near = torch.tensor([[[3, 9], [0, 9]]], dtype=torch.int32, device="cuda")
    a = T.qk_norm_rope(q, k, v, cos, sin, positions=far)
    with pytest.raises(T.TopkError):
        T.topk_check()
    b = T.qk_norm_rope(q, k, v, cos, sin, positions=near)
    T.topk_check()
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_strided_inputs_and_streams():
    # q, k, v from tensors of their own layout (heads before tokens, padded rows), on a side stream
    B, L, Hq, Hkv, d = 2, 37, 6, 3, 64
    q, k, v, qw, kw = _inputs(B, L, Hq, Hkv, d, torch.bfloat16, 8)
    cos, sin = T.rope_tables(64, d)
    want = T.qk_norm_rope(q, k, v, cos, sin, q_weight=qw, k_weight=kw)
    q2 = q.transpose(1, 2).contiguous().transpose(1, 2)
    k2 = torch.zeros(B, L, Hkv, d + 4, dtype=torch.bfloat16, device="cuda")[..., :d].copy_(k)
    v2 = v.contiguous()[:1].expand(B, L, Hkv, d)  # a stride of 0
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = T.qk_norm_rope(q2, k2, v2, cos, sin, q_weight=qw, k_weight=kw)
    st.synchronize()
    T.topk_check()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(got[2], v2.transpose(1, 2))


def test_zero_and_nonfinite_rows():
    # a zero row has r = eps^-1/2 and stays zero; a NaN or infinity stays in its own head and token
    B, L, H, d = 1, 8, 4, 64
    q, k, v, qw, kw = _inputs(B, L, H, H, d, torch.float32, 12)
    q, k = q.clone(), k.clone()
    q[0, 2, 1] = 0
    k[0, 3, 2, 5] = float("nan")
    q[0, 4, 0, 7] = float("inf")
    cos, sin = T.rope_tables(16, d)
    qo, ko, _ = T.qk_norm_rope(q, k, v, cos, sin, q_weight=qw, k_weight=kw)
    T.topk_check()
    assert (qo[0, 1, 2] == 0).all()
    assert torch.isnan(ko[0, 2, 3]).all() and int(torch.isnan(ko).any(-1).sum()) == 1
    assert not torch.isfinite(qo[0, 0, 4]).all() and int((~torch.isfinite(qo)).any(-1).sum()) == 1
    dq = torch.ones_like(qo)
    packed, _, _ = T.qk_norm_rope_bwd(dq, dq, dq, q, k, cos, sin, q_weight=qw, k_weight=kw)
    bad = (~torch.isfinite(packed)).any(-1).nonzero().tolist()
    assert bad == [[0, 3, H + 2], [0, 4, 0]]


def test_offsets_beyond_32_bits():
    # the last rows of a cache of more than 2^32 elements (B 1, 2 heads of 64, 2^25 + 64 rows): 8.6 GB each
    cap = (1 << 25) + 64
    q, k, v, qw, kw = _inputs(1, 3, 2, 2, 64, torch.bfloat16, 14)
    cos, sin = T.rope_tables(8, 64)
    kc = torch.zeros(1, 2, cap, 64, dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    start = torch.tensor([cap - 3], dtype=torch.int32, device="cuda")
    T.qk_norm_rope(q, k, v, cos, sin, cache=(kc, vc), cache_start=start, q_weight=qw, k_weight=kw)
    T.topk_check()
    want = T.qk_norm_rope(q, k, v, cos, sin, q_weight=qw, k_weight=kw)
    assert torch.equal(kc[:, :, -3:], want[1]) and torch.equal(vc[:, :, -3:], want[2])
    assert int(torch.count_nonzero(kc[:, :, :-3])) == 0
