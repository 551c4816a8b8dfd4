"""Log probabilities, entropy, alternatives and their gradient against 64 bits.

Tolerances.  Powers of two and the products before them are within 2^-22 + |d| 2^-22 for a distance d from the largest logit; a thread adds
at most V / 256 + 64 terms one after the other, so a sum of V positive terms is off by at most (V / 256 + 64) 2^-24 of itself.  With c =
(V / 256 + 80) 2^-23: lse and log p are within c + 2^-22 (|value| + range), the entropy, a mean of distances, within (c + 2^-21) (1 + range), for the
range of the logits that count.  The gradient's p is e^(z - lse) from fp32 z and lse: 2^-22 (|z| + |lse| + 4) of itself; what it
multiplies is as exact, and the result is rounded once (2^-8 in bf16, 2^-24 in fp32).
"""
import math

import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
F64, F32, BF = torch.float64, torch.float32, torch.bfloat16
INF, NAN = math.inf, math.nan


def _logits(g, N, V, dtype, kind="random", pad=0):
    x = torch.randn(N, V, generator=g) * 3
    if kind == "rising":  # every element beats all before it
        x = torch.linspace(-8, 8, V).expand(N, V).clone()
    elif kind == "ties":
        x = x.round()
    elif kind == "equal":
        x = torch.full((N, V), 1.5)
    elif kind == "masked":
        x[torch.rand(N, V, generator=g) < 0.7] = -INF
    elif kind == "sure":  # one token has nearly all of the probability
        x[:, V // 3] = 40
    elif kind == "late":  # the large ones at the end
        x[:, -max(1, V // 100):] += 30
    x = x.to(dtype)
    if pad:  # rows in a wider tensor, at an odd offset
        wide = torch.full((N, V + pad), NAN, dtype=dtype)
        wide[:, pad // 2:pad // 2 + V] = x
        return wide.cuda()[:, pad // 2:pad // 2 + V]
    return x.cuda()


def _reference(x, scale):
    z = x.to(F64) * scale
    lse = torch.logsumexp(z, 1)
    logp = z - lse[:, None]
    return z, lse, logp, torch.special.entr(logp.exp()).sum(1)


def _best(x, top):
    """(values, indices) by the attention's rule: larger first, then the lower index."""
    v, i = torch.sort(x.to(F64) + 0.0, dim=1, descending=True, stable=True)
    v, i = v[:, :top], i[:, :top].int()
    i[v == -INF] = -1
    return v, i


def _check_forward(x, t, top, scale):
    r = T.token_logprobs(x, t, top=top, scale=scale)
    T.topk_check()
    N, V = x.shape
    z, lse, logp, H = _reference(x, scale)
    d = torch.where(z == -INF, z.amax(1, keepdim=True), z)
    span = (d.amax(1) - d.amin(1)).clamp_max(100)
    c = (V / 256 + 80) * 2.0 ** -23
    assert bool(((r.lse.to(F64) - lse).abs() <= c + 2.0 ** -22 * (lse.abs() + span)).all()), float((r.lse.to(F64) - lse).abs().max())
    assert bool(((r.entropy.to(F64) - H).abs() <= (c + 2.0 ** -21) * (1 + span)).all()), float((r.entropy.to(F64) - H).abs().max())
    if t is not None:
        want = logp.gather(1, t.long().clamp_min(0)[:, None])[:, 0]
        want[t < 0] = 0
        assert torch.equal(r.logp.isinf(), want.isinf())
        fine = ~want.isinf()
        assert bool(((r.logp.to(F64) - want).abs() <= c + 2.0 ** -22 * (want.abs() + lse.abs() + span))[fine].all())
        assert not r.logp[t < 0].any()
    if top:
        v, i = _best(x, min(top, V))
        assert torch.equal(r.top_ids[:, :V], i)
        want = v * scale - lse[:, None]
        assert torch.equal(r.top_logp[:, :V].isinf(), want.isinf())
        off = (r.top_logp[:, :V].to(F64) - want).abs()
        assert bool((off <= (c + 2.0 ** -22 * (want.abs() + (lse.abs() + span)[:, None])))[~want.isinf()].all())
        assert bool((r.top_ids[:, V:] == -1).all()) and bool((r.top_logp[:, V:] == -INF).all())
    return r


def _targets(g, N, V, wide=True):
    t = torch.randint(0, V, (N,), generator=g)
    t[3::5] = -100
    return t.to(torch.int64 if wide else torch.int32).cuda()


FORWARD = [(1, 1, 1), (1, 2, 3), (3, 7, 8), (2, 100, 20), (5, 1000, 64), (4, 4097, 128), (300, 513, 5), (2000, 64, 4), (1, 131072, 20), (7, 50001, 8),
           (160, 32000, 1), (400, 9999, 0), (2, 262147, 64), (9, 16384, 128), (33, 8191, 17)]


@pytest.mark.parametrize("N,V,top", FORWARD)
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_forward(N, V, top, dtype):
    g = torch.Generator().manual_seed(V)
    _check_forward(_logits(g, N, V, dtype), _targets(g, N, V, V % 2), top, 1.0 if V % 3 else 0.6)


@pytest.mark.parametrize("kind", ["rising", "ties", "equal", "masked", "sure", "late"])
@pytest.mark.parametrize("dtype,N,V,top,pad", [(BF, 3, 50001, 20, 0), (F32, 200, 3001, 64, 0), (BF, 170, 20000, 128, 7), (F32, 2, 131071, 3, 5), (BF, 6, 257, 100, 1)], ids=str)
def test_forward_hard_rows(kind, dtype, N, V, top, pad):
    g = torch.Generator().manual_seed(V)
    x = _logits(g, N, V, dtype, kind, pad)
    _check_forward(x, _targets(g, N, V), top, 1.0)


def test_rows_that_are_masked_infinite_or_not_numbers():
    for V in (5, 3000, 40000):
        x = torch.randn(6, V, device="cuda")
        x[0] = -INF
        x[1, V - 1] = NAN
        x[2, V // 2] = INF
        x[3, 1:] = -INF
        x[4, 2] = -NAN
        t = torch.tensor([1, 0, V // 2, 0, -1, 2], device="cuda")
        r = T.token_logprobs(x, t, top=3)
        T.topk_check()
        assert r.lse[0] == -INF and r.entropy[0] == 0 and r.logp[0] == -INF and bool((r.top_ids[0] == -1).all()) and bool((r.top_logp[0] == -INF).all())
        for n in (1, 2, 4):
            assert r.lse[n].isnan() and r.entropy[n].isnan() and r.top_logp[n].isnan().all() and bool((r.top_ids[n] == -1).all())
        assert r.logp[1].isnan() and r.logp[2].isnan() and r.logp[4] == 0
        assert r.logp[3] == 0 and r.entropy[3] == 0 and r.top_ids[3].tolist() == [0, -1, -1] and r.lse[3] == x[3, 0]
        assert torch.equal(r.top_ids[5], torch.topk(x[5], 3)[1].int())


def test_signed_zeros_are_equal():
    x = torch.tensor([[-0.0, 0.0, -0.0, 0.0, -1.0]], device="cuda")
    assert T.token_logprobs(x, top=5).top_ids.tolist() == [[0, 1, 2, 3, 4]]
    assert T.token_logprobs(x.to(BF), top=2).top_ids.tolist() == [[0, 1]]


def test_targets_behind_the_vocabulary_are_reported():
    x = torch.randn(3, 50, device="cuda")
    r = T.token_logprobs(x, torch.tensor([1, 50, 1 << 40], device="cuda"))
    with pytest.raises(T.TopkError, match="-8"):
        T.topk_check()
    assert r.logp[0] < 0 and r.logp[1] == 0 and r.logp[2] == 0


def test_large_and_small_logits():
    # values far from zero and far apart: the sum is taken around the largest
    for base in (-3e4, 3e4, 1e30):
        x = torch.tensor([[base, base - 1.0, -INF]], device="cuda")
        r = T.token_logprobs(x, torch.tensor([0], device="cuda"), top=2)
        want = torch.log_softmax(x.to(F64), 1)[0, 0]
        assert abs(float(r.logp[0]) - float(want)) <= 2.0 ** -20
    x = torch.zeros(1, 5000, device="cuda")
    x[0, 4000] = 3e38
    x[0, 4999] = -3e38
    r = T.token_logprobs(x, torch.tensor([4000], device="cuda"), top=1)
    assert float(r.logp[0]) == 0 and r.top_ids.tolist() == [[4000]] and float(r.entropy[0]) == 0


def _check_backward(x, t, top, entropy, scale, seed=0, inplace=False):
    N, V = x.shape
    g = torch.Generator().manual_seed(seed)
    r = T.token_logprobs(x, t, top=top, scale=scale)
    dl = torch.randn(N, generator=g).cuda() if t is not None else None
    dh = torch.randn(N, generator=g).cuda() if entropy else None
    dt = torch.randn(N, top, generator=g).cuda() if top else None
    z, lse, logp, H = _reference(x, scale)
    p = logp.exp()
    want, mag = torch.zeros_like(p), torch.zeros_like(p)
    pairs = ([(t.long(), dl)] if t is not None else []) + [(r.top_ids[:, m].long(), dt[:, m]) for m in range(top)]
    for at, dg in pairs:
        dg = torch.where(at < 0, 0.0, dg.to(F64))[:, None]
        at = at.clamp_min(0)[:, None]
        want.scatter_add_(1, at, dg)
        mag.scatter_add_(1, at, dg.abs())
        want -= p * dg
        mag += p * dg.abs()
    if entropy:
        term = torch.where(p == 0, 0.0, p * (logp + H[:, None])) * dh.to(F64)[:, None]
        want -= term
        mag += torch.where(p == 0, 0.0, p * (logp.abs() + H[:, None] + 1)) * dh.abs().to(F64)[:, None]
    want, mag = want * scale, mag * scale
    got = T.token_logprobs_bwd(x, r.lse, targets=t, dlogp=dl, entropy=r.entropy, dentropy=dh, top_ids=r.top_ids, dtop=dt, scale=scale, out=x if inplace else None)
    T.topk_check()
    assert got.dtype == x.dtype and (not inplace or got.data_ptr() == x.data_ptr())
    far = torch.where(z == -INF, 0.0, z.abs()) + lse.abs()[:, None] + 4
    tol = (2.0 ** -8 if x.dtype == BF else 2.0 ** -23) * want.abs() + 2.0 ** -22 * far * mag + (V / 256 + 80) * 2.0 ** -23 * mag + 1e-38
    err = (got.to(F64) - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


BACKWARD = [(1, 1, 0, False), (2, 3, 2, True), (5, 1000, 20, True), (300, 513, 0, False), (4, 50001, 8, True), (64, 8191, 0, True), (1, 131072, 128, False), (2000, 65, 1, False)]


@pytest.mark.parametrize("N,V,top,entropy", BACKWARD)
@pytest.mark.parametrize("dtype,pad", [(BF, 0), (F32, 0), (BF, 3), (F32, 1)], ids=str)
def test_backward(N, V, top, entropy, dtype, pad):
    g = torch.Generator().manual_seed(V)
    _check_backward(_logits(g, N, V, dtype, pad=pad), _targets(g, N, V, V % 2), top, entropy, 1.0 if V % 3 else 0.6)


def test_backward_of_parts():
    g = torch.Generator().manual_seed(3)
    _check_backward(_logits(g, 9, 2000, BF), None, 4, False, 1.0)
    _check_backward(_logits(g, 9, 2000, F32), None, 0, True, 2.0)
    _check_backward(_logits(g, 9, 2000, F32, "masked"), _targets(g, 9, 2000), 5, True, 1.0)
    _check_backward(_logits(g, 9, 2000, F32, "sure"), _targets(g, 9, 2000), 5, True, 1.0)


@pytest.mark.parametrize("dtype,pad", [(BF, 0), (F32, 5), (BF, 6)], ids=str)
def test_backward_in_place(dtype, pad):
    g = torch.Generator().manual_seed(4)
    for N, V in ((3, 4099), (200, 1000)):
        x = _logits(g, N, V, dtype, pad=pad)
        frame = x._base
        around = None if frame is None else frame.clone()
        _check_backward(x, _targets(g, N, V), 3, True, 1.0, inplace=True)
        if frame is not None:  # what lies between the rows stays
            assert torch.equal(frame[:, :pad // 2].isnan(), around[:, :pad // 2].isnan()) and frame[:, pad // 2 + V:].isnan().all()


def test_backward_against_differences():
    g = torch.Generator().manual_seed(5)
    x = torch.randn(2, 40, generator=g).cuda()
    t = torch.tensor([3, 17], device="cuda")
    a, b = torch.randn(2, generator=g).cuda(), torch.randn(2, generator=g).cuda()
    r = T.token_logprobs(x, t, scale=0.7)
    got = T.token_logprobs_bwd(x, r.lse, targets=t, dlogp=a, entropy=r.entropy, dentropy=b, scale=0.7)
    h = 2.0 ** -7

    def value(y):
        o = T.token_logprobs(y, t, scale=0.7)
        return (o.logp.to(F64) * a + o.entropy.to(F64) * b).sum()

    for n in range(2):
        for j in (0, 3, 17, 39):
            up, down = x.clone(), x.clone()
            up[n, j] += h
            down[n, j] -= h
            slope = float((value(up) - value(down)) / (float(up[n, j]) - float(down[n, j])))
            # the third derivative's part, h^2 / 6 times a few units, and the values' rounding over 2 h
            assert abs(slope - float(got[n, j])) <= 2 * h * h + 2.0 ** -20 / h


def test_rows_without_a_gradient():
    x = torch.randn(4, 3000, device="cuda")
    x[0] = NAN
    x[2] = -INF
    t = torch.tensor([-1, 5, 7, 9], device="cuda")
    r = T.token_logprobs(x, t)
    d = T.token_logprobs_bwd(x, r.lse, targets=t, dlogp=torch.tensor([1.0, 0.0, 1.0, 1.0], device="cuda"))
    assert not d[:3].any() and d[3].abs().sum() > 1
    x[1, 0] = NAN
    r = T.token_logprobs(x, t)
    d = T.token_logprobs_bwd(x, r.lse, targets=t, dlogp=torch.ones(4, device="cuda"))
    assert d[1].isnan().all()


def test_no_rows():
    x = torch.empty(0, 100, device="cuda")
    r = T.token_logprobs(x, torch.empty(0, dtype=torch.int64, device="cuda"), top=3)
    assert r.logp.shape == (0,) and r.top_ids.shape == (0, 3)
    assert T.token_logprobs_bwd(x, r.lse, entropy=r.entropy, dentropy=r.entropy).shape == (0, 100)


def test_graph_and_streams():
    g = torch.Generator().manual_seed(6)
    x, y = _logits(g, 3, 60000, BF), _logits(g, 900, 500, F32)
    want = [T.token_logprobs(v, top=9) for v in (x, y)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = [T.token_logprobs(v, top=9) for v in (x, y)]
    for _ in range(2):
        graph.replay()
        assert all(torch.equal(o[i], w[i]) for o, w in zip(out, want) for i in (1, 2, 3, 4))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        a, b = T.token_logprobs(x, top=9), T.token_logprobs(y, top=9, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a.top_logp, want[0].top_logp) and torch.equal(b.top_logp, want[1].top_logp) and torch.equal(b.entropy, want[1].entropy)
