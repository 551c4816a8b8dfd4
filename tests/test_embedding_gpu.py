"""The embedding lookup and its gradient against 64 bits.

Tolerances.  A result is rounded once: 2^-8 of its magnitude in bf16, 2^-24 in fp32, after one fp32 product (2^-24).  The fp32
sum of n rows of dy, in any order, is off by at most n 2^-24 of the sum of their magnitudes; the scale and the addition to
what is there add 2^-24 each.
"""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
F64, F32, BF = torch.float64, torch.float32, torch.bfloat16
HALF = {F32: 2.0 ** -24, BF: 2.0 ** -8}


def _ids(g, N, rows, kind):
    if kind == "one":
        return torch.full((N,), rows - 1)
    if kind == "few":  # most tokens of a few ids
        u = torch.rand(N, generator=g)
        return ((rows + 1) ** u.double()).long().clamp(1, rows) - 1
    if kind == "own":
        return torch.randperm(max(N, rows), generator=g)[:N] % rows
    ids = torch.randint(0, rows, (N,), generator=g)
    ids[torch.rand(N, generator=g) < 0.3] = -1  # padding
    return ids


@pytest.mark.parametrize("dtype", [F32, BF], ids=str)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("N,rows,D,scale", [(1, 1, 1, 1.0), (1, 50, 768, 27.7), (8, 1000, 637, 1.0), (33, 7, 8, -0.5), (257, 301, 100, 1.0),
                                            (1000, 4096, 2048, 32.0), (5000, 129, 66, 2.0)])
def test_lookup(N, rows, D, scale, wide, dtype):
    g = torch.Generator().manual_seed(N + D)
    w = torch.randn(rows, D, generator=g).to(dtype).cuda()
    ids = _ids(g, N, rows, "padded").to(torch.int64 if wide else torch.int32).cuda()
    got = T.embedding(ids, w, scale=scale)
    T.topk_check()
    want = w[ids.long().clamp_min(0)].to(F64) * scale
    want[ids < 0] = 0
    assert got.dtype == dtype and got.shape == (N, D)
    assert bool(((got.to(F64) - want).abs() <= (HALF[dtype] + 2.0 ** -22) * want.abs()).all())
    if scale == 1.0:
        assert torch.equal(got.to(F64), want)


def test_lookup_shapes():
    w = torch.randn(10, 24, device="cuda")
    ids = torch.randint(0, 10, (2, 3, 5), device="cuda")
    assert torch.equal(T.embedding(ids, w), w[ids])
    assert T.embedding(ids[:0], w).shape == (0, 3, 5, 24)
    w[3] = float("nan")
    w[4, 0] = float("inf")
    assert torch.equal(T.embedding(torch.tensor([3, 4], device="cuda"), w).isnan(), w[3:5].isnan())


def test_ids_behind_the_table_are_reported():
    w = torch.randn(10, 24, device="cuda")
    ids = torch.tensor([1, 10, 2, 1 << 40], device="cuda")
    got = T.embedding(ids, w)
    with pytest.raises(T.TopkError, match="-8"):
        T.topk_check()
    assert torch.equal(got[::2], w[[1, 2]]) and not got[1::2].any()
    dw = T.embedding_bwd(torch.ones(4, 24, device="cuda"), ids, 10)
    with pytest.raises(T.TopkError, match="-8"):
        T.topk_check()
    want = torch.zeros(10, 24, device="cuda")
    want[1:3] = 1
    assert torch.equal(dw, want)


GRADS = [(1, 1, 1, "one"), (1, 50, 768, "few"), (31, 40, 96, "padded"), (32, 2, 64, "padded"), (33, 3, 637, "few"), (64, 64, 128, "own"), (100, 1, 8, "one"),
         (500, 1000, 100, "few"), (1025, 70, 256, "padded"), (4096, 4096, 48, "own"), (5000, 3, 33, "few"), (9001, 50001, 72, "few"), (20000, 257, 1032, "few"),
         (40000, 70000, 24, "padded"), (3000, 2500, 2048, "one"), (131073, 1000, 8, "few")]


@pytest.mark.parametrize("N,rows,D,kind", GRADS)
@pytest.mark.parametrize("dtype,grad", [(BF, BF), (BF, F32), (F32, F32), (F32, BF)], ids=str)
@pytest.mark.parametrize("into", [False, True])
def test_gradient(N, rows, D, kind, dtype, grad, into):
    g = torch.Generator().manual_seed(N + rows)
    dy = torch.randn(N, D, generator=g).to(dtype).cuda()
    ids = _ids(g, N, rows, kind).to(torch.int32 if D % 3 else torch.int64).cuda()
    before = torch.randn(rows, D, generator=g).to(grad).cuda() if into else None
    have = before.clone() if into else None
    got = T.embedding_bwd(dy, ids, rows, scale=1.5, grad_dtype=grad, into=have)
    T.topk_check()
    assert got.dtype == grad and (not into or got is have)
    at = torch.where(ids < 0, rows, ids.long())
    want, mag = (torch.zeros(rows + 1, D, dtype=F64, device="cuda").index_add_(0, at, x.to(F64) * 1.5)[:rows] for x in (dy, dy.abs()))
    count = torch.zeros(rows + 1, device="cuda", dtype=F64).index_add_(0, at, torch.ones(N, device="cuda", dtype=F64))[:rows, None]
    if into:
        want, mag = want + before.to(F64), mag + before.abs().to(F64)
        assert torch.equal(got[count[:, 0] == 0], before[count[:, 0] == 0])
    tol = (count + 2) * 2.0 ** -24 * mag + HALF[grad] * want.abs() * (1 + 2.0 ** -10)
    err = (got.to(F64) - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    again = T.embedding_bwd(dy, ids, rows, scale=1.5, grad_dtype=grad, into=before.clone() if into else None)
    assert torch.equal(got, again)  # the same order every time


def test_gradient_without_tokens():
    dy, ids = torch.randn(0, 16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    assert not T.embedding_bwd(dy, ids, 5).any()
    have = torch.randn(5, 16, device="cuda")
    assert torch.equal(T.embedding_bwd(dy, ids, 5, into=have), have)
    pad = torch.full((40,), -1, device="cuda")
    assert not T.embedding_bwd(torch.randn(40, 16, device="cuda"), pad, 5).any()
    before = have.clone()
    assert torch.equal(T.embedding_bwd(torch.randn(40, 16, device="cuda"), pad, 5, into=have), before)


def test_gradient_spoils_only_its_row():
    dy, ids = torch.randn(300, 40, device="cuda"), torch.arange(300, device="cuda") % 7
    dy[17] = float("nan")
    bad = T.embedding_bwd(dy, ids, 9).isnan()
    assert bad[17 % 7].all() and int(bad.sum()) == 40


def test_gradient_in_a_graph_and_beside_another_call():
    # two captured calls share nothing: replayed in turn and on two streams they give what they gave alone
    g = torch.Generator().manual_seed(1)
    data = [(torch.randn(n, 64, generator=g).cuda(), torch.randint(0, r, (n,), generator=g).cuda(), r) for n, r in ((700, 90), (3000, 500))]
    want = [T.embedding_bwd(*d) for d in data]
    graphs, outs = [], []
    for d in data:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(T.embedding_bwd(*d))
        graphs.append(graph)
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            out.zero_()
            graph.replay()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a = T.embedding_bwd(*data[0])
        b = T.embedding_bwd(*data[1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
