"""Attention of drafted tokens over caches against 64 bits (tests/_attention.py has the tolerances)."""
import math

import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from tests._attention import attend

pytestmark = pytest.mark.gpu
F64, BF = torch.float64, torch.bfloat16


def _inputs(B, Hq, Hkv, T_, cap, d, seed=0):
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn(B, Hq, T_, d, generator=g) * d ** -0.5 * 1.5).to(BF).cuda()
    return q, *((torch.randn(B, Hkv, cap, d, generator=g)).to(BF).cuda() for _ in range(2))


def _parents(B, T_, seed=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.rand(B, T_, generator=g) * (torch.arange(T_) + 1)).long() - 1


def _reads(parents):
    """[B, T, T]: does token i read drafted token j?"""
    B, n = parents.shape
    ok = torch.zeros(B, n, n, dtype=torch.bool)
    for b in range(B):
        for i in range(n):
            j = i
            while j >= 0:
                ok[b, i, j] = True
                j = int(parents[b, j])
    return ok.cuda()


def _verify(got, q, keys, values, lens, reads, cap, weight=2.0 ** -8):
    B, Hq, n, d = q.shape
    group = Hq // keys.shape[1]
    for b, m in enumerate(lens):
        total = min(max(m, 0) + n, cap) if m >= 0 else 0
        ok = torch.ones(n, total, dtype=torch.bool, device="cuda")
        ok[:, max(m, 0):] = reads[b][:, :max(0, total - max(m, 0))]
        for h in range(0, Hq, max(1, Hq // 5)):
            want, tol = attend(q[b, h], keys[b, h // group, :total], values[b, h // group, :total], ok, weight)
            err = (got[b, h].to(F64) - want).abs()
            assert bool((err <= tol).all()), (b, h, float((err / tol).max()))


CASES = [(1, 1, 1, 1, 8, [0]), (1, 12, 12, 1, 300, [299]), (4, 12, 12, 1, 4096, [0, 1, 2048, 4095]), (3, 8, 2, 5, 700, [0, 127, 695]), (2, 32, 8, 16, 2000, [1984, 130]),
         (2, 4, 4, 64, 1000, [64, 936]), (1, 16, 1, 33, 500, [128]), (2, 40, 8, 7, 400, [121, 3]), (1, 64, 1, 64, 300, [200]), (1, 128, 1, 2, 260, [126]),
         (2, 9, 3, 31, 12000, [11900, 7]), (6, 2, 1, 3, 129, [126, 125, 0, 1, 60, 64]), (40, 4, 2, 2, 150, [3 * i for i in range(40)])]


@pytest.mark.parametrize("B,Hq,Hkv,n,cap,lens", [CASES[i] for i in (1, 2, 4, 5, 10)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sharp", [0.02, 1.0, 4.0])
def test_weights_are_not_rounded_to_bf16(B, Hq, Hkv, n, cap, lens, d, sharp):
    # scores that hardly differ, so that weights lie side by side in a binade, and rows of few keys
    q, keys, values = _inputs(B, Hq, Hkv, n, cap, d, seed=cap + 1)
    q = (q.float() * sharp).to(BF)
    got = T.tree_attention(q, keys, values, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    chain = torch.ones(n, n, dtype=torch.bool, device="cuda").tril().expand(B, n, n)
    _verify(got, q, keys, values, lens, chain, cap, weight=2.0 ** -16)
    T.topk_check()


@pytest.mark.parametrize("B,Hq,Hkv,n,cap,lens", CASES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_trees(B, Hq, Hkv, n, cap, lens, d):
    q, keys, values = _inputs(B, Hq, Hkv, n, cap, d, seed=cap)
    parents = _parents(B, n, seed=n)
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = T.tree_attention(q, keys, values, kv_len, tree=T.tree_mask(parents.cuda()))
    T.topk_check()
    _verify(got, q, keys, values, lens, _reads(parents), cap)


@pytest.mark.parametrize("Hq,Hkv,n", [(4, 1, 8), (32, 1, 1), (31, 1, 1), (33, 1, 1), (11, 1, 3), (2, 2, 32), (2, 2, 33), (3, 3, 31)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_few_rows(Hq, Hkv, n, d):
    cap, lens = 1400, [0, 1, 63, 64, 65, 127, 128, -1, 1300, 1200, 190, 700]
    q, keys, values = _inputs(len(lens), Hq, Hkv, n, cap, d, seed=n)
    parents = _parents(len(lens), n, seed=Hq)
    for b, m in enumerate(lens):
        keys[b, :, max(0, m + n) if m >= 0 else 0:] = math.nan
        values[b, :, max(0, m + n) if m >= 0 else 0:] = math.nan
    got = T.tree_attention(q, keys, values, torch.tensor(lens, dtype=torch.int32, device="cuda"), tree=T.tree_mask(parents).cuda())
    T.topk_check()
    _verify(got, q, keys, values, lens, _reads(parents), cap, weight=2.0 ** -16)


@pytest.mark.parametrize("d", [64, 128])
def test_chain(d):
    # without a tree a token reads those before it: the last tokens of a causal sequence
    q, keys, values = _inputs(2, 6, 2, 20, 400, d, seed=1)
    kv_len = torch.tensor([380, 55], dtype=torch.int32, device="cuda")
    got = T.tree_attention(q, keys, values, kv_len)
    T.topk_check()
    chain = torch.arange(-1, 19).expand(2, 20)
    _verify(got, q, keys, values, [380, 55], _reads(chain), 400)
    assert torch.equal(got, T.tree_attention(q, keys, values, kv_len, tree=T.tree_mask(chain.cuda())))


def test_one_tree_for_all():
    q, keys, values = _inputs(3, 4, 2, 9, 200, 64, seed=2)
    kv_len = torch.tensor([100, 7, 191], dtype=torch.int32, device="cuda")
    parents = _parents(1, 9, seed=3)
    words = T.tree_mask(parents.cuda())
    got = T.tree_attention(q, keys, values, kv_len, tree=words)
    assert torch.equal(got, T.tree_attention(q, keys, values, kv_len, tree=words.expand(3, 9).contiguous()))
    _verify(got, q, keys, values, [100, 7, 191], _reads(parents.expand(3, 9)), 200)


def test_rows_behind_a_sequence_are_not_read():
    for d in (64, 128):
        q, keys, values = _inputs(3, 4, 2, 5, 300, d, seed=4)
        lens = [0, 123, 250]
        kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
        want = T.tree_attention(q, keys, values, kv_len)
        for x in (math.nan, math.inf, -math.inf):
            for b, m in enumerate(lens):
                keys[b, :, m + 5:], values[b, :, m + 5:] = x, x
            assert torch.equal(T.tree_attention(q, keys, values, kv_len), want)
        T.topk_check()


def test_tokens_that_read_nothing_and_sequences_that_are_not_there():
    q, keys, values = _inputs(3, 4, 2, 4, 100, 64, seed=5)
    kv_len = torch.tensor([0, -1, 30], dtype=torch.int32, device="cuda")
    words = torch.tensor([[1, 0, 5, 0]], dtype=torch.int64, device="cuda")
    got = T.tree_attention(q, keys, values, kv_len, tree=words)
    T.topk_check()
    reads = torch.tensor([[[1, 0, 0, 0], [0, 0, 0, 0], [1, 0, 1, 0], [0, 0, 0, 0]]], device="cuda").bool().expand(3, 4, 4)
    _verify(got, q, keys, values, [0, -1, 30], reads, 100)
    assert not got[0, :, 1].any() and not got[1].any() and got[2].abs().sum() > 0


def test_more_tokens_than_the_cache_holds():
    q, keys, values = _inputs(2, 2, 1, 8, 64, 64, seed=6)
    lens = [60, 64]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    got = T.tree_attention(q, keys, values, kv_len)
    with pytest.raises(T.TopkError, match="-8"):
        T.topk_check()
    _verify(got, q, keys, values, lens, _reads(torch.arange(-1, 7).expand(2, 8)), 64)
    got = T.tree_attention(q, keys, values, torch.tensor([1 << 30, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    with pytest.raises(T.TopkError, match="-8"):
        T.topk_check()
    assert got.isfinite().all()


def test_layouts():
    q, keys, values = _inputs(2, 8, 2, 6, 150, 128, seed=7)
    kv_len = torch.tensor([100, 140], dtype=torch.int32, device="cuda")
    want = T.tree_attention(q, keys, values, kv_len)
    turned = [t.transpose(1, 2).contiguous().transpose(1, 2) for t in (q, keys, values)]  # rows before heads
    assert torch.equal(T.tree_attention(*turned, kv_len), want)
    both = torch.cat((keys, values), 1)
    assert torch.equal(T.tree_attention(q, both[:, :2], both[:, 2:], kv_len), want)


def test_a_decoding_step_agrees_with_the_prompt():
    # the last token of each packed sequence, and the same one against a cache
    lens = [200, 77, 1]
    q, k, v = (torch.randn(sum(lens), h, 64, device="cuda").to(BF) for h in (6, 2, 2))
    starts = torch.tensor([0, 200, 277, 278], dtype=torch.int32, device="cuda")
    whole = T.prompt_attention(q, k, v, starts)
    keys, values = (torch.zeros(3, 2, 256, 64, dtype=BF, device="cuda") for _ in range(2))
    for b, n in enumerate(lens):
        rows = slice(int(starts[b]), int(starts[b]) + n)
        keys[b, :, :n], values[b, :, :n] = k[rows].transpose(0, 1), v[rows].transpose(0, 1)
    last = starts[1:].long() - 1
    one = T.tree_attention(q[last][:, :, None], keys, values, torch.tensor(lens, dtype=torch.int32, device="cuda") - 1)
    # two roundings of the result and of the weights
    assert bool(((one[:, :, 0].double() - whole[last].double()).abs() <= 2.0 ** -6 * v.abs().max()).all())


def test_graph_and_streams():
    data = []
    for s, (B, n, cap, d) in enumerate(((3, 1, 3000, 64), (2, 12, 900, 128))):
        q, keys, values = _inputs(B, 8, 2, n, cap, d, seed=s)
        data.append((q, keys, values, torch.tensor([cap - 50 - 7 * b for b in range(B)], dtype=torch.int32, device="cuda")))
    want = [T.tree_attention(*x) for x in data]
    graphs, outs = [], []
    for x in data:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(T.tree_attention(*x))
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            out.zero_()
            graph.replay()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    data[0][3].sub_(1000)  # the captured lengths are read at every replay
    graphs[0].replay()
    assert torch.equal(outs[0], T.tree_attention(*data[0]))
    data[0][3].add_(1000)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a, b = T.tree_attention(*data[0]), T.tree_attention(*data[1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


@pytest.mark.parametrize("B,Hq,Hkv,n,cap,d", [(6, 32, 8, 4, 7944, 128), (2, 1, 1, 6, 55568, 128), (4, 12, 12, 1, 8192, 64), (16, 32, 8, 16, 20000, 128)])
def test_long_caches_again_and_again(B, Hq, Hkv, n, cap, d):
    # loads that arrive in any order, over many key tiles: every run gives the same bits, and the first one is right
    q, keys, values = _inputs(B, Hq, Hkv, n, cap, d, seed=9)
    lens = [max(0, cap - n - 1000 * b - 13 * b * b) for b in range(B)]
    kv_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    first = T.tree_attention(q, keys, values, kv_len)
    T.topk_check()
    _verify(first[:, :, -1:], q[:, :, -1:], keys, values, [m + n - 1 for m in lens], torch.ones(B, 1, 1, dtype=torch.bool, device="cuda"), cap)
    for _ in range(60):
        assert torch.equal(T.tree_attention(q, keys, values, kv_len), first)
    T.topk_check()
