"""Attention over packed prompts against 64 bits (tests/_attention.py has the tolerances)."""
import math

import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from tests._attention import attend

pytestmark = pytest.mark.gpu
F64, BF = torch.float64, torch.bfloat16
NAN = math.nan


def _inputs(lq, lk, Hq, Hkv, d, seed=0, rest=0, scale=1.5):
    """q, and k and v as views of one projection; `rest` rows of no sequence at the end hold NaN."""
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn(sum(lq) + rest, Hq, d, generator=g) * d ** -0.5 * scale).to(BF)
    kv = torch.randn(sum(lk) + rest, 2 * Hkv, d, generator=g).to(BF)
    if rest:
        q[-rest:], kv[-rest:] = NAN, NAN
    q, kv = q.cuda(), kv.cuda()
    return q, kv[:, :Hkv], kv[:, Hkv:]


def _edges(lens):
    return torch.tensor([0] + torch.tensor(lens).cumsum(0).tolist(), dtype=torch.int32, device="cuda")


def _verify(got, q, k, v, lq, lk, causal, heads=None, weight=2.0 ** -8):
    group = q.shape[1] // k.shape[1]
    at = bt = 0
    for n, m in zip(lq, lk):
        i, j = torch.arange(n, device="cuda"), torch.arange(m, device="cuda")
        ok = (j <= i[:, None] + m - n) if causal else torch.ones(n, m, dtype=torch.bool, device="cuda")
        for h in heads or range(q.shape[1]):
            want, tol = attend(q[at:at + n, h], k[bt:bt + m, h // group], v[bt:bt + m, h // group], ok, weight)
            err = (got[at:at + n, h].to(F64) - want).abs()
            assert bool((err <= tol).all()), (n, m, h, float((err / tol).max()))
        at, bt = at + n, bt + m


CASES = [([1], 1, 1), ([1, 1, 1], 4, 2), ([2, 3], 2, 2), ([127], 1, 1), ([128], 2, 1), ([129], 3, 1), ([255, 1, 257], 4, 4), ([64, 200, 5, 0, 33], 8, 2), ([0, 0, 7], 6, 1),
         ([300, 0, 0], 5, 5), ([700], 12, 4), ([1000, 31, 130], 16, 1), ([1, 2, 3, 4, 5, 6, 7, 8, 9, 10] * 7, 6, 2), ([513, 384], 40, 5), ([100], 128, 1),
         ([3, 150], 96, 2), ([2049], 2, 1)]


@pytest.mark.parametrize("lens,Hq,Hkv", CASES, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts(lens, Hq, Hkv, d, causal):
    q, k, v = _inputs(lens, lens, Hq, Hkv, d, seed=sum(lens))
    got = T.prompt_attention(q, k, v, _edges(lens), causal=causal)
    T.topk_check()
    _verify(got, q, k, v, lens, lens, causal, heads=range(0, Hq, max(1, Hq // 6)))


@pytest.mark.parametrize("lens,Hq,Hkv", CASES[:11] + CASES[12:13] + CASES[14:], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_padded_to_more_rows(lens, Hq, Hkv, d, causal):
    # the same prompts before so many rows of no sequence that weights are one bf16 each
    q, k, v = _inputs(lens, lens, Hq, Hkv, d, seed=sum(lens), rest=76 * 152 // Hq)
    got = T.prompt_attention(q, k, v, _edges(lens), causal=causal)
    T.topk_check()
    assert not got[sum(lens):].any()
    _verify(got, q, k, v, lens, lens, causal, heads=range(0, Hq, max(1, Hq // 6)))


@pytest.mark.parametrize("lq,lk,Hq,Hkv", [([1], [4000], 4, 1), ([200], [200], 12, 12), ([40, 3, 0, 61], [40, 1003, 5, 61], 16, 4)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sharp", [0.02, 1.0, 4.0])
def test_weights_of_few_rows_are_not_rounded_to_bf16(lq, lk, Hq, Hkv, d, sharp):
    # scores that hardly differ, so that weights lie side by side in a binade, and rows of few keys
    q, k, v = _inputs(lq, lk, Hq, Hkv, d, seed=sum(lk), scale=1.5 * sharp)
    got = T.prompt_attention(q, k, v, _edges(lq), _edges(lk))
    T.topk_check()
    _verify(got, q, k, v, lq, lk, True, weight=2.0 ** -16)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lq,lk", [([5, 100], [300, 101]), ([1, 1, 1], [1, 128, 1000]), ([64], [4096]), ([130, 4, 260], [70, 0, 129]), ([3, 3], [0, 0]), ([200], [1]),
                                   ([0, 9], [40, 50])], ids=str)
@pytest.mark.parametrize("causal", [True, False])
def test_keys_of_other_lengths(lq, lk, d, causal):
    # more keys than queries (a prompt that goes on), and fewer: rows without a key are zeros
    q, k, v = _inputs(lq, [*lk[:-1], lk[-1] + 1], 4, 2, d, seed=1)
    got = T.prompt_attention(q, k, v, _edges(lq), k_starts=_edges(lk), causal=causal)
    T.topk_check()
    _verify(got, q, k, v, lq, lk, causal)


def test_one_long_prompt():
    lens = [9000]
    q, k, v = _inputs(lens, lens, 3, 1, 128, seed=2)
    got = T.prompt_attention(q, k, v, _edges(lens))
    T.topk_check()
    _verify(got, q, k, v, lens, lens, True, heads=[1])


@pytest.mark.parametrize("d", [64, 128])
def test_large_scores_move_the_maximum(d):
    # scores that rise by far more than e^88 along the keys, and rows of one dominant key
    lens = [600, 77]
    q, k, v = _inputs(lens, lens, 2, 1, d, seed=3, scale=30.0)
    k = k * torch.linspace(0.1, 4, k.shape[0], device="cuda", dtype=BF)[:, None, None]
    got = T.prompt_attention(q, k.contiguous(), v, _edges(lens))
    T.topk_check()
    _verify(got, q, k, v, lens, lens, True)


@pytest.mark.parametrize("d", [64, 128])
def test_rows_of_no_sequence(d):
    lens, rest = [70, 130], 60
    q, k, v = _inputs(lens, lens, 6, 3, d, seed=4, rest=rest)
    out = torch.full((q.shape[0], 6, d), 7.0, dtype=BF, device="cuda")
    assert T.prompt_attention(q, k, v, _edges(lens), out=out) is out
    T.topk_check()
    assert bool((out[200:] == 7).all())
    _verify(out[:200], q, k, v, lens, lens, True)
    got = T.prompt_attention(q, k, v, _edges(lens))
    assert torch.equal(got[:200], out[:200]) and not got[200:].any()
    # sequences that begin further on: the rows before them are of none
    starts = _edges([100]) + 50
    got = T.prompt_attention(q[:200], k[:200], v[:200], starts)
    T.topk_check()
    assert not got[:50].any() and not got[150:].any()
    _verify(got[50:150], q[50:150], k[50:150], v[50:150], [100], [100], True)


def test_other_sequences_cannot_spoil_one():
    # a sequence of NaN and infinities next to two that share its tiles
    lens = [40, 30, 50]
    q, k, v = _inputs(lens, lens, 4, 2, 64, seed=5)
    want = T.prompt_attention(q, k, v, _edges(lens))
    for x in (NAN, math.inf, -math.inf):
        q2, k2, v2 = q.clone(), k.clone(), v.clone()
        for t in (q2, k2, v2):
            t[40:70] = x
        got = T.prompt_attention(q2, k2, v2, _edges(lens))
        assert torch.equal(got[:40], want[:40]) and torch.equal(got[70:], want[70:])
        assert got[40:70].isnan().all()


def test_bounds_outside_the_tensors_are_cut_and_reported():
    q, k, v = _inputs([100], [100], 2, 2, 64, seed=6)
    want = T.prompt_attention(q, k, v, _edges([60, 40]))
    for bad in ([0, 60, 500], [-3, 60, 100]):
        got = T.prompt_attention(q, k, v, torch.tensor(bad, dtype=torch.int32, device="cuda"))
        with pytest.raises(T.TopkError, match="-8"):
            T.topk_check()
        assert torch.equal(got, want)
    T.prompt_attention(q, k, v, torch.tensor([0, 60, 40, 100], dtype=torch.int32, device="cuda"))  # bounds that fall
    with pytest.raises(T.TopkError, match="-8"):
        T.topk_check()


def test_layouts():
    # head-major tensors, as the query/key norm writes them, and a wider projection's columns
    lens = [33, 150]
    q, k, v = _inputs(lens, lens, 8, 2, 128, seed=7)
    want = T.prompt_attention(q, k, v, _edges(lens))
    major = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    assert torch.equal(T.prompt_attention(*major, _edges(lens)), want)
    packed = torch.cat((q, k, v, q[:, :1]), 1)
    assert torch.equal(T.prompt_attention(packed[:, :8], packed[:, 8:10], packed[:, 10:12], _edges(lens)), want)
    one = T.prompt_attention(q[:33], k[:33], v[:33], _edges([33]))
    assert torch.equal(one, want[:33])


def test_graph_and_streams():
    lens = [[300, 20], [64, 1000, 3]]
    data = [(*_inputs(n, n, 4, 2, d, seed=8), _edges(n)) for n, d in zip(lens, (64, 128))]
    want = [T.prompt_attention(*x) for x in data]
    graphs, outs = [], []
    for x in data:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(T.prompt_attention(*x))
    for _ in range(3):
        for graph, out in zip(graphs, outs):
            out.zero_()
            graph.replay()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
    # the captured lengths are read at every replay
    starts = data[0][3]
    starts.copy_(_edges([20, 300]))
    graphs[0].replay()
    assert torch.equal(outs[0], T.prompt_attention(*data[0]))
    starts.copy_(_edges(lens[0]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        a, b = T.prompt_attention(*data[0]), T.prompt_attention(*data[1], stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_no_queries():
    q = torch.empty(0, 4, 64, dtype=BF, device="cuda")
    assert T.prompt_attention(q, q[:, :2], q[:, :2], _edges([0, 0])).shape == (0, 4, 64)
