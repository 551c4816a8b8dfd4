"""Tables, logits and caches of more than 2^31 elements: what lies at their ends gives what it gives by itself."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
BF, F64 = torch.bfloat16, torch.float64


def test_embedding():
    rows, D = 2_200_000, 1024  # 2.25e9 elements
    weight = torch.empty(rows, D, dtype=BF, device="cuda")
    weight[-3:].normal_(), weight[:2].normal_()
    ids = torch.tensor([rows - 1, 0, rows - 3, 1, rows - 2, -1], device="cuda")
    got = T.embedding(ids, weight)
    assert torch.equal(got[:5], weight[ids[:5]]) and not got[5].any()
    dy = torch.randn(6, D, device="cuda").to(BF)
    weight.fill_(1.0)
    T.topk_embedding_bwd(dy, ids, weight)
    assert torch.equal(weight[ids[:5]], dy[:5])
    weight[ids[:5]] = 0
    assert not any(part.any() for part in weight.split(500_000))
    T.topk_embedding_bwd(dy, ids, weight, accumulate=True)
    assert torch.equal(weight[ids[:5]], dy[:5])
    T.topk_check()


def test_logprobs():
    N, V = 17_000, 131_072  # 2.23e9 elements
    x = torch.zeros(N, V, dtype=BF, device="cuda")
    x[-2:].normal_(std=3)
    targets = torch.full((N,), V - 1, device="cuda")
    whole, part = T.token_logprobs(x, targets, top=6), T.token_logprobs(x[-2:].clone(), targets[-2:], top=6)
    # sums of 131,072 numbers in fp32 in different orders, a thread's of at most 512 and then a tree of 17 joins
    for name in ("logp", "entropy", "lse", "top_logp"):
        w, p = getattr(whole, name)[-2:], getattr(part, name)
        assert bool(((w - p).abs() <= 600 * 2.0 ** -23 * p.abs().clamp_min(16)).all()), name
    assert torch.equal(whole.top_ids[-2:], part.top_ids)
    g = torch.ones(N, device="cuda")
    want = T.token_logprobs_bwd(x[-2:].clone(), whole.lse[-2:].clone(), targets=targets[-2:], dlogp=g[-2:])
    out = T.token_logprobs_bwd(x, whole.lse, targets=targets, dlogp=g, out=x)
    assert out.data_ptr() == x.data_ptr() and torch.equal(out[-2:], want)
    T.topk_check()


def test_attention():
    cap, d = 18_000_000, 64
    cache = torch.empty(2, 1, cap, d, dtype=BF, device="cuda")  # 2.3e9 elements
    cache[1, 0, :300].normal_(), cache[0, 0, :6].normal_(), cache[1, 0, -400:].normal_()
    q = torch.randn(2, 4, 1, d, device="cuda").mul(d ** -0.5).to(BF)
    lens = torch.tensor([5, 299], dtype=torch.int32, device="cuda")
    got = T.tree_attention(q, cache, cache, lens)
    assert torch.equal(got, T.tree_attention(q, *(cache[:, :, :300].contiguous(),) * 2, lens))
    # the same memory as one row of keys, a prompt's at its end
    keys = cache.view(2 * cap, 1, d)
    p = torch.randn(70, 4, d, device="cuda").mul(d ** -0.5).to(BF)
    starts, at = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 70], [2 * cap - 400, 2 * cap]))
    near = torch.tensor([0, 400], dtype=torch.int32, device="cuda")
    got = T.prompt_attention(p, keys, keys, starts, at)
    assert torch.equal(got, T.prompt_attention(p, *(keys[-400:].clone(),) * 2, starts, near))
    T.topk_check()
