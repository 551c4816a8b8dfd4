"""Which keys drafted tokens keep with top-k attention, against 64 bits over the cache's rows and each token's ancestors."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from tests._attention import attend
from tests.test_token_serving_gpu import D, H, V, _filled, _model
from tests.test_tree_attention_gpu import _parents, _reads

pytestmark = pytest.mark.gpu
F64 = torch.float64


@pytest.mark.parametrize("topk,n,start", [(8, 7, [0, 40]), (24, 16, [100, 3]), (3, 1, [50, 2]), (64, 33, [200, 70])], ids=str)
def test_drafted_tokens_keep_the_best_of_what_they_read(monkeypatch, topk, n, start):
    m = _model(topk, layers=1)
    caches = _filled(m, 2, 256)
    calls, attention = [], T.attention

    def spy(q, keys, values, k, mask=None, **kw):
        out, idx, score = attention(q, keys, values, k, mask=mask, return_indices=True, **kw)
        calls.append((q, k, idx, out))
        return out

    monkeypatch.setattr(T, "attention", spy)
    parents = _parents(2, n, seed=n)
    lens = torch.tensor(start, dtype=torch.int32, device="cuda")
    m.step_tree(torch.randint(0, V, (2, n), device="cuda"), caches, lens, tree=T.tree_mask(parents.cuda()))
    T.topk_check()
    ((q, k, idx, out),), ((keys, values),) = calls, caches
    assert k == topk
    reads, far = _reads(parents), 0
    for b, s in enumerate(start):
        ok = torch.zeros(n, 256, dtype=torch.bool, device="cuda")
        ok[:, :s] = True
        ok[:, s:s + n] = reads[b]
        for h in range(H):
            scores = (q[b, h].to(F64) @ keys[b, h].to(F64).t()).masked_fill(~ok, -torch.inf)
            best, at = scores.sort(dim=1, descending=True, stable=True)
            # fp32 sums of d products (tests/_attention.py): nearer scores than twice their error may go either way
            off = (D // H / 16 + 32) * 2.0 ** -23 * (q[b, h].to(F64).abs() @ keys[b, h].to(F64).abs().t()).amax(1)
            for i in range(n):
                valid = int(ok[i].sum())
                kept = idx[b, h, i][idx[b, h, i] >= 0].long()
                assert len(kept) == min(topk, valid) and bool(ok[i, kept].all())
                if valid <= topk or best[i, topk - 1] - best[i, topk] > 2 * off[i]:
                    far += 1
                    assert set(kept.tolist()) == set(at[i, :min(topk, valid)].tolist())
                mine = torch.zeros(1, 256, dtype=torch.bool, device="cuda")
                mine[0, kept] = True
                want, tol = attend(q[b, h, i:i + 1], keys[b, h], values[b, h], mine)
                assert bool(((out[b, h, i].to(F64) - want[0]).abs() <= tol[0]).all())
    assert far >= 0.95 * 2 * H * n
