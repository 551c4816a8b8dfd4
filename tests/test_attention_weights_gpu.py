"""The weights' precision does not depend on how much a call holds: every prompt, whatever it is packed with, and every number of drafted
tokens is held against 64 bits with weights within 2^-16 (tests/_attention.py has the tolerances)."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from tests.test_prompt_attention_gpu import _edges, _verify
from tests.test_prompt_attention_gpu import _inputs as _prompt_inputs
from tests.test_tree_attention_gpu import _inputs as _tree_inputs
from tests.test_tree_attention_gpu import _parents, _reads
from tests.test_tree_attention_gpu import _verify as _verify_tree

pytestmark = pytest.mark.gpu
FINE = 2.0 ** -16


@pytest.mark.parametrize("lens,Hq,Hkv,rest", [([40, 3, 0, 61], 16, 4, 1000), ([1], 4, 1, 3000), ([700, 33, 1500], 16, 4, 0), ([4100], 4, 2, 0)], ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sharp", [0.02, 1.0, 4.0])
@pytest.mark.parametrize("causal", [True, False])
def test_prompts_of_many_rows(lens, Hq, Hkv, rest, d, sharp, causal):
    # as many rows as a large batch has, of other sequences or of none
    q, k, v = _prompt_inputs(lens, lens, Hq, Hkv, d, seed=sum(lens), rest=rest, scale=1.5 * sharp)
    got = T.prompt_attention(q, k, v, _edges(lens), causal=causal)
    T.topk_check()
    _verify(got, q, k, v, lens, lens, causal, heads=range(0, Hq, 3), weight=FINE)


@pytest.mark.parametrize("lq,lk", [([300, 9, 700], [3000, 9, 1400])], ids=str)
@pytest.mark.parametrize("d", [64, 128])
def test_prompts_that_go_on(lq, lk, d):
    q, k, v = _prompt_inputs(lq, lk, 16, 4, d, seed=11)
    got = T.prompt_attention(q, k, v, _edges(lq), _edges(lk))
    T.topk_check()
    _verify(got, q, k, v, lq, lk, True, heads=range(0, 16, 3), weight=FINE)


@pytest.mark.parametrize("B,Hq,Hkv,n,cap,lens", [(2, 8, 2, 64, 1500, [64, 1436]), (1, 64, 1, 5, 300, [200]), (3, 40, 8, 33, 900, [0, 867, 130]), (1, 128, 1, 64, 260, [126])],
                         ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sharp", [0.02, 1.0, 4.0])
def test_trees_of_many_rows(B, Hq, Hkv, n, cap, lens, d, sharp):
    q, keys, values = _tree_inputs(B, Hq, Hkv, n, cap, d, seed=cap)
    q = (q.float() * sharp).to(q.dtype)
    parents = _parents(B, n, seed=n)
    got = T.tree_attention(q, keys, values, torch.tensor(lens, dtype=torch.int32, device="cuda"), tree=T.tree_mask(parents.cuda()))
    T.topk_check()
    _verify_tree(got, q, keys, values, lens, _reads(parents), cap, weight=FINE)
