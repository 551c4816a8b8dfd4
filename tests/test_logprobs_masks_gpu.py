"""Log probabilities of rows that mask tokens in two ways at once, by -inf and by a value near the type's lowest (tests/test_logprobs_gpu.py has
the tolerances)."""
import math

import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from tests.test_logprobs_gpu import _check_backward, _check_forward

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
INF = math.inf


def _rows(V, dtype, fill, real, seed):
    """Rows with `real` logits at the front, in the middle, at the end and anywhere; the others fill or -inf, by halves."""
    g = torch.Generator().manual_seed(seed)
    x = torch.where(torch.rand(4, V, generator=g) < 0.5, fill, -INF)
    for n, at in enumerate((torch.arange(real), V // 2 + torch.arange(real), V - 1 - torch.arange(real), torch.randperm(V, generator=g)[:real])):
        x[n, at] = torch.randn(real, generator=g) * 3
    return x.to(dtype).cuda()


# below -3.3e38, which is -248 2^120 in bf16, a floor 33 / 32 times as far is finite in 32 bits and -inf in bf16
@pytest.mark.parametrize("fill", [-3.3e38, -3.27e38, -3.31e38, torch.finfo(BF).min, torch.finfo(F32).min, -1e38, -1e30, -65504.0, -1e4], ids=str)
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
@pytest.mark.parametrize("V,top", [(300, 3), (40000, 0), (131072, 8)])
@pytest.mark.parametrize("scale", [1.0, 0.6])
def test_two_masks(fill, dtype, V, top, scale):
    if fill == torch.finfo(F32).min and dtype == BF:
        fill = torch.finfo(BF).min  # the other one rounds to -inf
    x = _rows(V, dtype, fill, 40, V)
    _check_forward(x, torch.tensor([3, V // 2 + 5, V - 2, -1], device="cuda"), top, scale)


@pytest.mark.parametrize("fill", [-3.3e38, torch.finfo(BF).min, -1e4], ids=str)
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_two_masks_many_rows(fill, dtype):
    x = _rows(9000, dtype, fill, 64, 1)
    r = _check_forward(x.repeat(160, 1), None, 5, 1.0)  # a block for each row
    assert torch.equal(r.entropy[:4].repeat(160), r.entropy)


@pytest.mark.parametrize("fill", [-3.3e38, torch.finfo(BF).min, -1e4], ids=str)
@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
@pytest.mark.parametrize("V", [300, 40000])
def test_nothing_but_masked_tokens(fill, dtype, V):
    # a fill is as likely as another where nothing else is there; the sum's logarithm is lost beside it, but not the entropy
    x = torch.where(torch.arange(V, device="cuda") % 3 == 0, fill, -INF)[None].to(dtype)
    n = V // 3 + (V % 3 > 0)
    r = T.token_logprobs(x, torch.zeros(1, dtype=torch.int64, device="cuda"), top=2)
    T.topk_check()
    c = (V / 256 + 80) * 2.0 ** -23 + 2.0 ** -20
    assert abs(float(r.entropy) - math.log(n)) <= c and abs(float(r.logp) + math.log(n)) <= c
    assert abs(float(r.lse) / float(x[0, 0]) - 1) <= 1e-3 and r.top_ids.tolist() == [[0, 3]]


@pytest.mark.parametrize("dtype", [BF, F32], ids=str)
def test_gradient_of_two_masks(dtype):
    x = _rows(9000, dtype, -3.3e38, 64, 2)
    _check_backward(x, torch.tensor([5, 4502, 8998, -1], device="cuda"), 3, True, 1.0)
