"""Alternatives of large vocabularies whose likely tokens lie anywhere, so that more elements than a block notes reach its first tile's threshold and
the row is read again; and of rows that begin with masked tokens (tests/test_logprobs_gpu.py has the tolerances)."""
import math

import pytest
import torch

from tests.test_logprobs_gpu import _check_forward

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("kind", ["anywhere", "masked front", "common last"])
@pytest.mark.parametrize("N,V,top,dtype", [(320, 131072, 64, F32), (320, 131072, 128, BF), (310, 262147, 64, BF), (320, 50001, 128, F32), (3, 262147, 128, F32)], ids=str)
def test_large_vocabularies(kind, N, V, top, dtype):
    g = torch.Generator(device="cuda").manual_seed(V + top)
    x = torch.randn(N, V, generator=g, device="cuda") * 3
    if kind == "masked front":
        x[:, :9000] = -math.inf
    elif kind == "common last":
        x -= 0.5 * torch.log1p(torch.arange(V, device="cuda")).flip(0)
    x = x.to(dtype)
    t = torch.randint(9000, V, (N,), generator=g, device="cuda")
    _check_forward(x, t, top, 1.0)
    _check_forward(x, None, 0, 1.0)
