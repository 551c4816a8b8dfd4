"""Sizes that a C int cannot hold are refused by the binding: ctypes would cut them off without a word (no GPU needed)."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

BF = torch.bfloat16


@pytest.fixture
def no_library(monkeypatch):
    def called(*_):
        raise AssertionError("the library was called")

    monkeypatch.setattr(T, "_on_gpu", lambda *a: None)
    monkeypatch.setattr(T, "lib", called)


def _meta(*shape, dtype=BF):
    return torch.empty(*shape, dtype=dtype, device="meta")


LONG = 2 ** 32 + 16


@pytest.mark.parametrize("M,K,N", [(LONG, 8, 8), (16, LONG, 8), (16, 8, LONG), (2 ** 31, 8, 8)])
def test_linear(no_library, M, K, N):
    x, w, y = _meta(M, K), _meta(N, K), _meta(M, N)
    with pytest.raises(ValueError, match="2\\^31"):
        T.topk_linear_fwd(x, w, y)
    with pytest.raises(ValueError, match="2\\^31"):
        T.topk_linear_bwd(y, x, w, x, w, None)


def test_cache_rows(no_library):
    q, cache = _meta(1, 1, 1, 8), _meta(1, 1, LONG, 8)
    cos = _meta(4, 4, dtype=torch.float32)
    with pytest.raises(ValueError, match="2\\^31"):
        T.topk_qk_norm_rope_fwd(q, q, q, cos, cos, _meta(1, 1, 1, 8), cache, cache, cache_start=_meta(1, dtype=torch.int32))
