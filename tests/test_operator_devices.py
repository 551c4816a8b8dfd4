"""The operators around the attention refuse tensors that are not on the GPU, before the library is called (no GPU needed)."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

BF = torch.bfloat16


@pytest.fixture
def no_library(monkeypatch):
    def called(*_):
        raise AssertionError("the library was called")

    monkeypatch.setattr(T, "lib", called)


def _bf(*shape):
    return torch.zeros(*shape, dtype=BF)


def test_linear_refuses_host_tensors(no_library):
    x, w, z = _bf(4, 16), _bf(8, 16), _bf(4, 8)
    with pytest.raises(ValueError, match="CUDA"):
        T.linear(x, w, _bf(8), "gelu", z, True)
    with pytest.raises(ValueError, match="CUDA"):
        T.linear_bwd(z, x, w, z, "gelu", bias=True)


def test_qk_norm_rope_refuses_host_tensors(no_library):
    q = _bf(1, 8, 2, 64)
    cos, sin = T.rope_tables(8, 64, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        T.qk_norm_rope(q, q, q, cos, sin)
    with pytest.raises(ValueError, match="CUDA"):
        T.qk_norm_rope(q, q, q, cos, sin, cache=(_bf(1, 2, 9, 64),) * 2, cache_start=torch.zeros(1, dtype=torch.int32))
    g = _bf(1, 2, 8, 64)
    with pytest.raises(ValueError, match="CUDA"):
        T.qk_norm_rope_bwd(g, g, g, q, q, cos, sin)
