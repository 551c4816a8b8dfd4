"""Scratch of the embedding's gradient is what its documentation says (no GPU needed)."""
import pytest

from paper_2106_06899_gb300 import build
from paper_2106_06899_gb300 import topk as T


@pytest.mark.parametrize("N", [1, 127, 128, 129, 1024, 8193, 1 << 15, 100_003])
@pytest.mark.parametrize("D", [1, 768, 1001])
def test_embedding_gradient(N, D):
    # 16 bytes for each id, each half of them in whole 256 bytes, and two rows of 32-bit sums for every 128 ids
    build.build_library()
    half = (8 * N + 255) // 256 * 256
    want = 2 * half + (N + 127) // 128 * 2 * D * 4
    assert T.topk_embedding_bwd_workspace_bytes(N, 5, D) == T.topk_embedding_bwd_workspace_bytes(N, 1 << 20, D) == want
