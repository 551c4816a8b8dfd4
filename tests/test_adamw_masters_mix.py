"""topk_adamw_step: all tensors or none have a master, wherever empty ones stand (no GPU needed: refused before a launch)."""
import numpy as np
import pytest

from paper_2106_06899_gb300 import build, optim
from paper_2106_06899_gb300 import topk as T


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return T.lib()


def _step(lib, tensors, bits=8):
    """tensors: (elements, has a master)"""
    t = np.zeros(len(tensors), optim._TENSOR)
    for k in ("param", "grad", "m", "v", "m_scale", "v_scale"):
        t[k] = 16
    t["n"] = [n for n, _ in tensors]
    t["master"] = [16 if m else 0 for _, m in tensors]
    t["lr"] = 1e-3
    return lib.topk_adamw_step(t.ctypes.data, len(t), T.TOPK_BF16, T.TOPK_BF16, bits, 0.9, 0.999, 1e-8, 1, None, 0, None)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("tensors", [
    [(8, True), (8, False)], [(8, False), (8, True)],
    [(0, True), (8, True), (8, False)], [(0, True), (8, False), (8, True)],
    [(0, False), (8, True), (8, False)], [(0, False), (8, False), (8, True)],
    [(0, False), (0, True), (8, True), (0, False), (8, False)],
], ids=str)
def test_a_mix_is_refused(lib, bits, tensors):
    assert _step(lib, tensors, bits) == -1


def test_an_empty_tensors_master_does_not_count(lib):
    # no device here: a list that passes every check is answered with TOPK_ERR_NO_DEVICE
    import torch

    if torch.cuda.is_available():
        pytest.skip("the addresses are not real: host checks only")
    for tensors in ([(0, True), (8, False)], [(0, False), (8, True)], [(8, True), (0, False), (8, True)]):
        assert _step(lib, tensors) == -6
