"""The linear layer on shapes that reach each way of cutting a product (152 SMs): 128 x 128 and 128 x 256 tiles of a CTA, 256 x 256
tiles of a pair, each whole and with its sum split.  References and tolerances are test_linear_gpu.py's."""
import pytest
import torch

from tests import test_linear_gpu as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,K,N", [
    (1859, 64, 2392), (2572, 320, 1600),    # 128 x 256
    (139, 1552, 1968),                      # 256 x 256, the sum in five parts
    (66, 1152, 128), (257, 2048, 520),      # 128 x 128, in four and eight
    (4888, 72, 400),                        # 256 x 256
])
@pytest.mark.parametrize("act,bias,res,keep", [("none", False, False, False), ("relu", True, True, True), ("gelu", True, True, False), ("silu", False, True, False),
                                               ("silu", True, False, True)])
def test_forward(M, K, N, act, bias, res, keep):
    base._forward(M, K, N, act, bias, res, keep, seed=M + N)


@pytest.mark.parametrize("M,K,N", [
    (3180, 1488, 72),   # dx: 128 x 256
    (2267, 136, 1544),  # dx: 256 x 256 in five parts; dW: 256 x 256 in six
    (80, 1888, 2320),   # dW: 128 x 256
    (3474, 264, 2360),  # dW: 128 x 256 in four
])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("grad", [torch.bfloat16, torch.float32])
def test_backward(M, K, N, act, grad):
    base.test_backward(M, K, N, act, grad)
