"""A step that a non-finite gradient scale voids, taken back, leaves no trace."""
import pytest
import torch

from paper_2106_06899_gb300 import optim

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_a_void_step_taken_back(bits):
    g = torch.Generator("cuda").manual_seed(1)
    p0 = torch.randn(5000, device="cuda", generator=g).bfloat16()
    grads = [torch.randn(5000, device="cuda", generator=g).bfloat16() for _ in range(3)]
    one, bad = torch.ones((), device="cuda"), torch.full((), float("inf"), device="cuda")
    runs = []
    for void in (False, True):
        p = p0.clone()
        opt = optim.AdamW([p], lr=1e-2, state_bits=bits, seed=3)
        for x in grads:
            if void:
                opt.step([x], grad_scale=bad)
                opt.state["step"] -= 1
            opt.step([x], grad_scale=one)
        runs.append([p, *opt.moments(0)])
        assert opt.state["step"] == 3
    assert all(torch.equal(a, b) for a, b in zip(*runs))
