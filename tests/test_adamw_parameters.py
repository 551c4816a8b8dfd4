"""optim.AdamW.step looks at its parameters every time, before the library is called (no GPU needed)."""
import pytest
import torch

from paper_2106_06899_gb300 import build, optim


@pytest.fixture
def adamw():
    build.build_library()

    def make(p, **kw):
        opt = optim.AdamW([p], **kw)

        def called(*_):
            raise AssertionError("the library was called")

        opt._step = called
        return opt

    return make


def test_adamw_refuses_host_parameters(adamw):
    for kw in ({}, dict(state_bits=8)):
        p = torch.zeros(8, 4)
        with pytest.raises(ValueError, match="CUDA"):
            adamw(p, **kw).step([torch.zeros(8, 4)])
    p = torch.zeros(8, 4, dtype=torch.bfloat16)
    opt = adamw(p, masters=True)
    with pytest.raises(ValueError, match="CUDA"):
        opt.step([torch.zeros(8, 4, dtype=torch.bfloat16)])
    assert opt.state["step"] == 0


@pytest.mark.parametrize("change", [
    lambda t: t.bfloat16(), lambda t: t.double(), lambda t: t[:5], lambda t: torch.zeros(0), lambda t: t.t(),
    lambda t: torch.cat((t, t))])
def test_adamw_refuses_parameters_that_are_not_what_they_were(adamw, change):
    p = torch.nn.Parameter(torch.zeros(8, 4))
    opt = adamw(p)
    p.data = change(p.data)
    with pytest.raises(ValueError, match="parameters are no longer"):
        opt.step([torch.zeros(8, 4)])
    assert opt.state["step"] == 0
