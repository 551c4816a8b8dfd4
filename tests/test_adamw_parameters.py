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


def test_adamw_refuses_buffers_that_are_not_the_ones_it_writes(adamw):
    # the kernel writes to the addresses of the buffers that the optimizer was made with
    def replaced(opt, p):
        with pytest.raises(ValueError, match="replaced"):
            opt.step([torch.zeros_like(p)])

    for bits, names in ((32, ("exp_avg", "exp_avg_sq")), (8, ("exp_avg", "exp_avg_scale", "exp_avg_root", "exp_avg_root_scale"))):
        for name in names:
            p = torch.zeros(8, 4)
            opt = adamw(p, state_bits=bits)
            opt.state[name] = opt.state[name].clone()
            replaced(opt, p)
    opt = adamw(torch.zeros(8, 4))
    opt.state = {"note": 1, **dict(reversed(opt.state.items()))}
    with pytest.raises(ValueError, match="CUDA"):  # the same buffers
        opt.step([torch.zeros(8, 4)])
    p = torch.zeros(8, 4, dtype=torch.bfloat16)
    opt = adamw(p, masters=True)
    opt.masters[0] = opt.masters[0].clone()
    replaced(opt, p)
    opt = adamw(p, masters=True)
    opt.masters = None
    replaced(opt, p)
