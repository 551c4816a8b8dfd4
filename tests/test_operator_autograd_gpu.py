"""What autograd is told of the library's calls: in-place changes are counted, for tensors that a graph may hold."""
import pytest
import torch

from paper_2106_06899_gb300 import optim
from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,masters", [(32, None), (8, None), (32, True)])
def test_a_graph_kept_over_an_optimizer_step_is_refused(bits, masters):
    w = torch.randn(64, device="cuda", dtype=torch.bfloat16 if masters else torch.float32).requires_grad_()
    idle = torch.randn(64, device="cuda", dtype=w.dtype).requires_grad_()
    opt = optim.AdamW([w, idle], state_bits=bits, masters=masters)
    loss, other = w.float().square().sum() + (w * w).float().sum(), (idle * idle).float().sum()
    w.grad = torch.ones_like(w)
    opt.step()
    with pytest.raises(RuntimeError, match="inplace"):
        loss.backward()
    other.backward()  # a parameter without a gradient was left alone


def test_a_graph_kept_over_a_cache_write_is_refused():
    q = torch.randn(1, 1, 2, 64, device="cuda")
    cos, sin = T.rope_tables(8, 64)
    keys, values = (torch.randn(1, 2, 8, 64, device="cuda") for _ in range(2))
    scale = torch.ones((), device="cuda", requires_grad=True)
    uses = [(scale * c).sum() for c in (keys, values)]
    T.qk_norm_rope(q, q, q, cos, sin, cache=(keys, values), cache_start=torch.tensor([3], dtype=torch.int32, device="cuda"))
    for loss in uses:
        with pytest.raises(RuntimeError, match="inplace"):
            loss.backward()


def test_outputs_that_a_caller_hands_over_are_counted():
    x, w = (torch.randn(16, 16, device="cuda").bfloat16() for _ in range(2))
    y, z, dx, dw, db = (torch.zeros(*s, device="cuda", dtype=torch.bfloat16) for s in ((16, 16), (16, 16), (16, 16), (16, 16), (16,)))
    T.topk_linear_fwd(x, w, y, preact=z)
    T.topk_linear_bwd(y, x, w, dx, dw, db)
    assert [t._version for t in (y, z, dx, dw, db)] == [1] * 5 and x._version == w._version == 0


def test_caches_made_in_inference_mode_are_written():
    with torch.inference_mode():
        q = torch.randn(1, 1, 2, 64, device="cuda")
        cos, sin = T.rope_tables(8, 64)
        keys, values = (torch.zeros(1, 2, 8, 64, device="cuda") for _ in range(2))
        T.qk_norm_rope(q, q, q, cos, sin, cache=(keys, values), cache_start=torch.tensor([3], dtype=torch.int32, device="cuda"))
        T.topk_check()
        assert torch.equal(values[0, :, 3], q[0, 0])
