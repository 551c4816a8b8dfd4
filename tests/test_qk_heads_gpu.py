"""Query/key norm with more heads than a launch has groups, one row a lane."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
D, ROT = 136, 64  # 17 lanes: a head to a warp


def _inputs(Hq, Hkv, dtype):
    g = torch.Generator("cuda").manual_seed(1)
    qkv = torch.randn(1, 2, Hq + 2 * Hkv, D, device="cuda", generator=g).to(dtype)
    w = (1 + 0.2 * torch.randn(D, device="cuda", generator=g)).to(dtype)
    return qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:], w, *T.rope_tables(2, ROT)


@pytest.mark.parametrize("dtype,Hq,Hkv", [(torch.bfloat16, 65536, 65536), (torch.float32, 60000, 30000)])
def test_forward(dtype, Hq, Hkv):
    # a head's row is computed by itself: the same bits as in calls of few heads
    q, k, v, w, cos, sin = _inputs(Hq, Hkv, dtype)
    got = T.qk_norm_rope(q, k, v, cos, sin, q_weight=w, k_weight=w, q_scale=0.5)
    T.topk_check()
    for h in (0, 9000, Hkv - 64):
        at = slice(h, h + 64)
        want = T.qk_norm_rope(q[:, :, at], k[:, :, at], v[:, :, at], cos, sin, q_weight=w, k_weight=w, q_scale=0.5)
        assert all(torch.equal(a[:, at], b) for a, b in zip(got, want))


def test_backward():
    Hq, Hkv = 60000, 5000
    q, k, v, w, cos, sin = _inputs(Hq, Hkv, torch.bfloat16)
    dq, dk, dv = (torch.randn(1, h, 2, D, device="cuda") for h in (Hq, Hkv, Hkv))
    opts = dict(q_weight=w, k_weight=w, q_scale=0.5)
    packed, gq, gk = T.qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, **opts)
    T.topk_check()
    total = torch.zeros(D, dtype=torch.float64, device="cuda")
    magnitude = total.clone()
    for h in range(0, Hq, 2500):
        at, kat = slice(h, h + 2500), slice(0, 2500)
        p, a, _ = T.qk_norm_rope_bwd(dq[:, at].contiguous(), dk[:, kat].contiguous(), dv[:, kat].contiguous(), q[:, :, at], k[:, :, kat], cos, sin, **opts)
        assert torch.equal(packed[:, :, at], p[:, :, :2500])
        total += a.double()
        # terms of a sum: |g| |x| r, of which x r has a mean square of 1
        magnitude += dq[:, at].double().abs().sum((0, 1, 2)) * 0.5
    # sums of 120,000 terms in fp32, in chains of at most 2,000 and trees: 2,000 units of their magnitude, with a margin of 4
    # for |x r| beyond 1 and the turned gradients
    assert bool(((gq.double() - total).abs() <= 4 * 2000 * 2.0 ** -24 * magnitude).all())


def test_more_than_a_launch_holds_is_refused():
    q, k, v, w, cos, sin = _inputs(40000, 20000, torch.bfloat16)
    pos = torch.zeros(3, 1, 2, dtype=torch.int32, device="cuda")
    opts = dict(positions=pos, sections=(30, 1, 1), q_weight=w, k_weight=w)  # narrow axes: one row a lane
    with pytest.raises(T.TopkError) as e:
        T.qk_norm_rope(q, k, v, cos, sin, **opts)
    assert e.value.code == -2
    g = [torch.zeros(1, h, 2, D, device="cuda", dtype=torch.bfloat16) for h in (40000, 20000, 20000)]
    with pytest.raises(T.TopkError) as e:
        T.qk_norm_rope_bwd(*g, q, k, cos, sin, **opts)
    assert e.value.code == -2
    T.topk_check()
