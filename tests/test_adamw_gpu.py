"""AdamW over many tensors against the formulas in 64 bits.

Tolerances (u = 2^-24, the rounding of one fp32 operation).  m and v are two products and a sum: 4 u of
the magnitudes added, with the coefficients' own rounding.  p adds a root, a product, a sum, a
quotient, a product and a difference: 4 u of |p| and 16 u of the update.  What is rounded
stochastically lies on one of the two neighbours of the exact value (of a value moved by
those bounds), with a mean error of at most 2^-11 of a place (ten random bits, centred) and sampling noise.
"""
import math

import pytest
import torch

from paper_2106_06899_gb300 import optim
from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
F64 = torch.float64
U = 2.0 ** -24
SIZES = [1, 7, 8, 255, 256, 257, 2048, 2049, 10007, 70001, 3]
LR, WD, BETAS, EPS = 3e-3, 0.1, (0.9, 0.99), 1e-8


def _make(sizes, pdt, gdt, seed=0, offset=0):
    """Parameters and gradients as views `offset` elements into larger buffers."""
    g = torch.Generator().manual_seed(seed)

    def view(n, dt, scale):
        return (scale * torch.randn(n + offset, generator=g)).to(dt).cuda()[offset:]

    return [view(n, pdt, 0.5) for n in sizes], [view(n, gdt, 0.1) for n in sizes]


def _reference(p, m, v, g, step, lr=LR, wd=WD):
    """One step in 64 bits: (p, m, v) and the magnitudes that their roundings scale with."""
    b1, b2 = BETAS
    p, m, v, g = (x.to(F64) for x in (p, m, v, g))
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    upd = lr / (1 - b1 ** step) * m1 / ((v1 / (1 - b2 ** step)).sqrt() + EPS)
    mm = b1 * m.abs() + (1 - b1) * g.abs()
    um = lr / (1 - b1 ** step) * mm / ((v1 / (1 - b2 ** step)).sqrt() + EPS)
    return p * (1 - lr * wd) - upd, m1, v1, p.abs(), mm, v1, um


def _near(got, want, tol):
    err = (got.to(F64) - want).abs() / (tol + 1e-38)
    assert bool((err <= 1).all()), float(err.max())


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("gdt", [torch.float32, torch.bfloat16])
def test_fp32_parameters_32_bit_states(offset, gdt):
    ps, gs = _make(SIZES, torch.float32, gdt, 1, offset)
    opt = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD)
    for step in (1, 2, 3):
        before = [(p.clone(), *opt.moments(i)) for i, p in enumerate(ps)]
        opt.step(gs)
        T.topk_check()
        for i, (p, m, v) in enumerate(before):
            rp, rm, rv, pm, mm, vm, um = _reference(p, m, v, gs[i], step)
            m1, v1 = opt.moments(i)
            _near(m1, rm, 4 * U * mm)
            _near(v1, rv, 4 * U * vm)
            _near(ps[i], rp, 4 * U * pm + 16 * U * um)


def test_against_torch():
    # the same algorithm in PyTorch, fp32: twenty steps stay together to fp32 rounding (32 roundings a step)
    ps, _ = _make(SIZES, torch.float32, torch.float32, 2)
    qs = [p.clone().requires_grad_() for p in ps]
    a = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD)
    b = torch.optim.AdamW(qs, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD)
    for k in range(20):
        _, gs = _make(SIZES, torch.float32, torch.float32, 50 + k)
        a.step(gs)
        for q, g in zip(qs, gs):
            q.grad = g.clone()
        b.step()
    for p, q in zip(ps, qs):
        _near(p, q.detach().to(F64), 20 * 32 * U * (q.detach().abs().to(F64) + LR))


@pytest.mark.parametrize("bits", [32, 8])
def test_master_and_its_copy(bits):
    ps, gs = _make(SIZES, torch.bfloat16, torch.bfloat16, 3)
    opt = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD, state_bits=bits, masters=True)
    for step in (1, 2):
        before = [(x.clone(), *opt.moments(i)) for i, x in enumerate(opt.masters)]
        opt.step(gs)
        T.topk_check()
        for i, (p, m, v) in enumerate(before):
            rp, _, _, pm, _, _, um = _reference(p, m, v, gs[i], step)
            # 8-bit moments are products of a float and a scale, two more roundings, and v a square
            _near(opt.masters[i].view(-1), rp.view(-1), 4 * U * pm.view(-1) + 24 * U * um.view(-1))
            assert torch.equal(ps[i].view(-1), opt.masters[i].view(-1).to(torch.bfloat16))


def _place(x, bits):
    """The last place of a float of `bits` significand bits at x."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp_min(1e-300))) - (bits - 1))


def test_bf16_parameters_round_stochastically():
    n = 1 << 20
    ps, gs = _make([n], torch.bfloat16, torch.float32, 4)
    opt = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD, seed=7)
    p0 = ps[0].clone()
    opt.step(gs)
    want, _, _, pm, _, _, um = _reference(p0, torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), gs[0], 1)
    err = (ps[0].to(F64) - want) / _place(want, 8)
    slack = (4 * U * pm + 16 * U * um) / _place(want, 8)
    assert bool((err.abs() <= 1 + slack + 2.0 ** -12).all())
    # twelve random bits: a mean error of at most 2^-13 places, and noise of at most 1/2 per element
    assert abs(float(err.mean())) <= 2.0 ** -13 + 6 * 0.5 / math.sqrt(n)
    # what a rounding to nearest would lose moves the parameters: their mean change is the update's
    away = float((ps[0].to(F64) - p0.to(F64)).mean() - (want - p0.to(F64)).mean())
    assert abs(away) <= 6 * float((_place(want, 8) ** 2).mean().sqrt()) / math.sqrt(n) + float((2.0 ** -13 * _place(want, 8)).mean())


def _decoded(opt, name, n):
    s = opt.state
    return (s[name].float().view(-1, 256) * s[name + "_scale"][:, None]).view(-1)[:n]


@pytest.mark.parametrize("pdt", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("offset", [0, 1])
def test_8_bit_states(pdt, offset):
    sizes = [70001, 300, 1]
    ps, gs = _make(sizes, pdt, torch.float32, 5, offset)
    opt = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD, state_bits=8, seed=3)
    for step in (1, 2, 3):
        before = [(p.clone(), *opt.moments(i)) for i, p in enumerate(ps)]
        _, gs = _make(sizes, pdt, torch.float32, 5 + step, offset)
        opt.step(gs)
        T.topk_check()
        for i, (p, m, v) in enumerate(before):
            n = sizes[i]
            rp, rm, rv, pm, mm, vm, um = _reference(p, m, v, gs[i], step)
            if pdt == torch.float32:
                _near(ps[i], rp, 4 * U * pm + 24 * U * um)
            at = int(opt._table["index"][i])
            for name, want, slack in (("exp_avg", rm, 8 * U * mm), ("exp_avg_root", rv.sqrt(), 8 * U * rv.sqrt())):
                pad = torch.nn.functional.pad(want, (0, -n % 256)).view(-1, 256)
                scale = (pad.abs().amax(1) / 448).repeat_interleave(256)[:n]
                got_scale = opt.state[name + "_scale"][at // 256:at // 256 + pad.shape[0]]
                _near(got_scale, pad.abs().amax(1) / 448, 12 * U * pad.abs().amax(1) / 448)
                code = opt.state[name][at:at + n].float()
                y = want / scale
                place = _place(y.abs().clamp_min(2.0 ** -6), 4)
                err = (code.to(F64) - y) / place
                # a neighbour of the exact value; y's own error is of the sums, the scale and two products
                assert bool((err.abs() <= 1 + (slack / scale + 16 * U * y.abs()) / place + 2.0 ** -10).all()), float(err.abs().max())
                if n > 10000:
                    assert abs(float((err * torch.sign(y)).mean())) <= 2.0 ** -11 + 6 * 0.5 / math.sqrt(n)


def test_8_bit_moments_do_not_stall():
    # without gradients v decays by b2 a step, 1 % of a place or less: to the nearest it would never move.
    # After 64 steps the mean of the roots has fallen by b2^32; a block's values wander by less than a place
    # (1/8) each, independently: 1/8 sqrt(64) / sqrt(n) of the mean
    n = 1 << 18
    p = [torch.zeros(n, device="cuda")]
    opt = optim.AdamW(p, lr=0.0, betas=(0.9, 0.999), weight_decay=0.0, state_bits=8, seed=11)
    g = [1 + torch.rand(n, device="cuda", generator=torch.Generator("cuda").manual_seed(1))]
    opt.step(g)
    before = float(_decoded(opt, "exp_avg_root", n).double().mean())
    zero = [torch.zeros(n, device="cuda")]
    for _ in range(64):
        opt.step(zero)
    after = float(_decoded(opt, "exp_avg_root", n).double().mean())
    assert abs(after / before - 0.999 ** 32) <= 1.0 / math.sqrt(n) * 4 + 64 * 2.0 ** -14, (after / before, 0.999 ** 32)


def test_steps_repeat_and_seeds_differ():
    def once(seed, sizes=(5000, 300)):
        ps, gs = _make(list(sizes), torch.bfloat16, torch.bfloat16, 6)
        opt = optim.AdamW(ps, lr=LR, state_bits=8, seed=seed)
        for _ in range(3):
            opt.step(gs)
        return [p.clone() for p in ps] + [opt.state["exp_avg"].float(), opt.state["exp_avg_root_scale"]]

    a, b, c = once(1), once(1), once(2)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert not torch.equal(a[0], c[0]) and not torch.equal(a[2], c[2])


def test_alignment_does_not_change_results():
    outs = []
    for offset in (0, 1):
        ps, gs = _make([1000, 9000], torch.float32, torch.float32, 8, 0)
        if offset:
            ps, gs = ([torch.cat((x[:1], x))[1:] for x in xs] for xs in (ps, gs))
            assert ps[0].data_ptr() % 16 == 4
        opt = optim.AdamW(ps, lr=LR, state_bits=8, seed=1)
        opt.step(gs)
        outs.append([*ps, opt.state["exp_avg"].float()])
    assert all(torch.equal(x, y) for x, y in zip(*outs))


def test_more_tensors_than_a_launch_holds():
    sizes = [1 + 37 * k % 700 for k in range(800)]
    ps, gs = _make(sizes, torch.float32, torch.float32, 9)
    before = [p.clone() for p in ps]
    opt = optim.AdamW(ps, lr=LR, betas=BETAS, eps=EPS, weight_decay=WD)
    opt.step(gs)
    assert T.topk_last_launch_count() == 3
    for p, p0, g in zip(ps, before, gs):
        rp, _, _, pm, _, _, um = _reference(p0, torch.zeros_like(p0), torch.zeros_like(p0), g, 1)
        _near(p, rp, 4 * U * pm + 16 * U * um)


def test_groups_missing_gradients_and_empty_tensors():
    ps, gs = _make([300, 400, 500, 0], torch.float32, torch.float32, 10)
    before = [p.clone() for p in ps]
    opt = optim.AdamW([{"params": ps[:2], "weight_decay": 0.0}, {"params": ps[2:], "lr": 0.5}], lr=LR, betas=BETAS, eps=EPS, weight_decay=WD)
    for p, g in zip(ps, gs):
        p.grad = g
    ps[1].grad = None
    opt.step()
    for i, (lr, wd) in ((0, (LR, 0.0)), (2, (0.5, WD))):
        rp, _, _, pm, _, _, um = _reference(before[i], torch.zeros_like(before[i]), torch.zeros_like(before[i]), gs[i], 1, lr, wd)
        _near(ps[i], rp, 4 * U * pm + 16 * U * um)
    assert torch.equal(ps[1], before[1]) and float(opt.moments(1)[0].abs().max()) == 0
    opt.zero_grad()
    assert ps[0].grad is None
    opt.step()  # nothing to do: not a step
    assert opt.state["step"] == 1


def test_gradient_scale_and_skipped_step():
    a, ga = _make([5000], torch.float32, torch.float32, 12)
    b, gb = _make([5000], torch.float32, torch.float32, 12)
    oa, ob = optim.AdamW(a, lr=LR), optim.AdamW(b, lr=LR)
    oa.step([0.25 * ga[0]])
    ob.step(gb, grad_scale=torch.tensor(0.25, device="cuda"))
    assert torch.equal(a[0], b[0])  # a power of two: the same bits
    for bad in (float("inf"), float("nan")):
        ob.step(gb, grad_scale=torch.tensor(bad, device="cuda"))
    assert torch.equal(a[0], b[0]) and torch.equal(oa.moments(0)[1], ob.moments(0)[1])


def test_nonfinite_gradients_stay_where_they_are():
    for bits, reach in ((32, 1), (8, 256)):
        ps, gs = _make([2000], torch.float32, torch.float32, 13)
        gs[0][700] = float("nan")
        gs[0][1500] = float("inf")
        opt = optim.AdamW(ps, lr=LR, state_bits=bits)
        opt.step(gs)
        assert torch.nonzero(~torch.isfinite(ps[0])).view(-1).tolist() == [700, 1500]
        bad = torch.nonzero(~torch.isfinite(opt.moments(0)[0])).view(-1)
        blocks = set((bad // reach).tolist())
        assert {700 // reach, 1500 // reach} == blocks


def test_zero_blocks_and_wide_ranges():
    # a block of zeros stays zeros; magnitudes over 2^30 in one block: the small ones go to zero or their place
    g = torch.zeros(1024, device="cuda")
    g[256:512] = 2.0 ** torch.linspace(-30, 0, 256, device="cuda")
    g[512:768] = 1e-42  # below the smallest block that is held
    p = [torch.zeros(1024, device="cuda")]
    opt = optim.AdamW(p, lr=LR, state_bits=8)
    opt.step([g])
    m, v = opt.moments(0)
    assert float(m[:256].abs().max()) == 0 and float(m[512:].abs().max()) == 0 and torch.isfinite(p[0]).all()
    assert float(opt.state["exp_avg_scale"][2]) == 0
    err = (m[256:512] - 0.1 * g[256:512]).abs() / (0.1 * g[256:512] / 8 + 0.1 / 448 * 2.0 ** -9)
    assert float(err.max()) <= 1.001


def test_stream_and_state_dict():
    ps, gs = _make([3000, 40], torch.bfloat16, torch.bfloat16, 14)
    qs = [p.clone() for p in ps]
    a = optim.AdamW(ps, lr=LR, state_bits=8, seed=5, masters=True)
    a.step(gs)
    torch.cuda.synchronize()
    b = optim.AdamW(qs, lr=1.0, state_bits=8, seed=9, masters=True)
    b.load_state_dict(a.state_dict())
    for q, p in zip(qs, ps):
        q.copy_(p)
    a.step(gs)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    b.step(gs, stream=st)
    st.synchronize()
    T.topk_check()
    assert all(torch.equal(p, q) for p, q in zip(ps, qs)) and all(torch.equal(p, q) for p, q in zip(a.masters, b.masters))
    # buffers handed over are used as they are
    c = optim.AdamW(qs, lr=LR, state_bits=8, seed=5, masters=b.masters, state=b.state)
    assert c.state["exp_avg"].data_ptr() == b.state["exp_avg"].data_ptr() and c.state["step"] == 2
