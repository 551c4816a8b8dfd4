"""The library's autograd functions, with stand-ins for the library's calls on the CPU (no GPU needed)."""
import pytest
import torch

from paper_2106_06899_gb300 import decoder


def _act(z, act):
    return {"none": lambda: z, "relu": lambda: z.relu(), "gelu": lambda: torch.nn.functional.gelu(z), "silu": lambda: torch.nn.functional.silu(z)}[act]()


class _StandIn:
    """linear, qk_norm_rope, attention and ffn with their gradients, as torch operations that leave no graph."""

    def __init__(self):
        self.calls = []

    def linear(self, x, w, bias=None, act="none", residual=None, return_preact=False, stream=None):
        self.calls.append(("linear", return_preact))
        with torch.no_grad():
            z = x @ w.t()
            y = _act(z, act) + (0 if residual is None else residual)
        return (y, z) if return_preact else y

    def linear_bwd(self, dy, x, w, preact=None, act="none", bias=False, need_dx=True, need_dw=True, grad_dtype=None, stream=None):
        assert need_dx or need_dw, "the library refuses a call that asks for nothing"
        assert (preact is None) == (act == "none")
        self.calls.append(("linear_bwd", need_dx, need_dw))
        with torch.enable_grad():
            z = (torch.zeros_like(dy) if preact is None else preact).detach().clone().requires_grad_()
            (dz,) = torch.autograd.grad(_act(z, act), z, dy.detach())
        return (dz @ w).detach() if need_dx else None, (dz.t() @ x).detach() if need_dw else None, None

    def qk_norm_rope(self, q, k, v, cos, sin, q_weight=None, k_weight=None, q_scale=1.0):
        self.calls.append(("qk_norm_rope",))
        with torch.no_grad():
            return tuple(t.transpose(1, 2).contiguous() for t in (q * q_weight * q_scale, k * k_weight, v))

    def qk_norm_rope_bwd(self, dq, dk, dv, q, k, cos, sin, q_weight=None, k_weight=None, q_scale=1.0):
        self.calls.append(("qk_norm_rope_bwd",))
        with torch.no_grad():
            dq, dk, dv = (t.transpose(1, 2).to(q.dtype) for t in (dq, dk, dv))
            return (torch.cat((dq * q_weight * q_scale, dk * k_weight, dv), 2), (dq * q * q_scale).sum((0, 1, 2)), (dk * k).sum((0, 1, 2)))

    def attention(self, q, k, v, topk, causal=False, return_indices=False):
        with torch.no_grad():
            out = q * k * v
        return out, torch.zeros(1, dtype=torch.int32), torch.zeros(1)

    def attention_bwd(self, q, k, v, dout, idx, score):
        with torch.no_grad():
            return dout * k * v, dout * q * v, dout * q * k

    def ffn(self, x, w1, w2, topk, return_indices=False):
        with torch.no_grad():
            return (x @ w1.t()) @ w2, torch.zeros(1, dtype=torch.int32), torch.zeros(1)

    def ffn_bwd(self, x, w1, w2, dout, idx, score):
        with torch.no_grad():
            return (dout @ w2.t()) @ w1, (dout @ w2.t()).t() @ x, (x @ w1.t()).t() @ dout


@pytest.fixture
def stand_in(monkeypatch):
    s = _StandIn()
    monkeypatch.setattr(decoder, "T", s)
    return s


def _rand(*shape):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(sum(shape))).requires_grad_()


def _cases():
    qkv, w, tables = _rand(1, 4, 6, 8), _rand(8), (torch.zeros(4, 4), torch.zeros(4, 4))
    q, x, wx, w1, w2 = _rand(1, 2, 4, 8), _rand(4, 8), _rand(6, 8), _rand(16, 8), _rand(16, 8)
    return {
        "linear": (x, lambda: decoder.LinearFunction.apply(x, wx, "none", None)),
        "linear with an activation and a residual": (x, lambda: decoder.LinearFunction.apply(x, wx, "silu", x[:, :6])),
        "norms, rotation and attention": (qkv, lambda: decoder.RotaryAttentionFunction.apply(qkv, w, w, *tables, 4)),
        "norms and rotation": (qkv, lambda: torch.cat(decoder.QKNormRopeFunction.apply(qkv, w, w, *tables))),
        "attention": (q, lambda: decoder.TopKAttentionFunction.apply(q, q, q, 4, True)),
        "feed-forward": (x, lambda: decoder.TopKFFNFunction.apply(x, w1, w2, 4)),
    }


NAMES = ["linear", "linear with an activation and a residual", "norms, rotation and attention", "norms and rotation", "attention", "feed-forward"]


@pytest.mark.parametrize("name", NAMES)
def test_second_derivatives_are_refused(stand_in, name):
    # the gradient of a gradient would be that of the torch operations around alone: an error, not a part of it
    x, run = _cases()[name]
    (g,) = torch.autograd.grad(run().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        g.square().sum().backward()


@pytest.mark.parametrize("name", NAMES)
def test_first_derivatives_are_the_same_with_create_graph(stand_in, name):
    x, run = _cases()[name]
    (a,) = torch.autograd.grad(run().square().sum(), x)
    (b,) = torch.autograd.grad(run().square().sum(), x, create_graph=True)
    assert torch.equal(a, b) and float(a.abs().max()) > 0


def test_a_linear_layer_of_frozen_inputs_passes_the_residuals_gradient(stand_in):
    x, w, r = _rand(4, 8).detach(), _rand(6, 8).detach(), _rand(4, 6)
    for act in ("none", "gelu"):
        (g,) = torch.autograd.grad(decoder.LinearFunction.apply(x, w, act, r).square().sum(), r)
        y = decoder.LinearFunction.apply(x, w, act, r).detach()
        assert torch.equal(g, 2 * y)


def _held(fn):
    """The bytes that the graph of fn's result holds, each storage once."""
    seen = {}

    def pack(t):
        seen[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
        return t

    with torch.autograd.graph.saved_tensors_hooks(pack, lambda t: t):
        out = fn()
    return out, seen


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("residual", [False, True])
def test_linear_keeps_pre_activations_only_where_they_are_needed(stand_in, act, residual):
    x, w = _rand(4, 8), _rand(6, 8)
    r = _rand(4, 6).detach() if residual else None
    y, held = _held(lambda: decoder.LinearFunction.apply(x, w, act, r))
    # ReLU's slope is its output's sign, unless a residual was added to it
    needs = act in ("gelu", "silu") or (act == "relu" and residual)
    assert stand_in.calls[-1] == ("linear", needs)
    more = {k for k in held if k not in (x.data_ptr(), w.data_ptr())}
    assert len(more) == (act != "none") and (not more or needs or more == {y.data_ptr()})
    gx, gw = torch.autograd.grad(y.square().sum(), (x, w))
    u, v = (t.detach().clone().requires_grad_() for t in (x, w))
    want = _act(u @ v.t(), act) + (0 if r is None else r)
    hx, hw = torch.autograd.grad(want.square().sum(), (u, v))
    assert torch.allclose(gx, hx, rtol=1e-5, atol=1e-6) and torch.allclose(gw, hw, rtol=1e-5, atol=1e-6)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_linear_keeps_nothing_without_gradients(stand_in, act):
    x, w, r = _rand(4, 8), _rand(6, 8), _rand(4, 6)
    with torch.no_grad():
        decoder.linear(x, w, act, r)
    decoder.linear(x.detach(), w.detach(), act)
    assert [c for c in stand_in.calls if c[0] == "linear"] == [("linear", False)] * 2
    assert decoder.linear(x, w, act).requires_grad and decoder.linear(x.detach(), w.detach(), act, r).requires_grad


def test_attention_after_the_rotation_keeps_its_inputs_once(stand_in):
    qkv, w, tables = _rand(1, 4, 6, 8), _rand(8), (torch.zeros(4, 4), torch.zeros(4, 4))
    out, held = _held(lambda: decoder.RotaryAttentionFunction.apply(qkv, w, w, *tables, 4))
    size = qkv.numel() * qkv.element_size()
    assert sum(held.values()) < 1.5 * size  # the projection's output; what it is turned into is made again from it
    g, gw = torch.autograd.grad(out.square().sum(), (qkv, w))
    u, v = qkv.detach().clone().requires_grad_(), w.detach().clone().requires_grad_()
    q, k, x = (t.transpose(1, 2) for t in (u[:, :, :2] * v * 8 ** -0.5, u[:, :, 2:4] * v, u[:, :, 4:]))
    hu, hv = torch.autograd.grad((q * k * x).square().sum(), (u, v))
    assert torch.allclose(g, hu, rtol=1e-5, atol=1e-6) and torch.allclose(gw, hv, rtol=1e-5, atol=1e-6)
