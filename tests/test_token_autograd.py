"""What the decoder's ends do where derivatives are asked for, and with views, with stand-ins for the library's calls on the CPU (no GPU needed)."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from paper_2106_06899_gb300 import decoder
from paper_2106_06899_gb300 import topk


class _StandIn:
    """The calls of the decoder's ends as torch operations that leave no graph and drop tangents, as the library does."""

    TokenLogProbs = topk.TokenLogProbs

    @staticmethod
    def _bare(*tensors):
        return (None if t is None else forward_ad.unpack_dual(t.detach()).primal for t in tensors)

    def linear(self, x, w, bias=None, act="none", residual=None, return_preact=False, stream=None):
        assert x.is_contiguous() and (residual is None or residual.is_contiguous())
        x, w, residual = self._bare(x, w, residual)
        z = x @ w.t()
        y = {"none": z, "relu": z.relu()}[act] + (0 if residual is None else residual)
        return (y, z) if return_preact else y

    def linear_bwd(self, dy, x, w, preact=None, act="none", bias=False, need_dx=True, need_dw=True, grad_dtype=None, stream=None):
        return dy @ w if need_dx else None, dy.t() @ x if need_dw else None, None

    def embedding(self, ids, weight, scale=1.0, stream=None):
        assert ids.is_contiguous()
        (weight,) = self._bare(weight)
        return torch.where((ids >= 0)[..., None], weight[ids.clamp_min(0)] * scale, 0)

    def embedding_bwd(self, dy, ids, rows, scale=1.0, grad_dtype=None, into=None, stream=None):
        flat = dy.reshape(-1, dy.shape[-1]) * scale
        return torch.zeros(rows + 1, dy.shape[-1]).index_add_(0, torch.where(ids < 0, rows, ids).reshape(-1), flat)[:-1]

    def token_logprobs(self, logits, targets=None, top=0, scale=1.0, stream=None):
        assert targets is None or targets.is_contiguous()
        (logits,) = self._bare(logits)
        lse = torch.logsumexp(logits * scale, 1)
        logp = logits * scale - lse[:, None]
        best = logp.topk(top, 1) if top else (None, None)
        return topk.TokenLogProbs(None if targets is None else logp.gather(1, targets[:, None])[:, 0], -(logp.exp() * logp).sum(1), lse, best[0],
                                  None if best[1] is None else best[1].int())

    def token_logprobs_bwd(self, logits, lse, targets=None, dlogp=None, entropy=None, dentropy=None, top_ids=None, dtop=None, scale=1.0, out=None, stream=None):
        with torch.enable_grad():
            x = logits.detach().requires_grad_()
            logp = torch.log_softmax(x * scale, 1)
            total = 0.0
            if dlogp is not None:
                total = total + (logp.gather(1, targets[:, None])[:, 0] * dlogp).sum()
            if dentropy is not None:
                total = total - ((logp.exp() * logp).sum(1) * dentropy).sum()
            return torch.autograd.grad(total, x)[0]


V, D = 16, 8


@pytest.fixture
def model(monkeypatch):
    torch.manual_seed(0)
    m = decoder.Decoder(0, D, 1, 16, fused=True, max_positions=8, vocab=V, device="cpu").float()
    monkeypatch.setattr(decoder, "T", _StandIn())
    return m


def _tangent(t):
    return forward_ad.make_dual(t.detach(), torch.ones_like(t))


def test_tangents_are_refused(model):
    # a tangent that went no further would be a derivative without the part behind it: an error in place of that
    x, w, r = torch.randn(4, D), torch.randn(6, D), torch.randn(4, 6)
    ids = torch.arange(4)
    with forward_ad.dual_level():
        calls = [lambda: decoder.linear(_tangent(x), w), lambda: decoder.linear(x, _tangent(w)), lambda: decoder.linear(x, w, "relu", _tangent(r)),
                 lambda: model.logprobs(_tangent(x)), lambda: model.logprobs(_tangent(x), ids)]
        for grad in (True, False):
            with torch.set_grad_enabled(grad):
                for call in calls:
                    with pytest.raises(NotImplementedError):
                        call()
        model.embedding.requires_grad_(False)
        plain, weight = model.embedding, _tangent(model.embedding)
        del model.embedding
        model.embedding = weight
        for grad in (True, False):
            with torch.set_grad_enabled(grad):
                for call in (lambda: model(ids), lambda: model.logprobs(x)):
                    with pytest.raises(NotImplementedError):
                        call()
        model.embedding = plain
        # numbers without one are taken as ever
        assert model(ids).shape == (4, D) and decoder.linear(x, w).shape == (4, 6)


def test_tangents_are_refused_by_generation(model):
    x, start = torch.randn(2, D), torch.zeros(2, dtype=torch.int32)
    calls = {"step": (x, [], start), "step_tree": (x[:, None], [], start)}
    model.layers = torch.nn.ModuleList()
    for name, args in calls.items():
        call = getattr(model, name)
        assert call(*args).shape == args[0].shape
        with forward_ad.dual_level():
            assert call(*args).shape == args[0].shape
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call(_tangent(args[0]), *args[1:])

            class Call(torch.nn.Module):
                def __init__(self):
                    super().__init__()
                    self.m = model

                def forward(self, *a):
                    return getattr(self.m, name)(*a)

            with pytest.raises(NotImplementedError, match="forward-mode"):
                torch.func.functional_call(Call(), {"m.norm.weight": _tangent(model.norm.weight)}, args)


def test_a_loss_with_the_sums_logarithm_is_refused(model):
    # its gradient is not made: an error in place of a gradient without that term
    ids = torch.arange(6).view(2, 3)
    r = model.logprobs(model(ids)[:, :-1], ids[:, 1:])
    with pytest.raises(RuntimeError, match="lse"):
        (-r.logp.mean() + 1e-4 * r.lse.square().mean()).backward()
    with pytest.raises(RuntimeError, match="lse"):
        model.logprobs(model(ids)).lse.sum().backward()
    for p in model.parameters():
        p.grad = None
    r = model.logprobs(model(ids)[:, :-1], ids[:, 1:])
    assert torch.equal(r.lse, torch.logsumexp(model(ids)[:, :-1].reshape(-1, D) @ model.embedding.t(), 1))
    loss = -r.logp.mean() - 0.1 * r.entropy.mean() + 0 * r.lse.detach().mean()  # as a number it may be used
    loss.backward()
    got = model.embedding.grad.clone()
    model.embedding.grad = None
    h = torch.nn.functional.layer_norm(model.embedding[ids] * D ** 0.5, (D,), model.norm.weight, model.norm.bias)
    logp = torch.log_softmax(h[:, :-1].reshape(-1, D) @ model.embedding.t(), 1)
    (-logp.gather(1, ids[:, 1:].reshape(-1, 1)).mean() + 0.1 * (logp.exp() * logp).sum(1).mean()).backward()
    assert torch.allclose(got, model.embedding.grad, rtol=1e-4, atol=1e-5)
    with torch.no_grad():
        assert not model.logprobs(model(ids)).lse.requires_grad


def test_views_of_features_and_targets(model):
    # the last token of each sequence, and a column of a batch's ids
    ids = torch.arange(12).view(3, 4)
    features = model(ids)
    for grad in (True, False):
        with torch.set_grad_enabled(grad):
            r = model.logprobs(features[:, -1], ids[:, 2], top=2)
            want = model.logprobs(features[:, -1].contiguous(), ids[:, 2].contiguous(), top=2)
            assert all(torch.equal(a, b) for a, b in zip(r, want))
            # features by columns, and one row for all
            assert torch.equal(model.logprobs(features[:, -1].t().contiguous().t()).lse, want.lse)
            assert model.logprobs(features[0, 0].expand(3, D)).lse.shape == (3,)
