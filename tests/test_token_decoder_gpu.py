"""The fused decoder on token ids: trained through its embedding and log probabilities, and served from packed prompts, single tokens and
drafted trees.

References are the same decoder with PyTorch operations at its two ends, in 64 bits where they add up; what runs twice through
bf16 layers may differ by some roundings (2^-8 each): 3e-2 in the 2-norm for two layers, as for single steps.
"""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from paper_2106_06899_gb300.decoder import Decoder, EmbeddingFunction, TokenLogProbsFunction
from paper_2106_06899_gb300.optim import AdamW

pytestmark = pytest.mark.gpu
F64, BF = torch.float64, torch.bfloat16
V, D, H, LAYERS = 1000, 256, 4, 2


def _rel(a, b):
    return ((a.double() - b.double()).norm() / b.double().norm()).item()


def _model(topk=None, cap=256, seed=0):
    torch.manual_seed(seed)
    return Decoder(LAYERS, D, H, 512, topk=topk, fused=True, max_positions=cap, vocab=V)


@pytest.mark.parametrize("topk", [None, 64])
def test_training_gradients(topk):
    m = _model(topk)
    ids = torch.randint(0, V, (2, 200), device="cuda")
    ids[1, 150:] = -1  # padding
    targets = torch.roll(ids, -1, 1)
    targets[:, -1] = -1
    r = m.logprobs(m(ids), targets, top=3)
    loss = -(r.logp.sum() + 0.01 * r.entropy.sum()) / 348 + 0.001 * r.top_logp.mean()
    loss.backward()
    T.topk_check()
    got = {n: p.grad.clone() for n, p in m.named_parameters()}
    m.zero_grad()
    # the ends in PyTorch operations: the gradient that reaches the layers, and those of the embedding from both of its uses
    w = m.embedding
    x = torch.where((ids >= 0)[..., None], (w[ids.clamp_min(0)].float() * D ** 0.5), 0.0).to(BF)
    h = x
    for layer in m.layers:
        h = layer.forward_fused(h, m.tables)
    h = m.norm(h)
    logits = (h.reshape(-1, D).to(F64) @ w.to(F64).t()).to(BF).to(F64)
    logp = torch.log_softmax(logits, 1)
    t = targets.reshape(-1)
    picked = torch.where(t >= 0, logp.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0)
    entropy = -(logp.exp() * logp).sum(1)
    want = -(picked.sum() + 0.01 * entropy.sum()) / 348 + 0.001 * logp.topk(3, 1)[0].mean()
    want.backward()
    loss, want = float(loss.detach()), float(want.detach())
    assert abs(loss - want) <= 1e-4 * abs(want)
    for n, p in m.named_parameters():
        # the gradient of the logits, that of the features and the parameter's own are rounded to bf16 on each side
        assert _rel(got[n], p.grad) <= 3e-2, n


def test_functions_against_64_bits():
    # gradcheck needs 64 bits; the functions' own gradients are held against autograd's of the definitions
    ids = torch.tensor([[3, 1, -1], [3, 0, 6]], device="cuda")
    w = torch.randn(7, 24, device="cuda", requires_grad=True)
    g = torch.randn(2, 3, 24, device="cuda")
    (EmbeddingFunction.apply(ids, w, 1.5) * g).sum().backward()
    w64 = w.detach().to(F64).requires_grad_()
    (torch.where((ids >= 0)[..., None], w64[ids.clamp_min(0)] * 1.5, 0.0) * g).sum().backward()
    assert (w.grad.to(F64) - w64.grad).abs().max() <= 2.0 ** -20
    x = torch.randn(5, 40, device="cuda", requires_grad=True)
    t = torch.tensor([1, 39, -1, 0, 7], device="cuda")
    a, b, c = torch.randn(5, device="cuda"), torch.randn(5, device="cuda"), torch.randn(5, 2, device="cuda")
    r = T.TokenLogProbs(*TokenLogProbsFunction.apply(x, t, 2, 0.8))
    assert not r.lse.requires_grad and not r.top_ids.requires_grad
    ((r.logp * a).sum() + (r.entropy * b).sum() + (r.top_logp * c).sum()).backward()
    x64 = x.detach().to(F64).requires_grad_()
    logp = torch.log_softmax(x64 * 0.8, 1)
    picked = torch.where(t >= 0, logp.gather(1, t.clamp_min(0)[:, None])[:, 0], 0.0)
    ((picked * a).sum() - ((logp.exp() * logp).sum(1) * b).sum() + (logp.topk(2, 1)[0] * c).sum()).backward()
    assert (x.grad.to(F64) - x64.grad).abs().max() <= 2.0 ** -16
    for part in ("entropy", "logp"):  # one output alone
        x.grad = None
        getattr(T.TokenLogProbs(*TokenLogProbsFunction.apply(x, t, 0, 1.0)), part).sum().backward()
        assert x.grad.isfinite().all()
    with pytest.raises(RuntimeError):  # no gradients of gradients
        (d,) = torch.autograd.grad(TokenLogProbsFunction.apply(x, t, 0, 1.0)[0].sum(), x, create_graph=True)
        d.sum().backward()


def test_a_training_step_lowers_the_loss_of_its_batch():
    m = _model(64)
    opt = AdamW(m.parameters(), lr=1e-3, weight_decay=0.0, masters=True)
    ids = torch.randint(0, V, (2, 128), device="cuda")
    for _ in range(2):
        opt.zero_grad()
        (-m.logprobs(m(ids)[:, :-1], ids[:, 1:]).logp.mean()).backward()
        assert all(p.grad.isfinite().all() for p in m.parameters())
        opt.step()
    T.topk_check()


def test_prompts_steps_and_trees_give_what_whole_sequences_give():
    m = _model()
    lens = [70, 1, 130]
    longest = max(lens) + 12
    ids = torch.randint(0, V, (3, longest), device="cuda")
    with torch.no_grad():
        whole = m(ids)
    caches = m.new_cache(3, 256)
    for c in caches:
        for t in c:
            t.fill_(float("nan"))  # rows that no token has been written to are read by none
    starts = torch.tensor([0, 70, 71, 201], dtype=torch.int32, device="cuda")
    y = m.prefill(torch.cat([ids[b, :n] for b, n in enumerate(lens)]), starts, caches)
    for b, n in enumerate(lens):
        assert _rel(y[starts[b]:starts[b + 1]], whole[b, :n]) <= 3e-2, b
    start = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # a chain of 4 drafted tokens, kept whole
    b = torch.arange(3, device="cuda")[:, None]
    at = start.long()[:, None] + torch.arange(4, device="cuda")
    y = m.step_tree(ids[b, at], caches, start)
    assert _rel(y, whole[b, at]) <= 3e-2
    start = start + 4
    # a tree: the sequence's next three tokens are tokens 0, 3 and 4 of six, the others branch off
    parents = torch.tensor([[-1, -1, 0, 0, 3, 2]]).expand(3, 6)
    draft = torch.randint(0, V, (3, 6), device="cuda")
    at = start.long()[:, None] + torch.arange(3, device="cuda")
    path = torch.tensor([[0, 3, 4]], device="cuda").expand(3, 3)
    draft[:, [0, 3, 4]] = ids[b, at]
    y = m.step_tree(draft, caches, start, tree=T.tree_mask(parents.cuda()))
    assert _rel(y[b, path], whole[b, at]) <= 3e-2
    m.keep(caches, start, path)
    start = start + 3
    # single tokens go on from the kept path
    for _ in range(3):
        y = m.step_tree(ids[b, start.long()[:, None]], caches, start)[:, 0]
        assert _rel(y, whole[b[:, 0], start.long()]) <= 3e-2
        start = start + 1
    # what they say of the next tokens
    r = m.logprobs(y, top=5)
    logits = (y.to(F64) @ m.embedding.to(F64).t()).to(BF).float()
    assert (r.top_logp[:, 0] - torch.log_softmax(logits, 1).amax(1)).abs().max() <= 1e-2  # a logit's rounding
    T.topk_check()


def test_padded_prompts_and_too_long_ones():
    m = _model()
    ids = torch.randint(0, V, (60,), device="cuda")
    a, b = m.new_cache(2, 40), m.new_cache(2, 40)
    starts = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    whole = m.prefill(ids[:50], starts, a)
    padded = torch.cat((ids[:50], torch.full((10,), -1, device="cuda")))  # rows of no sequence behind the last one
    assert torch.equal(m.prefill(padded, starts, b)[:50], whole)
    assert all(torch.equal(x, y) for p, q in zip(a, b) for x, y in zip(p, q))
    with pytest.raises(ValueError):
        m.prefill(ids, torch.tensor([0, 60], dtype=torch.int32, device="cuda"), m.new_cache(1, 40))
    T.topk_check()


def test_trees_with_topk_attention():
    m = _model(topk=256)  # more than there are keys: plain attention's result by the other path
    plain = _model()
    plain.load_state_dict(m.state_dict())
    ids = torch.randint(0, V, (2, 7), device="cuda")
    tree = T.tree_mask(torch.tensor([[-1, 0, 0, 1, 2, 2, -1]] * 2).cuda())
    start = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    outs = []
    for model in (m, plain):
        caches = model.new_cache(2, 64)
        g = torch.Generator("cuda").manual_seed(1)
        for c in caches:
            for t in c:
                t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        outs.append(model.step_tree(ids, caches, start, tree=tree))
    T.topk_check()
    assert _rel(*outs) <= 3e-2


def test_refusals():
    with pytest.raises(ValueError):
        Decoder(1, 256, 4, 512, vocab=1000)
    with pytest.raises(ValueError):
        Decoder(1, 256, 4, 512, fused=True, vocab=1001)
    m = _model(topk=8)
    with pytest.raises(ValueError):
        m.prefill(torch.zeros(4, dtype=torch.int64, device="cuda"), torch.tensor([0, 4], dtype=torch.int32, device="cuda"), m.new_cache(1, 8))
    with pytest.raises(ValueError):
        Decoder(1, 256, 4, 512, fused=True).logprobs(torch.zeros(1, 256, device="cuda", dtype=BF))


def test_more_sequences_than_the_caches_hold():
    m = _model()
    ids, caches = torch.zeros(6, dtype=torch.int64, device="cuda"), m.new_cache(2, 8)
    starts = torch.tensor([0, 2, 4, 6], dtype=torch.int32, device="cuda")
    for bad in (starts, starts[:1], starts[:0]):
        with pytest.raises(ValueError):
            m.prefill(ids, bad, caches)
    for sequences, rows in ((3, 3), (2, 1)):
        with pytest.raises(ValueError):
            m.keep(caches, torch.zeros(sequences, dtype=torch.int32, device="cuda"), torch.zeros((rows, 1), dtype=torch.int64, device="cuda"))
    assert not any(t.any() for pair in caches for t in pair)
