"""Serving calls of the decoder on views: the last tokens of a batch, a column of ids, a slice of features."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T
from paper_2106_06899_gb300.decoder import Decoder

pytestmark = pytest.mark.gpu
V, D, H = 1000, 256, 4


def _model(topk=None, layers=2, cap=256):
    torch.manual_seed(3)
    return Decoder(layers, D, H, 512, topk=topk, fused=True, max_positions=cap, vocab=V)


def _filled(m, batch, cap):
    g = torch.Generator("cuda").manual_seed(4)
    caches = m.new_cache(batch, cap)
    for c in caches:
        for t in c:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
    return caches


def test_views_of_features_and_ids():
    m = _model()
    ids = torch.randint(0, V, (3, 20), device="cuda")
    start = torch.tensor([5, 0, 40], dtype=torch.int32, device="cuda")
    with torch.no_grad():
        features = m._features(ids)  # [3, 20, D]
        whole = m(ids)
        # what the last token of each sequence says, of a column of ids
        r, want = m.logprobs(whole[:, -1], ids[:, 3], top=4), m.logprobs(whole[:, -1].contiguous(), ids[:, 3].contiguous(), top=4)
        assert all(torch.equal(a, b) for a, b in zip(r, want))
    # a column of ids or features to a step, a slice of them to drafted tokens and to packed prompts
    of = {"step": (lambda x, c: m.step(x, c, start), lambda x: x[:, 7]), "step_tree": (lambda x, c: m.step_tree(x, c, start), lambda x: x[:, 2:7]),
          "prefill": (lambda x, c: m.prefill(x, torch.tensor([0, 4, 10], dtype=torch.int32, device="cuda"), c), lambda x: x[1, ::2])}
    for name, (call, view) in of.items():
        outs = []
        for x in (view(ids), view(ids).contiguous(), view(features), view(features).contiguous()):
            caches = _filled(m, 3, 64)
            outs.append([call(x, caches), *(t for c in caches for t in c)])
        for other in outs[1:]:
            assert all(torch.equal(a, b) for a, b in zip(outs[0], other)), name
    T.topk_check()
