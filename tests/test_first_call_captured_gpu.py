"""A process whose first call of the library is captured into a graph: the calls that take scratch create its pool then."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import torch
from paper_2106_06899_gb300 import topk as T
dev, bf = dict(device="cuda"), dict(device="cuda", dtype=torch.bfloat16)
ids, dy, x = torch.randint(0, 100, (9000,), **dev), torch.randn(9000, 64, **dev), torch.randn(3, 50000, **dev)
q, starts = torch.randn(300, 4, 64, **bf), torch.tensor([0, 100, 300], dtype=torch.int32, **dev)
cache, one = torch.randn(2, 4, 512, 64, **bf), torch.randn(2, 4, 3, 64, **bf)
held = torch.tensor([100, 400], dtype=torch.int32, **dev)
call = dict(embedding=lambda: T.embedding(ids, dy[:100].contiguous()), embedding_bwd=lambda: T.embedding_bwd(dy, ids, 100),
            logprobs=lambda: T.token_logprobs(x, top=5).top_logp, prompt=lambda: T.prompt_attention(q, q, q, starts),
            tree=lambda: T.tree_attention(one, cache, cache, held), attention=lambda: T.attention(cache, cache, cache, 32, causal=True))["NAME"]
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = call()
for _ in range(2):
    out.zero_()
    graph.replay()
    got = out.clone()
T.topk_check()
assert torch.equal(got, call()) and got.abs().sum() > 0
print("as called")
"""


@pytest.mark.parametrize("name", ["embedding", "embedding_bwd", "logprobs", "prompt", "tree", "attention"])
def test_first_call(name):
    r = subprocess.run([sys.executable, "-c", SCRIPT.replace("NAME", name)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("as called"), r.stderr[-2000:]
