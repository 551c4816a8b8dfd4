"""Calls on a stream that is not the current one: what a call allocates for it belongs to that stream."""
import pytest
import torch

from paper_2106_06899_gb300 import topk as T

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def _stream_of(t):
    """The stream whose memory t lies in."""
    at = t.data_ptr()
    for s in torch.cuda.memory_snapshot():
        if s["address"] <= at < s["address"] + s["total_size"]:
            return s["stream"]
    raise AssertionError("not the allocator's memory")


def _calls():
    x, w, dy = (torch.randn(*s, device="cuda").to(BF) for s in ((300, 256), (512, 256), (300, 512)))
    z = torch.randn(300, 512, device="cuda").to(BF)
    qkv = torch.randn(2, 40, 12, 64, device="cuda").to(BF)
    q, k, v = qkv[:, :, :4], qkv[:, :, 4:8], qkv[:, :, 8:]
    cos, sin = T.rope_tables(40, 64)
    dq, dk, dv = (torch.randn(2, 4, 40, 64, device="cuda").to(BF) for _ in range(3))
    a, b, c = (torch.randn(1, 2, 256, 64, device="cuda").to(BF) for _ in range(3))
    out, idx, score = T.attention(a, b, c, 32, return_indices=True)
    mask = torch.ones(1, 1, 256, 256, dtype=torch.bool, device="cuda").tril()
    f1, f2 = (torch.randn(2048, 256, device="cuda").to(BF) for _ in range(2))
    fo, fi, fs = T.ffn(x, f1, f2, 64, return_indices=True)
    return {
        "linear": lambda s: T.linear(x, w, act="gelu", return_preact=True, stream=s),
        "linear_bwd": lambda s: T.linear_bwd(dy, x, w, z, "gelu", bias=True, stream=s),
        "qk_norm_rope": lambda s: T.qk_norm_rope(q, k, v, cos, sin, stream=s),
        "qk_norm_rope_bwd": lambda s: T.qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, stream=s),
        "attention": lambda s: T.attention(a, b, c, 32, return_indices=True, stream=s),
        "attention with a mask": lambda s: T.attention(a, b, c, 32, mask=mask, return_indices=True, stream=s),
        "attention_bwd": lambda s: T.attention_bwd(a, b, c, out, idx, score, stream=s),
        "vanilla_attention": lambda s: T.vanilla_attention(a, b, c, stream=s),
        "ffn": lambda s: T.ffn(x, f1, f2, 64, return_indices=True, stream=s),
        "ffn_bwd": lambda s: T.ffn_bwd(x, f1, f2, fo, fi, fs, stream=s),
        "vanilla_ffn": lambda s: T.vanilla_ffn(x, f1, f2, stream=s),
    }


# the attention's and the top-k layer's gradients of keys are added in an order that depends on atomic ranks
UNORDERED = ("attention_bwd", "ffn_bwd")
NAMES = ["linear", "linear_bwd", "qk_norm_rope", "qk_norm_rope_bwd", "attention", "attention with a mask", "attention_bwd",
         "vanilla_attention", "ffn", "ffn_bwd", "vanilla_ffn"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("handle", [False, True])
def test_outputs_belong_to_the_calls_stream(name, handle):
    torch.manual_seed(0)
    call = _calls()[name]
    as_tuple = lambda r: r if isinstance(r, tuple) else (r,)  # noqa: E731
    want = as_tuple(call(None))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got = as_tuple(call(st.cuda_stream if handle else st))
    st.synchronize()
    T.topk_check()
    assert torch.cuda.current_stream() != st
    for g, w in zip(got, want):
        assert _stream_of(g) == st.cuda_stream
        assert name in UNORDERED or torch.equal(g, w)


@pytest.mark.parametrize("handle", [0, 1, 2])
def test_default_streams_by_their_handles(handle):
    x, w = (torch.randn(64, 64, device="cuda").to(BF) for _ in range(2))
    want = T.linear(x, w)
    torch.cuda.synchronize()
    got = T.linear(x, w, stream=handle)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
