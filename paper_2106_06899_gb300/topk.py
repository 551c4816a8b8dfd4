"""Thin ctypes binding of libtopk.so (include/topk_attention.h).

Argument marshalling only: every step of the computation runs in the CUDA
library.  Functions carry the C-ABI names; they take torch tensors, read
sizes from their shapes, pass raw pointers and raise ``TopkError`` on a
non-zero return code.  There is no fallback: if libtopk.so is missing or
no GB300 is present the calls fail loudly.
"""
from __future__ import annotations

import ctypes
import os
import struct
import threading
from typing import NamedTuple, Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtopk.so")

TOPK_F32, TOPK_BF16 = 0, 1
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}  # TOPK_ACT_*
_lock = threading.Lock()
_lib = None


class TopkError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {error_string(code)} (code {code})")


def lib() -> ctypes.CDLL:
    """The loaded libtopk.so.  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                raise ImportError(f"{LIB_PATH} is not built; run `python -m paper_2106_06899_gb300.build` "
                                  "(nvcc for sm_103a) first")
            L = ctypes.CDLL(LIB_PATH)
            vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
            L.topk_attn_fwd.argtypes = [vp, vp, vp, vp] + [i32] * 9 + [vp]
            L.topk_attn_fwd_indices.argtypes = [vp, vp, vp, vp] + [i32] * 9 + [vp, vp, vp]
            L.topk_ffn_fwd.argtypes = [vp, vp, vp, vp] + [i32] * 4 + [vp]
            L.topk_ffn_fwd_indices.argtypes = [vp, vp, vp, vp] + [i32] * 4 + [vp, vp, vp]
            L.topk_attn_fwd_host.argtypes = [vp, vp, vp, vp] + [i32] * 9 + [vp]
            L.topk_ffn_fwd_host.argtypes = [vp, vp, vp, vp] + [i32] * 4 + [vp]
            L.topk_ffn_fwd_noalloc.argtypes = [vp, vp, vp, vp] + [i32] * 4 + [vp]
            L.topk_attn_workspace_bytes.argtypes = [i32] * 8
            L.topk_attn_workspace_bytes.restype = sz
            L.topk_ffn_workspace_bytes.argtypes = [i32] * 4
            L.topk_ffn_workspace_bytes.restype = sz
            L.topk_attn_fwd_masked.argtypes = [vp, vp, vp, vp] + [i32] * 8 + [vp, vp, ctypes.c_longlong,
                                                                            ctypes.c_longlong, i32, vp, vp, vp]
            L.topk_vanilla_attn_fwd.argtypes = [vp, vp, vp, vp] + [i32] * 7 + [vp, i32, vp]
            L.topk_vanilla_attn_workspace_bytes.argtypes = [i32] * 6
            L.topk_vanilla_attn_workspace_bytes.restype = sz
            L.topk_vanilla_ffn_fwd.argtypes = [vp, vp, vp, vp] + [i32] * 4 + [vp]
            L.topk_vanilla_ffn_workspace_bytes.argtypes = [i32] * 4
            L.topk_vanilla_ffn_workspace_bytes.restype = sz
            L.topk_attn_bwd.argtypes = [vp] * 9 + [i32] * 7 + [vp]
            L.topk_ffn_bwd.argtypes = [vp] * 9 + [i32] * 4 + [vp]
            L.topk_attn_bwd_workspace_bytes.argtypes = [i32] * 7
            L.topk_attn_bwd_workspace_bytes.restype = sz
            L.topk_ffn_bwd_workspace_bytes.argtypes = [i32] * 4
            L.topk_ffn_bwd_workspace_bytes.restype = sz
            L.topk_qk_norm_rope_fwd.argtypes = [vp, vp, vp, vp, i32, vp, vp]
            L.topk_qk_norm_rope_bwd.argtypes = [vp, vp, vp, vp, i32, vp, vp, vp, vp]
            L.topk_qk_norm_rope_bwd_workspace_bytes.argtypes = [i32] * 5
            L.topk_qk_norm_rope_bwd_workspace_bytes.restype = sz
            L.topk_linear_fwd.argtypes = [vp] * 6 + [i32] * 4 + [vp]
            L.topk_linear_bwd.argtypes = [vp] * 7 + [i32] * 5 + [vp]
            L.topk_linear_workspace_bytes.argtypes = [i32] * 3
            L.topk_linear_workspace_bytes.restype = sz
            L.topk_linear_bwd_workspace_bytes.argtypes = [i32] * 4
            L.topk_linear_bwd_workspace_bytes.restype = sz
            L.topk_adamw_step.argtypes = [vp, i32, i32, i32, i32, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                          ctypes.c_longlong, vp, ctypes.c_uint32, vp]
            f32, i64 = ctypes.c_float, ctypes.c_longlong
            L.topk_embedding_fwd.argtypes = [vp, i32, vp, vp, i32, i32, i32, f32, i32, vp]
            L.topk_embedding_bwd.argtypes = [vp, vp, i32, vp, i32, i32, i32, f32, i32, i32, i32, vp]
            L.topk_embedding_bwd_workspace_bytes.argtypes = [i32] * 3
            L.topk_embedding_bwd_workspace_bytes.restype = sz
            L.topk_token_logprobs_fwd.argtypes = [vp, i64, vp, i32, f32, i32] + [vp] * 5 + [i32] * 3 + [vp]
            L.topk_token_logprobs_bwd.argtypes = [vp, i64, vp, vp, i32] + [vp] * 5 + [i32, f32, vp, i64] + [i32] * 3 + [vp]
            L.topk_prompt_attn_fwd.argtypes = [vp, vp]
            L.topk_prompt_attn_workspace_bytes.argtypes = [i32]
            L.topk_prompt_attn_workspace_bytes.restype = sz
            L.topk_tree_attn_fwd.argtypes = [vp, vp]
            L.topk_check.argtypes = [vp]
            L.topk_error_string.argtypes = [i32]
            L.topk_error_string.restype = ctypes.c_char_p
            L.topk_last_launch_count.argtypes = []
            L.topk_set_wait_limit_us.argtypes = [ctypes.c_longlong]
            L.topk_set_wait_limit_us.restype = ctypes.c_longlong
            L.topk_debug_skip_arrive.argtypes = [i32]
            L.topk_pool_usage.argtypes = [ctypes.POINTER(sz), ctypes.POINTER(sz), i32]
            L.topk_pool_trim.argtypes = []
            for f in ("topk_attn_fwd", "topk_attn_fwd_indices", "topk_ffn_fwd", "topk_ffn_fwd_indices",
                      "topk_attn_fwd_host", "topk_ffn_fwd_host", "topk_ffn_fwd_noalloc", "topk_check",
                      "topk_last_launch_count",
                      "topk_debug_skip_arrive", "topk_pool_usage", "topk_pool_trim", "topk_attn_bwd",
                      "topk_ffn_bwd", "topk_attn_fwd_masked", "topk_vanilla_attn_fwd", "topk_vanilla_ffn_fwd",
                      "topk_qk_norm_rope_fwd", "topk_qk_norm_rope_bwd", "topk_adamw_step", "topk_linear_fwd", "topk_linear_bwd",
                      "topk_embedding_fwd", "topk_embedding_bwd", "topk_token_logprobs_fwd", "topk_token_logprobs_bwd",
                      "topk_prompt_attn_fwd", "topk_tree_attn_fwd"):
                getattr(L, f).restype = i32
            _lib = L
    return _lib


def error_string(code: int) -> str:
    return lib().topk_error_string(int(code)).decode()


def _check(rc: int, where: str) -> None:
    if rc != 0:
        raise TopkError(rc, where)


# The current stream's handle without building a Stream object (0.3 us in place of 12).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return TOPK_F32
    if t.dtype == torch.bfloat16:
        return TOPK_BF16
    raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _on_gpu(names: str, first, *others) -> None:
    """Refuses tensors (or None) that are not on the current CUDA device, where the kernels run."""
    device = first.get_device()  # -1: not on a GPU
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError(f"{names} must be CUDA tensors of one device")
    if device < 0 or device != torch.cuda.current_device():
        raise ValueError(f"{names} must be CUDA tensors on the current device")


def _changed(*tensors) -> None:
    """Counts tensors (or None) as changed in place, for graphs that hold them: autograd does not see a kernel's writes."""
    torch.autograd.graph.increment_version([t for t in tensors if t is not None])


def _attn_dims(q, k, v, out):
    for name, t in (("q", q), ("k", k), ("v", v), ("out", out)):
        if t.dim() != 4 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous [B, H, L, d] tensor")
    B, H, Lq, d = q.shape
    Lk = k.shape[2]
    if tuple(k.shape) != (B, H, Lk, d) or tuple(v.shape) != (B, H, Lk, d) or tuple(out.shape) != (B, H, Lq, d):
        raise ValueError("shape mismatch between q, k, v, out")
    if not (q.dtype == k.dtype == v.dtype == out.dtype):
        raise TypeError("q, k, v, out must share a dtype")
    return B, H, Lq, Lk, d


def topk_attn_fwd(q, k, v, out, topk: int, chunk: int = 1024, causal: bool = False, stream=None) -> None:
    """Eq. 4 top-k attention into ``out`` (device tensors [B,H,L,d], fp32 or bf16)."""
    B, H, Lq, Lk, d = _attn_dims(q, k, v, out)
    rc = lib().topk_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, Lq, Lk, d, int(topk), int(chunk),
                             int(bool(causal)), _dtype_code(q), _stream(stream))
    _check(rc, "topk_attn_fwd")


def topk_attn_fwd_indices(q, k, v, out, topk: int, chunk: int = 1024, causal: bool = False, idx=None,
                          score=None, stream=None) -> None:
    """topk_attn_fwd plus kept indices idx [B,H,Lq,topk] int32 and scores [B,H,Lq,topk] fp32."""
    B, H, Lq, Lk, d = _attn_dims(q, k, v, out)
    for name, t, dt in (("idx", idx, torch.int32), ("score", score, torch.float32)):
        if t is not None and (t.dtype != dt or tuple(t.shape) != (B, H, Lq, topk) or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous [B,H,Lq,topk] {dt} tensor")
    rc = lib().topk_attn_fwd_indices(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, Lq, Lk, d, int(topk), int(chunk),
                                     int(bool(causal)), _dtype_code(q), _ptr(idx), _ptr(score), _stream(stream))
    _check(rc, "topk_attn_fwd_indices")


def pack_mask(mask: torch.Tensor):
    """A boolean mask [B or 1, H or 1, Lq, Lk] (True = the key takes part, Eq. 2's B_ij = 0) in the
    C ABI's layout: bit j % 32 of int32 word j // 32 of each query row, on mask's device.

    Returns (words [B|1, H|1, Lq, ceil(Lk/32)] int32, batch stride, head stride) in words; a stride is
    0 where the mask has one entry for all batches or heads."""
    if mask.dim() != 4 or mask.dtype != torch.bool:
        raise ValueError("mask must be a 4-D bool tensor [B or 1, H or 1, Lq, Lk]")
    mb, mh, Lq, Lk = mask.shape
    W = (Lk + 31) // 32
    padded = torch.zeros(mb, mh, Lq, W * 32, dtype=torch.int64, device=mask.device)
    padded[..., :Lk] = mask.to(torch.int64)
    shifts = torch.arange(32, dtype=torch.int64, device=mask.device)
    words = (padded.view(mb, mh, Lq, W, 32) << shifts).sum(dim=-1)
    words = torch.where(words >= 2**31, words - 2**32, words).to(torch.int32).contiguous()
    hs = Lq * W if mh > 1 else 0
    bs = mh * Lq * W if mb > 1 else 0
    return words, bs, hs


def topk_attn_fwd_masked(q, k, v, out, topk: int, chunk: int = 1024, causal: bool = False, kv_len=None,
                         mask_words=None, mask_batch_stride: int = 0, mask_head_stride: int = 0, idx=None,
                         score=None, stream=None) -> None:
    """Eq. 4 under Eq. 2's masks: causal (queries are the last Lq positions), kv_len [B] int32 (keys per
    batch) and a packed bit mask (see pack_mask); idx/score as topk_attn_fwd_indices, or None."""
    B, H, Lq, Lk, d = _attn_dims(q, k, v, out)
    if kv_len is not None and (kv_len.dtype != torch.int32 or tuple(kv_len.shape) != (B,)):
        raise ValueError("kv_len must be a [B] int32 tensor")
    if mask_words is not None:
        W = (Lk + 31) // 32
        if mask_words.dtype != torch.int32 or not mask_words.is_contiguous() or mask_words.shape[-2:] != (Lq, W):
            raise ValueError("mask_words must be a contiguous int32 [..., Lq, ceil(Lk/32)] tensor (pack_mask)")
    for name, t, dt in (("idx", idx, torch.int32), ("score", score, torch.float32)):
        if t is not None and (t.dtype != dt or tuple(t.shape) != (B, H, Lq, topk) or not t.is_contiguous()):
            raise ValueError(f"{name} must be a contiguous [B,H,Lq,topk] {dt} tensor")
    rc = lib().topk_attn_fwd_masked(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, Lq, Lk, d, int(topk), int(chunk),
                                    int(bool(causal)), _ptr(kv_len), _ptr(mask_words), int(mask_batch_stride),
                                    int(mask_head_stride), _dtype_code(q), _ptr(idx), _ptr(score), _stream(stream))
    _check(rc, "topk_attn_fwd_masked")


def topk_vanilla_attn_fwd(q, k, v, out, chunk: int = 1024, causal: bool = False, kv_len=None,
                          stream=None) -> None:
    """Plain attention (Eq. 1) over every valid key, the comparison path (bf16, d 64 or 128)."""
    B, H, Lq, Lk, d = _attn_dims(q, k, v, out)
    if kv_len is not None and (kv_len.dtype != torch.int32 or tuple(kv_len.shape) != (B,)):
        raise ValueError("kv_len must be a [B] int32 tensor")
    rc = lib().topk_vanilla_attn_fwd(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, Lq, Lk, d, int(chunk),
                                     int(bool(causal)), _ptr(kv_len), _dtype_code(q), _stream(stream))
    _check(rc, "topk_vanilla_attn_fwd")


def _allocate(stream, make):
    """make()'s tuple of output tensors (or None) for a call on `stream`: memory of that stream, as on another's its kernels
    could write while work that was queued on the memory's last tenant still runs; and lent to the current stream, so that it is
    not given away under what reads the outputs there."""
    if stream is None:
        return make()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(0 if int(stream) == 1 else int(stream))  # 1: the default stream's other handle
    with torch.cuda.stream(stream):
        out = make()
    current = torch.cuda.current_stream()
    for t in out:
        if t is not None:
            t.record_stream(current)
    return out


def topk_vanilla_attn_workspace_bytes(B, H, Lq, Lk, d, dtype) -> int:
    return int(lib().topk_vanilla_attn_workspace_bytes(B, H, Lq, Lk, d, dtype))


def vanilla_attention(q, k, v, chunk: int = 1024, causal: bool = False, kv_len=None, stream=None):
    (out,) = _allocate(stream, lambda: (torch.empty_like(q),))
    topk_vanilla_attn_fwd(q, k, v, out, chunk, causal, kv_len, stream)
    return out


def topk_vanilla_ffn_fwd(x, W1, W2, out, chunk: int = 16384, stream=None) -> None:
    """The dense FF layer (Eq. 3 without top-k) in d_ff slices of `chunk` keys: out fp32 [N, d_model]."""
    N, dm, dff = _ffn_dims(x, W1, W2, out)
    rc = lib().topk_vanilla_ffn_fwd(_ptr(x), _ptr(W1), _ptr(W2), _ptr(out), N, dm, dff, int(chunk), _stream(stream))
    _check(rc, "topk_vanilla_ffn_fwd")


def topk_vanilla_ffn_workspace_bytes(N, d_model, d_ff, chunk) -> int:
    return int(lib().topk_vanilla_ffn_workspace_bytes(N, d_model, d_ff, chunk))


def vanilla_ffn(x, W1, W2, chunk: int = 16384, stream=None):
    (out,) = _allocate(stream, lambda: (torch.empty(x.shape[0], x.shape[1], dtype=torch.float32, device=x.device),))
    topk_vanilla_ffn_fwd(x, W1, W2, out, chunk, stream)
    return out


def topk_attn_fwd_host(q, k, v, out, topk: int, chunk: int = 1024, causal: bool = False, stream=None) -> None:
    """End-to-end call on HOST tensors (pinned is fastest); synchronises the stream."""
    B, H, Lq, Lk, d = _attn_dims(q, k, v, out)
    rc = lib().topk_attn_fwd_host(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, H, Lq, Lk, d, int(topk), int(chunk),
                                  int(bool(causal)), _dtype_code(q), _stream(stream))
    _check(rc, "topk_attn_fwd_host")


def _ffn_dims(x, W1, W2, out):
    for name, t in (("x", x), ("W1", W1), ("W2", W2), ("out", out)):
        if t.dim() != 2 or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous 2-D tensor")
    N, dm = x.shape
    dff = W1.shape[0]
    if tuple(W1.shape) != (dff, dm) or tuple(W2.shape) != (dff, dm) or tuple(out.shape) != (N, dm):
        raise ValueError("shape mismatch between x, W1, W2, out")
    if not (x.dtype == W1.dtype == W2.dtype == torch.bfloat16) or out.dtype != torch.float32:
        raise TypeError("x, W1, W2 must be bfloat16 and out float32")
    return N, dm, dff


def topk_ffn_fwd(x, W1, W2, out, topk: int, stream=None) -> None:
    """Eq. 3 with top-k: out [N, d_model] fp32 from x [N, d_model], W1/W2 [d_ff, d_model] bf16."""
    N, dm, dff = _ffn_dims(x, W1, W2, out)
    rc = lib().topk_ffn_fwd(_ptr(x), _ptr(W1), _ptr(W2), _ptr(out), N, dm, dff, int(topk), _stream(stream))
    _check(rc, "topk_ffn_fwd")


def topk_ffn_fwd_indices(x, W1, W2, out, topk: int, idx=None, score=None, stream=None) -> None:
    N, dm, dff = _ffn_dims(x, W1, W2, out)
    rc = lib().topk_ffn_fwd_indices(_ptr(x), _ptr(W1), _ptr(W2), _ptr(out), N, dm, dff, int(topk), _ptr(idx),
                                    _ptr(score), _stream(stream))
    _check(rc, "topk_ffn_fwd_indices")


def topk_ffn_fwd_host(x, W1, W2, out, topk: int, stream=None) -> None:
    N, dm, dff = _ffn_dims(x, W1, W2, out)
    rc = lib().topk_ffn_fwd_host(_ptr(x), _ptr(W1), _ptr(W2), _ptr(out), N, dm, dff, int(topk), _stream(stream))
    _check(rc, "topk_ffn_fwd_host")


# Size of the fixed scratch buffer of topk_ffn_fwd_noalloc (include/topk_attention.h).
TOPK_FFN_NOALLOC_SCRATCH_BYTES = 32 << 20


def topk_ffn_fwd_noalloc(x, W1, W2, out, topk: int, stream=None) -> None:
    """topk_ffn_fwd for callers that cannot allocate device memory at call time.

    Scratch comes from one fixed buffer inside the library instead of the
    stream-ordered pool (see the C header for the size limit and why calls
    that overlap on the GPU must be serialised).
    """
    N, dm, dff = _ffn_dims(x, W1, W2, out)
    rc = lib().topk_ffn_fwd_noalloc(_ptr(x), _ptr(W1), _ptr(W2), _ptr(out), N, dm, dff, int(topk), _stream(stream))
    _check(rc, "topk_ffn_fwd_noalloc")


def _cache_check(idx, score, rows_shape, topk):
    want = (*rows_shape, topk)
    for name, t, dt in (("idx", idx, torch.int32), ("score", score, torch.float32)):
        if t.dtype != dt or tuple(t.shape) != want or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {list(want)} {dt} tensor")


def topk_attn_bwd(q, k, v, dout, idx, score, dq, dk, dv, stream=None) -> None:
    """Backward pass of Eq. 4 for the cached kept set (Sec. 2.2): fp32 dq [B,H,Lq,d], dk/dv [B,H,Lk,d]."""
    B, H, Lq, Lk, d = _attn_dims(q, k, v, dout)
    topk = idx.shape[-1]
    _cache_check(idx, score, (B, H, Lq), topk)
    for name, t, shape in (("dq", dq, (B, H, Lq, d)), ("dk", dk, (B, H, Lk, d)), ("dv", dv, (B, H, Lk, d))):
        if t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {list(shape)} float32 tensor")
    rc = lib().topk_attn_bwd(_ptr(q), _ptr(k), _ptr(v), _ptr(dout), _ptr(idx), _ptr(score), _ptr(dq), _ptr(dk),
                             _ptr(dv), B, H, Lq, Lk, d, int(topk), _dtype_code(q), _stream(stream))
    _check(rc, "topk_attn_bwd")


def topk_ffn_bwd(x, W1, W2, dout, idx, score, dx, dW1, dW2, stream=None) -> None:
    """Backward pass of the top-k FF layer (Eq. 3) for the cached kept set: fp32 dx, dW1, dW2."""
    N, dm, dff = _ffn_dims(x, W1, W2, dout)
    topk = idx.shape[-1]
    _cache_check(idx, score, (N,), topk)
    for name, t, shape in (("dx", dx, (N, dm)), ("dW1", dW1, (dff, dm)), ("dW2", dW2, (dff, dm))):
        if t.dtype != torch.float32 or tuple(t.shape) != shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {list(shape)} float32 tensor")
    rc = lib().topk_ffn_bwd(_ptr(x), _ptr(W1), _ptr(W2), _ptr(dout), _ptr(idx), _ptr(score), _ptr(dx), _ptr(dW1),
                            _ptr(dW2), N, dm, dff, int(topk), _stream(stream))
    _check(rc, "topk_ffn_bwd")


def rope_tables(positions: int, rot: int, base: float = 10000.0, device="cuda"):
    """(cos, sin), fp32 [positions, rot / 2], of the angles p * base^(-2 i / rot), formed in fp64."""
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * float(base) ** (
        -torch.arange(rot // 2, dtype=torch.float64, device=device) * 2 / max(rot, 1))
    return angle.cos().float(), angle.sin().float()


_QK_PACK = struct.Struct("3P9q5P15i2f4x").pack  # topk_qk_args
_NO_STRIDE = (0, 0, 0)


def _qk_args(q, k, v, cos, sin, positions, q_weight, k_weight, eps, q_scale, sections, interleaved, normalize):
    """topk_qk_args as bytes, and (B, L, Hq, Hkv, d)."""
    sq, sk = q.stride(), k.stride()
    sv = None if v is None else v.stride()
    if len(sq) != 4 or sq[3] != 1 or len(sk) != 4 or sk[3] != 1 or (v is not None and (len(sv) != 4 or sv[3] != 1)):
        raise ValueError("q, k and v must be [B, L, H, d] tensors with contiguous rows")
    B, L, Hq, d = q.shape
    Hkv = k.shape[2]
    if tuple(k.shape) != (B, L, Hkv, d) or (v is not None and v.shape != k.shape):
        raise ValueError("shape mismatch between q, k, v")
    dtype = q.dtype
    if k.dtype != dtype or (v is not None and v.dtype != dtype):
        raise TypeError("q, k, v must share a dtype")
    if (cos.dtype != torch.float32 or sin.dtype != torch.float32 or cos.dim() != 2 or sin.shape != cos.shape
            or not (cos.is_contiguous() and sin.is_contiguous())):
        raise ValueError("cos and sin must be contiguous [positions, rot / 2] float32 tensors")
    rows, half = cos.shape
    sections = (half,) if sections is None else tuple(sections)
    axes = len(sections)
    if not 1 <= axes <= 4:
        raise ValueError("sections must name 1 to 4 axes")
    if positions is not None and (positions.dtype != torch.int32 or tuple(positions.shape) != (axes, B, L)
                                  or not positions.is_contiguous()):
        raise ValueError("positions must be a contiguous [axes, B, L] int32 tensor")
    for t in (q_weight, k_weight):
        if t is not None and (t.dtype != dtype or tuple(t.shape) != (d,) or not t.is_contiguous()):
            raise ValueError("q_weight and k_weight must be contiguous [d] tensors of q's dtype")
    args = _QK_PACK(q.data_ptr(), k.data_ptr(), _ptr(v) or 0, *sq[:3], *sk[:3], *(_NO_STRIDE if sv is None else sv[:3]),
                    _ptr(q_weight) or 0, _ptr(k_weight) or 0, cos.data_ptr(), sin.data_ptr(), _ptr(positions) or 0, rows, B, L, Hq, Hkv, d,
                    2 * half, axes, *sections, *_NO_STRIDE[axes - 1:], 1 if interleaved else 0, 1 if normalize else 0, _dtype_code(q), eps,
                    q_scale)
    return args, (B, L, Hq, Hkv, d)


def _written(name, t, shape, dtype) -> None:
    if t is not None and (t.dtype != dtype or tuple(t.shape) != shape or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous {list(shape)} {dtype} tensor")


def topk_qk_norm_rope_fwd(q, k, v, cos, sin, q_out, k_out, v_out, *, cache_start=None, positions=None, q_weight=None,
                          k_weight=None, eps: float = 1e-6, q_scale: float = 1.0, sections=None, interleaved: bool = False,
                          normalize: bool = True, stream=None) -> None:
    """RMS norm of each query and key head, rotation by position and q_scale: q [B,L,Hq,d], k/v
    [B,L,Hkv,d] (strided views allowed) into q_out [B,Hq,L,d] and k_out/v_out [B,Hkv,cap,d]; with
    cache_start ([B] int32) token t of batch b goes to row cache_start[b] + t of k_out/v_out."""
    a, (B, L, Hq, Hkv, d) = _qk_args(q, k, v, cos, sin, positions, q_weight, k_weight, eps, q_scale, sections, interleaved,
                                     normalize)
    cap = k_out.shape[2]
    _fits(cap)
    _written("q_out", q_out, (B, Hq, L, d), q.dtype)
    _written("k_out", k_out, (B, Hkv, cap, d), q.dtype)
    _written("v_out", v_out, (B, Hkv, cap, d), q.dtype)
    if cache_start is not None and (cache_start.dtype != torch.int32 or tuple(cache_start.shape) != (B,)
                                    or not cache_start.is_contiguous()):
        raise ValueError("cache_start must be a [B] int32 tensor")
    _on_gpu("q, k, v, the tables, positions, weights, outputs and cache_start", q, k, v, cos, sin, positions, q_weight, k_weight, q_out,
            k_out, v_out, cache_start)
    rc = lib().topk_qk_norm_rope_fwd(a, _ptr(q_out), _ptr(k_out), _ptr(v_out), cap, _ptr(cache_start),
                                     _stream(stream))
    _check(rc, "topk_qk_norm_rope_fwd")
    _changed(q_out, k_out, v_out)


def topk_qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, dqkv, dq_weight, dk_weight, *, positions=None, q_weight=None,
                          k_weight=None, eps: float = 1e-6, q_scale: float = 1.0, sections=None, interleaved: bool = False,
                          normalize: bool = True, stream=None) -> None:
    """Backward: dq [B,Hq,L,d], dk/dv [B,Hkv,L,d] (fp32 or bf16) into dqkv [B,L,Hq+2Hkv,d] (q's dtype; Hq+Hkv
    heads without dv) and the norms' weight gradients [d] fp32 (or None)."""
    a, (B, L, Hq, Hkv, d) = _qk_args(q, k, None, cos, sin, positions, q_weight, k_weight, eps, q_scale, sections, interleaved,
                                     normalize)
    _written("dq", dq, (B, Hq, L, d), dq.dtype)
    _written("dk", dk, (B, Hkv, L, d), dq.dtype)
    _written("dv", dv, (B, Hkv, L, d), dq.dtype)
    _written("dqkv", dqkv, (B, L, Hq + (Hkv if dv is None else 2 * Hkv), d), q.dtype)
    _written("dq_weight", dq_weight, (d,), torch.float32)
    _written("dk_weight", dk_weight, (d,), torch.float32)
    _on_gpu("gradients, q, k, the tables, positions, weights and outputs", q, k, cos, sin, positions, q_weight, k_weight, dq, dk, dv, dqkv,
            dq_weight, dk_weight)
    rc = lib().topk_qk_norm_rope_bwd(a, _ptr(dq), _ptr(dk), _ptr(dv), _dtype_code(dq), _ptr(dqkv), _ptr(dq_weight),
                                     _ptr(dk_weight), _stream(stream))
    _check(rc, "topk_qk_norm_rope_bwd")
    _changed(dqkv, dq_weight, dk_weight)


def topk_qk_norm_rope_bwd_workspace_bytes(B, L, Hq, Hkv, d) -> int:
    return int(lib().topk_qk_norm_rope_bwd_workspace_bytes(B, L, Hq, Hkv, d))


def _fits(*sizes) -> None:
    """Refuses sizes that the C ABI's ints cannot hold: ctypes would pass their low 32 bits."""
    if max(sizes) >= 1 << 31:
        raise ValueError("sizes must be below 2^31")


def _act_code(act: str) -> int:
    if act not in ACTIVATIONS:
        raise ValueError(f"act must be one of {sorted(ACTIVATIONS)}")
    return ACTIVATIONS[act]


def _bf16(name, t, shape) -> int:
    """t's address; t is None or a contiguous bf16 tensor of the shape."""
    if t is None:
        return 0
    if t.dtype != torch.bfloat16 or tuple(t.shape) != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} torch.bfloat16 tensor")
    return t.data_ptr()


def topk_linear_fwd(x, w, y, bias=None, residual=None, preact=None, act: str = "none", stream=None) -> None:
    """y = act(x w^T + bias) + residual: x [M,K], w [N,K], bias [N], residual, y and preact (z, written) [M,N], bf16."""
    (M, K), N = x.shape, w.shape[0]
    _fits(M, N, K)
    out = (M, N)
    tensors = (_bf16("x", x, (M, K)), _bf16("w", w, (N, K)), _bf16("bias", bias, (N,)), _bf16("residual", residual, out),
               _bf16("y", y, out), _bf16("preact", preact, out))
    code = _act_code(act)
    _on_gpu("x, w, bias, residual, y and preact", x, w, bias, residual, y, preact)
    rc = lib().topk_linear_fwd(*tensors, M, N, K, code, _stream(stream))
    _check(rc, "topk_linear_fwd")
    _changed(y, preact)


def topk_linear_bwd(dy, x, w, dx, dw, db, preact=None, act: str = "none", stream=None) -> None:
    """Gradients of topk_linear_fwd: dx [M,K] bf16, dw [N,K] and db [N] bf16 or fp32 (one dtype); None where not wanted."""
    (M, K), N = x.shape, w.shape[0]
    _fits(M, N, K)
    first = dw if dw is not None else db
    dtype = torch.bfloat16 if first is None else first.dtype
    _written("dw", dw, (N, K), dtype)
    _written("db", db, (N,), dtype)
    tensors = (_bf16("dy", dy, (M, N)), _bf16("x", x, (M, K)), _bf16("w", w, (N, K)), _bf16("preact", preact, (M, N)),
               _bf16("dx", dx, (M, K)), _ptr(dw), _ptr(db))
    code, grad_code = _act_code(act), TOPK_BF16 if first is None else _dtype_code(first)
    _on_gpu("dy, x, w, preact, dx, dw and db", x, w, dy, preact, dx, dw, db)
    rc = lib().topk_linear_bwd(*tensors, M, N, K, code, grad_code, _stream(stream))
    _check(rc, "topk_linear_bwd")
    _changed(dx, dw, db)


def topk_linear_workspace_bytes(M, N, K) -> int:
    return int(lib().topk_linear_workspace_bytes(M, N, K))


def topk_linear_bwd_workspace_bytes(M, N, K, act: str = "none") -> int:
    return int(lib().topk_linear_bwd_workspace_bytes(M, N, K, _act_code(act)))


def _whole(name, t, shape) -> int:
    """The bits of t's whole numbers; t is a contiguous int32 or int64 tensor of the shape."""
    if t.dtype not in (torch.int32, torch.int64) or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {list(shape)} int32 or int64 tensor")
    return 32 if t.dtype == torch.int32 else 64


def _embedding_args(ids, weight):
    """(tokens, bits of an id, rows, D, dtype code) of a lookup."""
    if weight.dim() != 2 or not weight.is_contiguous():
        raise ValueError("weight must be a contiguous [rows, D] tensor")
    rows, D = weight.shape
    N = ids.numel()
    _fits(N, rows, D)
    return N, _whole("ids", ids, ids.shape), rows, D, _dtype_code(weight)


def topk_embedding_fwd(ids, weight, out, scale: float = 1.0, stream=None) -> None:
    """out [*ids.shape, D] = scale weight[ids]: ids int32 or int64 (a negative one is padding and gives zeros), weight
    [rows, D] and out fp32 or bf16."""
    N, bits, rows, D, code = _embedding_args(ids, weight)
    _written("out", out, (*ids.shape, D), weight.dtype)
    _on_gpu("ids, weight and out", weight, ids, out)
    rc = lib().topk_embedding_fwd(ids.data_ptr(), bits, weight.data_ptr(), out.data_ptr(), N, rows, D, scale, code, _stream(stream))
    _check(rc, "topk_embedding_fwd")
    _changed(out)


def topk_embedding_bwd(dy, ids, dweight, scale: float = 1.0, accumulate: bool = False, stream=None) -> None:
    """dweight [rows, D] (fp32 or bf16) = scale x the sums of dy [*ids.shape, D] over each id's tokens, or with accumulate
    that added to it."""
    if dweight.dim() != 2 or not dweight.is_contiguous():
        raise ValueError("dweight must be a contiguous [rows, D] tensor")
    rows, D = dweight.shape
    N = ids.numel()
    _fits(N, rows, D)
    bits = _whole("ids", ids, ids.shape)
    _written("dy", dy, (*ids.shape, D), dy.dtype)
    code, grad_code = _dtype_code(dy), _dtype_code(dweight)
    _on_gpu("dy, ids and dweight", dweight, ids, dy)
    rc = lib().topk_embedding_bwd(_ptr(dy), _ptr(ids), bits, _ptr(dweight), N, rows, D, scale, 1 if accumulate else 0, code, grad_code,
                                  _stream(stream))
    _check(rc, "topk_embedding_bwd")
    _changed(dweight)


def topk_embedding_bwd_workspace_bytes(N, rows, D) -> int:
    return int(lib().topk_embedding_bwd_workspace_bytes(N, rows, D))


def _rows_of(name, t):
    """(N, V, row stride) of a [N, V] tensor with contiguous rows."""
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        raise ValueError(f"{name} must be a [N, V] tensor with contiguous rows")
    N, V = t.shape
    stride = t.stride(0) if N > 1 else V
    if stride < V:
        raise ValueError(f"the rows of {name} must not overlap")
    _fits(N, V, stride)
    return N, V, stride


def _logprobs_args(logits, targets):
    """(N, V, row stride, bits of a target, dtype code)."""
    N, V, stride = _rows_of("logits", logits)
    return N, V, stride, 32 if targets is None else _whole("targets", targets, (N,)), _dtype_code(logits)


def topk_token_logprobs_fwd(logits, targets=None, logp=None, entropy=None, lse=None, top_logp=None, top_ids=None, scale: float = 1.0,
                            stream=None) -> None:
    """Of each row of logits [N, V] (fp32 or bf16; rows may be strided) times scale: logp [N] of the targets ([N], int32 or int64,
    negative: none), entropy [N], lse [N], and the largest tokens' top_logp and top_ids (int32) [N, top]; None where not wanted."""
    N, V, stride, bits, code = _logprobs_args(logits, targets)
    top = 0 if top_ids is None else top_ids.shape[1]
    for name, t in (("logp", logp), ("entropy", entropy), ("lse", lse)):
        _written(name, t, (N,), torch.float32)
    _written("top_logp", top_logp, (N, top), torch.float32)
    _written("top_ids", top_ids, (N, top), torch.int32)
    _on_gpu("logits, targets and outputs", logits, targets, logp, entropy, lse, top_logp, top_ids)
    rc = lib().topk_token_logprobs_fwd(_ptr(logits), stride, _ptr(targets), bits, scale, top, _ptr(logp), _ptr(entropy), _ptr(lse),
                                       _ptr(top_logp), _ptr(top_ids), N, V, code, _stream(stream))
    _check(rc, "topk_token_logprobs_fwd")
    _changed(logp, entropy, lse, top_logp, top_ids)


def topk_token_logprobs_bwd(logits, lse, dlogits, targets=None, dlogp=None, entropy=None, dentropy=None, top_ids=None, dtop=None,
                            scale: float = 1.0, stream=None) -> None:
    """dlogits [N, V] (logits' dtype; may be logits itself) from the gradients of topk_token_logprobs_fwd's outputs: dlogp [N] with
    targets, dentropy [N] with entropy, dtop [N, top] with top_ids, all fp32."""
    N, V, stride = _rows_of("logits", logits)
    if dlogits.shape != logits.shape or dlogits.dtype != logits.dtype:
        raise ValueError("dlogits must have the shape and dtype of logits")
    _, _, out_stride = _rows_of("dlogits", dlogits)
    top = 0 if top_ids is None else top_ids.shape[1]
    bits = 32 if targets is None else _whole("targets", targets, (N,))
    for name, t in (("lse", lse), ("dlogp", dlogp), ("entropy", entropy), ("dentropy", dentropy)):
        _written(name, t, (N,), torch.float32)
    _written("top_ids", top_ids, (N, top), torch.int32)
    _written("dtop", dtop, (N, top), torch.float32)
    code = _dtype_code(logits)
    _on_gpu("logits, dlogits, targets, lse, entropy and gradients", logits, dlogits, lse, targets, dlogp, entropy, dentropy, top_ids, dtop)
    rc = lib().topk_token_logprobs_bwd(_ptr(logits), stride, _ptr(lse), _ptr(targets), bits, _ptr(dlogp), _ptr(entropy), _ptr(dentropy),
                                       _ptr(top_ids), _ptr(dtop), top, scale, _ptr(dlogits), out_stride, N, V, code, _stream(stream))
    _check(rc, "topk_token_logprobs_bwd")
    _changed(dlogits)


_PROMPT_PACK = struct.Struct("4P6q2P8i").pack  # topk_prompt_args
_TREE_PACK = struct.Struct("4P9q2Pq6i").pack  # topk_tree_args


def _heads_bf16(dims, **tensors) -> None:
    for name, t in tensors.items():
        if t.dtype != torch.bfloat16:
            raise TypeError(f"{name} must be bfloat16")
        shape = t.shape
        if len(shape) != dims or (t.stride(-1) != 1 and shape[-1] > 1):
            raise ValueError(f"{name} must be a {dims}-dimensional tensor with contiguous rows")
        if max(shape) >= 1 << 31:
            _fits(*shape)


def _starts(name, t) -> None:
    if t.dtype != torch.int32 or t.dim() != 1 or t.shape[0] < 2 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous [sequences + 1] int32 tensor")


def topk_prompt_attn_fwd(q, k, v, out, q_starts, k_starts=None, causal: bool = True, clear_rest: bool = False, stream=None) -> None:
    """Plain attention over packed sequences: q [Tq,Hq,d], k and v [Tk,Hkv,d] (bf16, strided views allowed), sequence b's queries in
    rows q_starts[b] to q_starts[b + 1] - 1 ([B + 1] int32), its keys by k_starts likewise (None: q_starts); out [Tq,Hq,d], whose
    rows of no sequence are left alone, or zeros with clear_rest."""
    _heads_bf16(3, q=q, k=k, v=v)
    (Tq, Hq, d), (Tk, Hkv, dk) = q.shape, k.shape
    if dk != d or v.shape != k.shape:
        raise ValueError("shape mismatch between q, k, v")
    _written("out", out, (Tq, Hq, d), torch.bfloat16)
    _starts("q_starts", q_starts)
    if k_starts is not None:
        _starts("k_starts", k_starts)
        if k_starts.shape != q_starts.shape:
            raise ValueError("q_starts and k_starts must have the same length")
    elif Tk != Tq:
        raise ValueError("keys in other rows than the queries need k_starts")
    _on_gpu("q, k, v, out and the starts", q, k, v, out, q_starts, k_starts)
    args = _PROMPT_PACK(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), *q.stride()[:2], *k.stride()[:2], *v.stride()[:2],
                        q_starts.data_ptr(), _ptr(k_starts) or 0, q_starts.shape[0] - 1, Tq, Tk, Hq, Hkv, d, 1 if causal else 0,
                        1 if clear_rest else 0)
    _check(lib().topk_prompt_attn_fwd(args, _stream(stream)), "topk_prompt_attn_fwd")
    _changed(out)


def topk_prompt_attn_workspace_bytes(d) -> int:
    return int(lib().topk_prompt_attn_workspace_bytes(d))


def topk_tree_attn_fwd(q, keys, values, out, kv_len, tree=None, stream=None) -> None:
    """Plain attention of T drafted tokens of each sequence, q [B,Hq,T,d], over caches [B,Hkv,cap,d] (bf16, strided views allowed) of
    kv_len[b] tokens ([B] int32) followed by the drafted ones; tree [B or 1, T] int64 has the drafted tokens that each one reads
    (tree_mask), None: those up to it."""
    _heads_bf16(4, q=q, keys=keys, values=values)
    B, Hq, T, d = q.shape
    Hkv, cap = keys.shape[1:3]
    if keys.shape != (B, Hkv, cap, d) or values.shape != keys.shape:
        raise ValueError("shape mismatch between q, keys, values")
    _written("out", out, (B, Hq, T, d), torch.bfloat16)
    if kv_len.dtype != torch.int32 or kv_len.shape != (B,) or not kv_len.is_contiguous():
        raise ValueError("kv_len must be a contiguous [B] int32 tensor")
    if tree is not None and (tree.dtype != torch.int64 or tree.dim() != 2 or tree.shape[0] not in (1, B) or tree.shape[1] != T
                             or not tree.is_contiguous()):
        raise ValueError("tree must be a contiguous [B or 1, T] int64 tensor")
    _on_gpu("q, keys, values, out, kv_len and tree", q, keys, values, out, kv_len, tree)
    args = _TREE_PACK(q.data_ptr(), keys.data_ptr(), values.data_ptr(), out.data_ptr(), *q.stride()[:3], *keys.stride()[:3],
                      *values.stride()[:3], kv_len.data_ptr(), _ptr(tree) or 0, 0 if tree is None or tree.shape[0] == 1 else T, B, T, Hq, Hkv,
                      cap, d)
    _check(lib().topk_tree_attn_fwd(args, _stream(stream)), "topk_tree_attn_fwd")
    _changed(out)


def topk_attn_bwd_workspace_bytes(B, H, Lq, Lk, d, topk, dtype) -> int:
    return int(lib().topk_attn_bwd_workspace_bytes(B, H, Lq, Lk, d, topk, dtype))


def topk_ffn_bwd_workspace_bytes(N, d_model, d_ff, topk) -> int:
    return int(lib().topk_ffn_bwd_workspace_bytes(N, d_model, d_ff, topk))


def topk_attn_workspace_bytes(B, H, Lq, Lk, d, topk, chunk, dtype) -> int:
    return int(lib().topk_attn_workspace_bytes(B, H, Lq, Lk, d, topk, chunk, dtype))


def topk_ffn_workspace_bytes(N, d_model, d_ff, topk) -> int:
    return int(lib().topk_ffn_workspace_bytes(N, d_model, d_ff, topk))


def topk_check(stream=None) -> None:
    """Synchronise and raise if a kernel recorded a device-side error since the last check."""
    _check(lib().topk_check(_stream(stream)), "topk_check")


def topk_last_launch_count() -> int:
    return int(lib().topk_last_launch_count())


def topk_set_wait_limit_us(us: int) -> int:
    return int(lib().topk_set_wait_limit_us(int(us)))


def topk_pool_usage(reset_high: bool = False) -> tuple[int, int]:
    """(bytes in use at most since the last reset, bytes reserved now) of the library's own
    device-memory pool on the current device."""
    hi, res = ctypes.c_size_t(0), ctypes.c_size_t(0)
    _check(lib().topk_pool_usage(ctypes.byref(hi), ctypes.byref(res), int(bool(reset_high))), "topk_pool_usage")
    return int(hi.value), int(res.value)


def topk_pool_trim() -> None:
    """Hand the pool's reserved but unused device memory back (synchronise the streams first)."""
    _check(lib().topk_pool_trim(), "topk_pool_trim")


# convenience wrappers that allocate the outputs ---------------------------------------------

def _kept(rows, topk: int, device):
    """Empty lists of the kept indices and scores."""
    return (torch.empty(*rows, topk, dtype=torch.int32, device=device), torch.empty(*rows, topk, dtype=torch.float32, device=device))


def attention(q, k, v, topk: int, chunk: int = 1024, causal: bool = False, return_indices: bool = False,
              stream=None, kv_len=None, mask=None):
    """Top-k attention; kv_len ([B] int32) and mask (bool [B|1, H|1, Lq, Lk], True = valid) add Eq. 2's
    general masks."""
    B, H, Lq, _ = q.shape
    out, idx, score = _allocate(stream, lambda: (
        torch.empty_like(q), *(_kept((B, H, Lq), topk, q.device) if return_indices else (None, None))))
    if kv_len is not None or mask is not None:
        strides = [0, 0]

        def pack():  # on the call's stream, as the kernel that reads the words
            words, *strides[:] = pack_mask(mask)
            return (words,)

        (words,) = _allocate(stream, pack) if mask is not None else (None,)
        topk_attn_fwd_masked(q, k, v, out, topk, chunk, causal, kv_len, words, *strides, idx, score, stream)
    elif return_indices:
        topk_attn_fwd_indices(q, k, v, out, topk, chunk, causal, idx, score, stream)
    else:
        topk_attn_fwd(q, k, v, out, topk, chunk, causal, stream)
    return (out, idx, score) if return_indices else out


def ffn(x, W1, W2, topk: int, return_indices: bool = False, stream=None):
    out, idx, score = _allocate(stream, lambda: (
        torch.empty(x.shape[0], x.shape[1], dtype=torch.float32, device=x.device),
        *(_kept((x.shape[0],), topk, x.device) if return_indices else (None, None))))
    if not return_indices:
        topk_ffn_fwd(x, W1, W2, out, topk, stream)
        return out
    topk_ffn_fwd_indices(x, W1, W2, out, topk, idx, score, stream)
    return out, idx, score


def attention_bwd(q, k, v, dout, idx, score, stream=None):
    """Gradients (dq, dk, dv), fp32, of top-k attention for the cache (idx, score) of attention(...,
    return_indices=True)."""
    dq, dk, dv = _allocate(stream, lambda: tuple(torch.empty(t.shape, dtype=torch.float32, device=t.device) for t in (q, k, v)))
    topk_attn_bwd(q, k, v, dout, idx, score, dq, dk, dv, stream)
    return dq, dk, dv


def ffn_bwd(x, W1, W2, dout, idx, score, stream=None):
    """Gradients (dx, dW1, dW2), fp32, of the top-k FF layer for the cache of ffn(..., return_indices=True)."""
    dx, dW1, dW2 = _allocate(stream, lambda: tuple(torch.empty(t.shape, dtype=torch.float32, device=t.device) for t in (x, W1, W2)))
    topk_ffn_bwd(x, W1, W2, dout, idx, score, dx, dW1, dW2, stream)
    return dx, dW1, dW2


def qk_norm_rope(q, k, v, cos, sin, cache=None, cache_start=None, stream=None, **options):
    """Norm, rotation and scale of a projection's q [B,L,Hq,d] and k, v [B,L,Hkv,d] for the attention:
    (q [B,Hq,L,d], k, v [B,Hkv,L,d]).  With cache = (keys, values), each [B,Hkv,cap,d], k and v are written
    into it from row cache_start[b] on ([B] int32) and the caches are returned.  v may be None (without a
    cache).  Options as topk_qk_norm_rope_fwd."""
    B, L, Hq, d = q.shape
    if cache is not None:
        if cache_start is None or v is None:
            raise ValueError("a cache needs cache_start and v")
        (qo,), (ko, vo) = _allocate(stream, lambda: (q.new_empty((B, Hq, L, d)),)), cache
    else:
        if cache_start is not None:
            raise ValueError("cache_start needs a cache")
        kv = (B, k.shape[2], L, d)
        qo, ko, vo = _allocate(stream, lambda: (q.new_empty((B, Hq, L, d)), q.new_empty(kv), None if v is None else q.new_empty(kv)))
    topk_qk_norm_rope_fwd(q, k, v, cos, sin, qo, ko, vo, cache_start=cache_start, stream=stream, **options)
    return qo, ko, vo


def qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, stream=None, **options):
    """Gradients (dqkv [B,L,Hq+2Hkv,d] packed in q's dtype, dq_weight, dk_weight fp32 [d]) of qk_norm_rope; the weight
    gradients are None with normalize=False.  dv may be None."""
    B, L, Hq, d = q.shape
    Hkv = k.shape[2]
    dqkv, both = _allocate(stream, lambda: (
        torch.empty(B, L, Hq + (Hkv if dv is None else 2 * Hkv), d, dtype=q.dtype, device=q.device),
        torch.empty(2, d, dtype=torch.float32, device=q.device) if options.get("normalize", True) else None))
    gq, gk = (None, None) if both is None else (both[0], both[1])
    topk_qk_norm_rope_bwd(dq, dk, dv, q, k, cos, sin, dqkv, gq, gk, stream=stream, **options)
    return dqkv, gq, gk


def linear(x, w, bias=None, act: str = "none", residual=None, return_preact: bool = False, stream=None):
    """act(x w^T + bias) + residual for x [M,K] and w [N,K] (bf16); with return_preact also x w^T + bias, which
    linear_bwd takes for an activation."""
    shape = (x.shape[0], w.shape[0])
    y, z = _allocate(stream, lambda: (x.new_empty(shape), x.new_empty(shape) if return_preact else None))
    topk_linear_fwd(x, w, y, bias, residual, z, act, stream)
    return (y, z) if return_preact else y


def linear_bwd(dy, x, w, preact=None, act: str = "none", bias: bool = False, need_dx: bool = True, need_dw: bool = True,
               grad_dtype=torch.bfloat16, stream=None):
    """Gradients (dx, dw, db) of linear; the residual's is dy.  dw and db are of grad_dtype; None where not wanted."""
    dx, dw, db = _allocate(stream, lambda: (
        torch.empty_like(x) if need_dx else None, torch.empty(w.shape, dtype=grad_dtype, device=w.device) if need_dw else None,
        torch.empty(w.shape[0], dtype=grad_dtype, device=w.device) if bias else None))
    topk_linear_bwd(dy, x, w, dx, dw, db, preact, act, stream)
    return dx, dw, db


def embedding(ids, weight, scale: float = 1.0, stream=None):
    """scale weight[ids], [*ids.shape, D]; a negative id is padding: zeros."""
    # a few tokens take 2 us on the GPU: what was made here is not checked again
    N, bits, rows, D, code = _embedding_args(ids, weight)
    _on_gpu("ids and weight", weight, ids)
    (out,) = _allocate(stream, lambda: (torch.empty((*ids.shape, D), dtype=weight.dtype, device=weight.device),))
    if N:
        rc = lib().topk_embedding_fwd(ids.data_ptr(), bits, weight.data_ptr(), out.data_ptr(), N, rows, D, scale, code, _stream(stream))
        _check(rc, "topk_embedding_fwd")
    return out


def embedding_bwd(dy, ids, rows: int, scale: float = 1.0, grad_dtype=None, into=None, stream=None):
    """The gradient [rows, D] of embedding's weight, of grad_dtype (None: dy's), or added to `into` (returned)."""
    dtype = dy.dtype if grad_dtype is None else grad_dtype
    shape = (rows, dy.shape[-1])
    if into is not None:
        _written("into", into, shape, into.dtype if grad_dtype is None else grad_dtype)
        dweight = into
    elif ids.numel():
        (dweight,) = _allocate(stream, lambda: (torch.empty(shape, dtype=dtype, device=dy.device),))
    else:
        (dweight,) = _allocate(stream, lambda: (torch.zeros(shape, dtype=dtype, device=dy.device),))
    if ids.numel():
        topk_embedding_bwd(dy, ids, dweight, scale, into is not None, stream)
    return dweight


class TokenLogProbs(NamedTuple):
    """token_logprobs' outputs; None where not asked for."""
    logp: Optional[torch.Tensor]  # [N], of the targets
    entropy: torch.Tensor  # [N]
    lse: torch.Tensor  # [N]
    top_logp: Optional[torch.Tensor]  # [N, top], largest first
    top_ids: Optional[torch.Tensor]  # [N, top] int32


def token_logprobs(logits, targets=None, top: int = 0, scale: float = 1.0, stream=None) -> TokenLogProbs:
    """Log probabilities, in fp32, under softmax(scale logits) for logits [N, V]: of the targets ([N]; negative: none, 0), the
    entropy, the log of the sum, and the `top` likeliest tokens (ties to the lower id; a masked token, -inf, is none: id -1)."""
    N, V, stride, bits, code = _logprobs_args(logits, targets)
    _on_gpu("logits and targets", logits, targets)
    device = logits.device

    def outputs():
        f32 = torch.float32
        return (None if targets is None else torch.empty(N, dtype=f32, device=device), torch.empty(N, dtype=f32, device=device),
                torch.empty(N, dtype=f32, device=device), torch.empty((N, top), dtype=f32, device=device) if top else None,
                torch.empty((N, top), dtype=torch.int32, device=device) if top else None)

    out = logp, entropy, lse, best, ids = _allocate(stream, outputs)
    if N:  # what was made here is not checked again
        rc = lib().topk_token_logprobs_fwd(logits.data_ptr(), stride, _ptr(targets), bits, scale, top, _ptr(logp), entropy.data_ptr(),
                                           lse.data_ptr(), _ptr(best), _ptr(ids), N, V, code, _stream(stream))
        _check(rc, "topk_token_logprobs_fwd")
    return TokenLogProbs(*out)


def token_logprobs_bwd(logits, lse, targets=None, dlogp=None, entropy=None, dentropy=None, top_ids=None, dtop=None, scale: float = 1.0,
                       out=None, stream=None):
    """The gradient of logits (their dtype) from those of token_logprobs' outputs; dentropy goes with its entropy, dtop with its
    top_ids.  out: where to write it; logits itself is allowed."""
    if dentropy is None:
        entropy = None
    if dlogp is None:
        targets = None
    if dtop is None:
        top_ids = None
    if out is None:
        (out,) = _allocate(stream, lambda: (torch.empty(logits.shape, dtype=logits.dtype, device=logits.device),))
    if logits.shape[0]:
        topk_token_logprobs_bwd(logits, lse, out, targets, dlogp, entropy, dentropy, top_ids, dtop, scale, stream)
    return out


def prompt_attention(q, k, v, q_starts, k_starts=None, causal: bool = True, out=None, stream=None):
    """Plain attention over packed sequences (topk_prompt_attn_fwd): [Tq,Hq,d], zeros in the rows of no sequence; with out those
    rows are left alone."""
    given = out is not None
    if not given:
        (out,) = _allocate(stream, lambda: (torch.empty(q.shape, dtype=q.dtype, device=q.device),))
    if q.shape[0] and k.shape[0]:
        topk_prompt_attn_fwd(q, k, v, out, q_starts, k_starts, causal, not given, stream)
    elif q.shape[0]:
        raise ValueError("no keys")
    return out


def tree_mask(parents: torch.Tensor) -> torch.Tensor:
    """Drafted tokens' words for tree_attention from their parents [.., T] (T up to 64): parents[i] < i, or negative where token
    i follows the cache directly.  Bit j of word i: token j is i or one of its ancestors."""
    T = parents.shape[-1]
    if T > 64:
        raise ValueError("at most 64 drafted tokens")
    i = torch.arange(T, device=parents.device)
    step = (parents[..., None] == i) | (i[:, None] == i)  # to the parent, or to oneself
    reach = step.float()
    for _ in range(6):  # paths of up to 64 steps
        reach = (reach @ reach).clamp_max(1)
    words = torch.where(i == 63, torch.iinfo(torch.int64).min, 1 << i.clamp_max(62))
    return (reach.long() * words).sum(-1)


def tree_attention(q, keys, values, kv_len, tree=None, stream=None):
    """Plain attention of drafted tokens over caches (topk_tree_attn_fwd): [B,Hq,T,d].  T = 1: ordinary decoding."""
    (out,) = _allocate(stream, lambda: (torch.empty(q.shape, dtype=q.dtype, device=q.device),))
    if out.numel():
        topk_tree_attn_fwd(q, keys, values, out, kv_len, tree, stream)
    return out
