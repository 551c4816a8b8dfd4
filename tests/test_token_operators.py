"""Embedding, token log probabilities and the packed and cached attention refuse bad arguments before anything is launched (no GPU
needed), and what of them runs on the CPU."""
import ctypes

import pytest
import torch

from paper_2106_06899_gb300 import build
from paper_2106_06899_gb300 import topk as T

BF = torch.bfloat16
LONG = 2 ** 32 + 16


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return T.lib()


@pytest.fixture
def no_library(monkeypatch):
    def called(*_):
        raise AssertionError("the library was called")

    monkeypatch.setattr(T, "lib", called)


@pytest.fixture
def anywhere(no_library, monkeypatch):
    monkeypatch.setattr(T, "_on_gpu", lambda *a: None)


def _meta(*shape, dtype=BF):
    return torch.empty(*shape, dtype=dtype, device="meta")


def test_embedding_arguments(lib):
    def fwd(ids=16, bits=64, w=16, out=16, N=4, rows=8, D=8, scale=1.0, dt=1):
        return lib.topk_embedding_fwd(ids, bits, w, out, N, rows, D, scale, dt, None)

    def bwd(dy=16, ids=16, bits=64, dw=16, N=4, rows=8, D=8, scale=1.0, acc=0, dt=1, gdt=0):
        return lib.topk_embedding_bwd(dy, ids, bits, dw, N, rows, D, scale, acc, dt, gdt, None)

    for kw, code in ((dict(ids=None), -1), (dict(bits=16), -1), (dict(N=0), -1), (dict(rows=-1), -1), (dict(D=0), -1), (dict(dt=2), -1),
                     (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(ids=20), -2), (dict(ids=18, bits=32), -2),
                     (dict(N=(1 << 30) + 1), -2), (dict(D=(1 << 20) + 1), -2)):
        assert fwd(**kw) == code, kw
        assert bwd(**kw) == code, kw
    for kw, code in ((dict(w=None), -1), (dict(out=None), -1), (dict(w=24), -2), (dict(out=8), -2)):
        assert fwd(**kw) == code, kw
    for kw, code in ((dict(dy=None), -1), (dict(dw=None), -1), (dict(acc=2), -1), (dict(gdt=3), -1), (dict(dy=24), -2), (dict(dw=24), -2)):
        assert bwd(**kw) == code, kw
    assert T.topk_embedding_bwd_workspace_bytes(0, 8, 8) == 0
    # the sorted ids and two rows for every 32 of them: linear in the ids, nothing for each row of the table
    size = T.topk_embedding_bwd_workspace_bytes
    assert 0 < size(1 << 15, 1 << 17, 768) <= (1 << 15) * 16 + (1 << 10) * 2 * 768 * 4 + (1 << 22)
    assert size(1 << 15, 1 << 17, 768) == size(1 << 15, 1 << 12, 768)


def test_logprobs_arguments(lib):
    def fwd(x=16, stride=8, t=16, bits=64, scale=1.0, top=2, logp=16, ent=16, lse=16, tl=16, ti=16, N=4, V=8, dt=1):
        return lib.topk_token_logprobs_fwd(x, stride, t, bits, scale, top, logp, ent, lse, tl, ti, N, V, dt, None)

    def bwd(x=16, stride=8, lse=16, t=16, bits=64, dl=16, ent=16, de=16, ti=16, dt_=16, top=2, scale=1.0, out=64, ostride=8, N=4, V=8, dt=1):
        return lib.topk_token_logprobs_bwd(x, stride, lse, t, bits, dl, ent, de, ti, dt_, top, scale, out, ostride, N, V, dt, None)

    for kw, code in ((dict(x=None), -1), (dict(stride=7), -1), (dict(N=0), -1), (dict(V=-2), -1), (dict(dt=3), -1), (dict(top=-1), -1), (dict(scale=0.0), -1),
                     (dict(scale=-1.0), -1), (dict(scale=float("inf")), -1), (dict(scale=float("nan")), -1), (dict(bits=8), -1), (dict(top=129), -2),
                     (dict(x=17), -2), (dict(x=18, dt=0), -2), (dict(t=12), -2), (dict(lse=18), -2), (dict(V=(1 << 30) + 1, stride=1 << 31, ostride=1 << 31), -2)):
        assert bwd(**kw) == code, kw
        kw.pop("ostride", None)
        assert fwd(**kw) == code, kw
    for kw, code in ((dict(t=None), -1), (dict(ti=None), -1), (dict(tl=None), -1), (dict(top=0), -1), (dict(logp=None, ent=None, lse=None, tl=None, ti=None, top=0), -1),
                     (dict(ti=18), -2)):
        assert fwd(**kw) == code, kw
    for kw, code in ((dict(lse=None), -1), (dict(out=None), -1), (dict(ostride=7), -1), (dict(t=None), -1), (dict(dl=None), -1), (dict(ent=None), -1), (dict(de=None), -1),
                     (dict(ti=None), -1), (dict(top=0), -1), (dict(t=None, dl=None, ent=None, de=None, ti=None, dt_=None, top=0), -1), (dict(out=16, ostride=9), -1),
                     (dict(out=65), -2), (dict(de=18), -2)):
        assert bwd(**kw) == code, kw


class _Prompt(ctypes.Structure):
    """topk_prompt_args"""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v", "out")] + [(n, ctypes.c_longlong * 2) for n in ("q_stride", "k_stride", "v_stride")]
                + [(n, ctypes.c_void_p) for n in ("q_starts", "k_starts")]
                + [(n, ctypes.c_int) for n in ("B", "Tq", "Tk", "Hq", "Hkv", "d", "causal", "clear_rest")])


class _Tree(ctypes.Structure):
    """topk_tree_args"""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "keys", "values", "out")] + [(n, ctypes.c_longlong * 3) for n in ("q_stride", "key_stride", "value_stride")]
                + [(n, ctypes.c_void_p) for n in ("kv_len", "tree")] + [("tree_stride", ctypes.c_longlong)]
                + [(n, ctypes.c_int) for n in ("B", "T", "Hq", "Hkv", "cap", "d")])


@pytest.mark.parametrize("kind,pack", [(_Prompt, T._PROMPT_PACK), (_Tree, T._TREE_PACK)])
def test_records_match_the_header(kind, pack):
    # the binding packs the records as bytes; different values through the header's layout
    fields, values = [], []
    for name, of in kind._fields_:
        n = getattr(of, "_length_", 0)
        here = [len(values) + 1 + i for i in range(n or 1)]
        values += here
        fields.append(tuple(here) if n else here[0])
    assert bytes(kind(*fields)) == pack(*values)


def _prompt(**kw):
    a = dict(q=16, k=16, v=16, out=16, q_stride=(256, 64), k_stride=(128, 64), v_stride=(128, 64), q_starts=16, k_starts=None, B=2, Tq=8, Tk=8, Hq=4, Hkv=2, d=64,
             causal=1, clear_rest=0)
    a.update(kw)
    return ctypes.byref(_Prompt(*[a[n] for n, _ in _Prompt._fields_]))


def _tree(**kw):
    a = dict(q=16, keys=16, values=16, out=16, q_stride=(256, 64, 64), key_stride=(4096, 1024, 64), value_stride=(4096, 1024, 64), kv_len=16, tree=None,
             tree_stride=0, B=2, T=1, Hq=4, Hkv=2, cap=16, d=64)
    a.update(kw)
    return ctypes.byref(_Tree(*[a[n] for n, _ in _Tree._fields_]))


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(out=None), -1), (dict(q_starts=None), -1), (dict(B=0), -1), (dict(Tq=0), -1), (dict(Tk=-1), -1),
    (dict(Hq=0), -1), (dict(Hkv=3), -1), (dict(causal=2), -1), (dict(clear_rest=-1), -1), (dict(q_stride=(0, 64)), -1), (dict(k_stride=(128, -64)), -1),
    (dict(d=96), -2), (dict(d=32), -2), (dict(Hq=258), -2), (dict(v_stride=(132, 64)), -2), (dict(q=24), -2), (dict(out=8), -2), (dict(q_starts=18), -2),
    (dict(k_starts=18), -2), (dict(B=(1 << 20) + 1), -2), (dict(k_stride=(1 << 38, 64)), -2)], ids=str)
def test_prompt_arguments(lib, kw, code):
    assert lib.topk_prompt_attn_fwd(_prompt(**kw), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), -1), (dict(keys=None), -1), (dict(values=None), -1), (dict(out=None), -1), (dict(kv_len=None), -1), (dict(B=0), -1), (dict(T=0), -1), (dict(cap=0), -1),
    (dict(Hq=3), -1), (dict(tree_stride=-1), -1), (dict(key_stride=(4096, 0, 64)), -1), (dict(q_stride=(-256, 64, 64)), -1), (dict(T=65), -2), (dict(d=80), -2),
    (dict(Hq=129, Hkv=1), -2), (dict(value_stride=(4096, 1024, 68)), -2), (dict(keys=8), -2), (dict(kv_len=18), -2), (dict(tree=20), -2)], ids=str)
def test_tree_arguments(lib, kw, code):
    assert lib.topk_tree_attn_fwd(_tree(**kw), None) == code


# of 8 rows of 4 heads of 64: q takes 4,096 bytes, k and v with two heads 2,048
@pytest.mark.parametrize("kw", [dict(out=1 << 16), dict(out=(1 << 16) + 4080), dict(out=(1 << 16) - 4080), dict(out=(2 << 16) + 2032), dict(out=(3 << 16) - 16)], ids=str)
def test_outputs_inside_the_inputs(lib, kw):
    assert lib.topk_prompt_attn_fwd(_prompt(**{**dict(q=1 << 16, k=2 << 16, v=3 << 16), **kw}), None) == -1
    tree = dict(B=1, T=8, cap=8, q_stride=(0, 64, 256), key_stride=(0, 64, 128), value_stride=(0, 64, 128))
    assert lib.topk_tree_attn_fwd(_tree(**{**tree, **dict(q=1 << 16, keys=2 << 16, values=3 << 16), **kw}), None) == -1


def test_outputs_beside_the_inputs(lib):
    # every argument is taken: what is missing here is a device (on one that has it, these addresses are never read)
    if torch.cuda.is_available():
        pytest.skip("made-up addresses")
    for out in ((1 << 16) + 4096, (1 << 16) - 4096, (2 << 16) + 2048):
        assert lib.topk_prompt_attn_fwd(_prompt(q=1 << 16, k=2 << 16, v=3 << 16, out=out), None) == -6


def test_null_records(lib):
    assert lib.topk_prompt_attn_fwd(None, None) == -1
    assert lib.topk_tree_attn_fwd(None, None) == -1
    assert T.topk_prompt_attn_workspace_bytes(96) == 0


def test_bindings_refuse_host_tensors(no_library):
    ids, w = torch.zeros(3, dtype=torch.int64), torch.zeros(5, 8)
    q, starts = torch.zeros(4, 2, 64, dtype=BF), torch.tensor([0, 4], dtype=torch.int32)
    for call in (lambda: T.embedding(ids, w), lambda: T.embedding_bwd(torch.zeros(3, 8), ids, 5), lambda: T.token_logprobs(w, ids.new_zeros(5)),
                 lambda: T.token_logprobs_bwd(w, w[:, 0].contiguous(), targets=ids.new_zeros(5), dlogp=torch.zeros(5)), lambda: T.prompt_attention(q, q, q, starts),
                 lambda: T.tree_attention(q[None], q[None], q[None], torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_bindings_refuse_shapes_and_types(anywhere):
    ids, w = torch.zeros(3, dtype=torch.int64), torch.zeros(5, 8)
    starts = torch.tensor([0, 4], dtype=torch.int32)
    q, kv = torch.zeros(4, 2, 64, dtype=BF), torch.zeros(4, 1, 64, dtype=BF)
    x, lse = torch.zeros(3, 8), torch.zeros(3)
    cache, one = torch.zeros(1, 1, 9, 64, dtype=BF), torch.zeros(1, 2, 3, 64, dtype=BF)
    n = torch.zeros(1, dtype=torch.int32)
    words = torch.zeros(1, 3, dtype=torch.int64)
    bad = [
        lambda: T.embedding(ids.float(), w), lambda: T.embedding(ids, w[:, ::2]), lambda: T.embedding(ids, w.t()), lambda: T.embedding(torch.arange(6)[::2], w),
        lambda: T.embedding(ids, w.double()), lambda: T.embedding(ids, w[0]),
        lambda: T.embedding_bwd(torch.zeros(4, 8), ids, 5), lambda: T.embedding_bwd(torch.zeros(3, 8).half(), ids, 5),
        lambda: T.embedding_bwd(torch.zeros(3, 8), ids, 5, into=w[:4]), lambda: T.embedding_bwd(torch.zeros(3, 8), ids, 5, grad_dtype=BF, into=w),
        lambda: T.token_logprobs(x[:, ::2]), lambda: T.token_logprobs(x[None]), lambda: T.token_logprobs(x.half()), lambda: T.token_logprobs(x, ids[:2]),
        lambda: T.token_logprobs(x, ids.float()), lambda: T.token_logprobs(x[:1].expand(3, 8)),
        lambda: T.token_logprobs_bwd(x, lse[:2], targets=ids, dlogp=lse), lambda: T.token_logprobs_bwd(x, lse, targets=ids, dlogp=lse.double()),
        lambda: T.token_logprobs_bwd(x, lse, targets=ids, dlogp=lse, out=x.to(BF)), lambda: T.token_logprobs_bwd(x, lse, top_ids=ids[:, None], dtop=x[:, :1]),
        lambda: T.prompt_attention(q.float(), kv, kv, starts), lambda: T.prompt_attention(q, kv, kv[:, :, :32], starts), lambda: T.prompt_attention(q, kv[:3], kv[:3], starts),
        lambda: T.prompt_attention(q, kv, kv, starts.long()), lambda: T.prompt_attention(q, kv, kv, starts[:1]), lambda: T.prompt_attention(q, kv, kv, starts, k_starts=starts[:1]),
        lambda: T.prompt_attention(q, kv, kv, starts, out=q[:3]), lambda: T.prompt_attention(q[None], kv, kv, starts), lambda: T.prompt_attention(q, kv[:0], kv[:0], starts),
        lambda: T.tree_attention(one, cache, cache[:, :, :8], n), lambda: T.tree_attention(one, cache.float(), cache, n), lambda: T.tree_attention(one, cache, cache, n.long()),
        lambda: T.tree_attention(one, cache, cache, n, tree=words[:, :2]), lambda: T.tree_attention(one, cache, cache, n, tree=words.int()),
        lambda: T.tree_attention(one[0], cache, cache, n), lambda: T.tree_mask(torch.zeros(2, 65, dtype=torch.int64)),
    ]
    for call in bad:
        with pytest.raises((ValueError, TypeError)):
            call()


def test_bindings_refuse_sizes_a_c_int_does_not_hold(anywhere):
    ids = _meta(3, dtype=torch.int64)
    f32 = torch.float32
    calls = [
        lambda: T.topk_embedding_fwd(ids, _meta(LONG, 8), _meta(3, 8)), lambda: T.topk_embedding_fwd(ids, _meta(8, LONG), _meta(3, LONG)),
        lambda: T.topk_embedding_fwd(_meta(LONG, dtype=torch.int64), _meta(8, 8), _meta(LONG, 8)), lambda: T.topk_embedding_bwd(_meta(3, 8), ids, _meta(LONG, 8)),
        lambda: T.topk_token_logprobs_fwd(_meta(LONG, 8), lse=_meta(LONG, dtype=f32)), lambda: T.topk_token_logprobs_fwd(_meta(8, LONG), lse=_meta(8, dtype=f32)),
        lambda: T.topk_prompt_attn_fwd(_meta(LONG, 1, 64), _meta(8, 1, 64), _meta(8, 1, 64), _meta(LONG, 1, 64), ids.int()),
        lambda: T.topk_tree_attn_fwd(_meta(1, 1, 1, 64), _meta(1, 1, LONG, 64), _meta(1, 1, LONG, 64), _meta(1, 1, 1, 64), ids.int()),
    ]
    for call in calls:
        with pytest.raises(ValueError, match="2\\^31"):
            call()


def test_tree_words():
    # 0 and 1 follow the cache, 2 and 3 token 0, 4 token 3
    parents = torch.tensor([[-1, -1, 0, 0, 3], [-1, 0, 1, 2, 3]])
    assert T.tree_mask(parents).tolist() == [[1, 2, 5, 9, 25], [1, 3, 7, 15, 31]]
    chain = T.tree_mask(torch.arange(-1, 63))
    assert chain.tolist() == [(1 << i + 1) - 1 for i in range(63)] + [-1]
    assert T.tree_mask(torch.full((64,), -1)).tolist() == [1 << i for i in range(63)] + [-(1 << 63)]
