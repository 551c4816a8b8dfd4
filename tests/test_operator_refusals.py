"""The operators around the attention refuse bad arguments before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2106_06899_gb300 import build
from paper_2106_06899_gb300 import topk as T


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return T.lib()


class _QkArgs(ctypes.Structure):
    """topk_qk_args"""
    _fields_ = ([(n, ctypes.c_void_p) for n in ("q", "k", "v")]
                + [(n, ctypes.c_longlong * 3) for n in ("q_stride", "k_stride", "v_stride")]
                + [(n, ctypes.c_void_p) for n in ("q_weight", "k_weight", "cos", "sin", "positions")]
                + [(n, ctypes.c_int) for n in ("table_rows", "B", "L", "Hq", "Hkv", "d", "rot", "axes")]
                + [("sections", ctypes.c_int * 4)]
                + [(n, ctypes.c_int) for n in ("interleaved", "normalize", "dtype")]
                + [(n, ctypes.c_float) for n in ("eps", "q_scale")])


def test_qk_record_matches_the_header():
    # the binding packs topk_qk_args as bytes; the same values through the header's layout
    values = [1, 2, 3, *range(10, 19), 4, 5, 6, 7, 8, *range(20, 28), *range(30, 34), 1, 0, 1, 0.5, 0.25]
    fields, at = [], 0
    for name, kind in _QkArgs._fields_:
        n = getattr(kind, "_length_", 0)
        fields.append(tuple(values[at:at + n]) if n else values[at])
        at += n or 1
    assert bytes(_QkArgs(*fields)) == T._QK_PACK(*values)


def _qk(**kw):
    a = dict(q=16, k=16, v=16, q_stride=(64, 64, 64), k_stride=(64, 64, 64), v_stride=(64, 64, 64), q_weight=None, k_weight=None,
             cos=16, sin=16, positions=None, table_rows=8, B=1, L=8, Hq=2, Hkv=1, d=64, rot=64, axes=1, sections=(32, 0, 0, 0),
             interleaved=0, normalize=1, dtype=1, eps=1e-6, q_scale=1.0)
    a.update(kw)
    return _QkArgs(*[a[n] for n, _ in _QkArgs._fields_])


BAD = [
    (dict(q=None), -1), (dict(k=None), -1), (dict(cos=None), -1), (dict(B=0), -1), (dict(L=-1), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1),
    (dict(rot=72), -1), (dict(axes=0), -1), (dict(axes=5), -1), (dict(sections=(31, 0, 0, 0)), -1), (dict(axes=2, sections=(33, -1, 0, 0)), -1),
    (dict(dtype=2), -1), (dict(normalize=0, q_weight=16), -1), (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1),
    (dict(table_rows=7), -1), (dict(q_stride=(-64, 64, 64)), -1), (dict(q_stride=(64, 66, 64)), -2),
    (dict(d=60, rot=56, sections=(28, 0, 0, 0)), -2), (dict(d=264), -2), (dict(rot=60, sections=(30, 0, 0, 0)), -2), (dict(q=24), -2), (dict(q_weight=8), -2), (dict(positions=18), -2),
]


@pytest.mark.parametrize("kw,code", BAD, ids=str)
def test_qk_arguments(lib, kw, code):
    a = _qk(**kw)
    assert lib.topk_qk_norm_rope_fwd(ctypes.byref(a), 16, 16, 16, 8, None, None) == code
    assert lib.topk_qk_norm_rope_bwd(ctypes.byref(a), 16, 16, 16, 0, 16, 16, 16, None) == code


def test_qk_outputs(lib):
    f, a = lib.topk_qk_norm_rope_fwd, _qk()
    ref = ctypes.byref(a)
    assert f(None, 16, 16, 16, 8, None, None) == -1
    assert f(ref, None, 16, 16, 8, None, None) == -1
    assert f(ref, 16, 16, None, 8, None, None) == -1   # v without v_out
    assert f(ref, 16, 16, 16, 9, None, None) == -1     # a cache without its start rows
    assert f(ref, 16, 16, 16, 0, 16, None) == -1
    assert f(ref, 24, 16, 16, 8, None, None) == -2
    assert f(ref, 16, 16, 16, 9, 18, None) == -2
    b = lib.topk_qk_norm_rope_bwd
    assert b(ref, None, 16, 16, 0, 16, 16, 16, None) == -1
    assert b(ref, 16, 16, 16, 3, 16, 16, 16, None) == -1
    assert b(ctypes.byref(_qk(dtype=0)), 16, 16, 16, 1, 16, 16, 16, None) == -2
    assert b(ref, 16, 16, 24, 0, 16, 16, 16, None) == -2
    assert T.topk_qk_norm_rope_bwd_workspace_bytes(1, 100, 2, 1, 64) == 13 * 3 * 64 * 4
    assert T.topk_qk_norm_rope_bwd_workspace_bytes(1, 1 << 20, 32, 8, 64) <= (8 * 160 + 40) * 64 * 4
    assert T.topk_qk_norm_rope_bwd_workspace_bytes(1, 100, 2, 1, 60) == 0


def test_qk_binding_shapes():
    q = torch.zeros(1, 8, 2, 64, dtype=torch.bfloat16)
    cos, sin = T.rope_tables(8, 64, device="cpu")
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q[:, :7], None, cos, sin)
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q[..., ::2], cos, sin)
    with pytest.raises(TypeError):
        T.qk_norm_rope(q, q.float(), None, cos, sin)
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q, cos.double(), sin)
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q, cos, sin, q_weight=torch.ones(64))
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q, cos, sin, positions=torch.zeros(2, 1, 8, dtype=torch.int32))
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q, cos, sin, sections=(8, 8, 8, 4, 4))
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q, cos, sin, cache_start=torch.zeros(1, dtype=torch.int32))
    with pytest.raises(ValueError):
        T.qk_norm_rope(q, q, q, cos, sin, cache=(q, q))


class _Tensor(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")]
                + [("n", ctypes.c_longlong), ("index", ctypes.c_longlong), ("lr", ctypes.c_double), ("weight_decay", ctypes.c_double)])


def _adamw(lib, count=1, pdt=0, gdt=0, bits=32, b1=0.9, b2=0.999, eps=1e-8, step=1, gs=None, **kw):
    a = dict(param=16, grad=16, master=None, m=16, v=16, m_scale=16, v_scale=16, n=8, index=0, lr=1e-3, weight_decay=0.0)
    a.update(kw)
    t = _Tensor(*[a[n] for n, _ in _Tensor._fields_])
    return lib.topk_adamw_step(ctypes.addressof(t), count, pdt, gdt, bits, b1, b2, eps, step, gs, 0, None)


@pytest.mark.parametrize("kw,code", [
    (dict(count=-1), -1), (dict(step=0), -1), (dict(pdt=2), -1), (dict(gdt=5), -1), (dict(bits=16), -1), (dict(b1=1.0), -1), (dict(b2=-0.1), -1),
    (dict(eps=-1.0), -1), (dict(eps=float("nan")), -1), (dict(n=-1), -1), (dict(lr=float("inf")), -1), (dict(weight_decay=float("nan")), -1),
    (dict(param=None), -1), (dict(grad=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(bits=8, m_scale=None), -1),
    (dict(master=16), -1), (dict(param=18), -2), (dict(pdt=1, param=17), -2), (dict(grad=18), -2), (dict(m=18), -2), (dict(gs=18), -2),
    (dict(bits=8, v_scale=18), -2),
], ids=str)
def test_adamw_arguments(lib, kw, code):
    assert _adamw(lib, **kw) == code


def test_adamw_record_matches_the_header(lib):
    from paper_2106_06899_gb300 import optim

    assert optim._TENSOR.itemsize == ctypes.sizeof(_Tensor)
    assert [(n, optim._TENSOR.fields[n][1]) for n in optim._TENSOR.names] == [(n, getattr(_Tensor, n).offset) for n, _ in _Tensor._fields_]


def test_adamw_binding():
    from paper_2106_06899_gb300 import optim

    p = torch.zeros(8, 4)
    for bad in (dict(params=[]), dict(params=[p], state_bits=4), dict(params=[p, p.bfloat16()]), dict(params=[p.t()]),
                dict(params=[p], masters=True), dict(params=[p.bfloat16()], masters=[p.bfloat16()]), dict(params=[p], state={"exp_avg": p})):
        with pytest.raises(ValueError):
            optim.AdamW(**bad)
    opt = optim.AdamW([p])
    with pytest.raises(ValueError):
        opt.step([])
    with pytest.raises(ValueError):
        opt.step([torch.zeros(31)])
    with pytest.raises(TypeError):
        opt.step([torch.zeros(8, 4, dtype=torch.float16)])
    with pytest.raises(ValueError):
        opt.step([p], grad_scale=torch.zeros(2))
    with pytest.raises(ValueError):
        opt.load_state_dict(optim.AdamW([p], state_bits=8).state_dict())
    assert optim.AdamW([p], state_bits=8).moments(0)[0].shape == p.shape


def test_linear_arguments(lib):
    f, b = lib.topk_linear_fwd, lib.topk_linear_bwd

    def fwd(x=16, w=16, bias=None, res=None, y=16, z=None, M=4, N=16, K=16, act=0):
        return f(x, w, bias, res, y, z, M, N, K, act, None)

    def bwd(dy=16, x=16, w=16, z=None, dx=16, dw=16, db=16, M=4, N=16, K=16, act=0, dt=1):
        return b(dy, x, w, z, dx, dw, db, M, N, K, act, dt, None)

    for kw, code in ((dict(x=None), -1), (dict(w=None), -1), (dict(M=0), -1), (dict(N=-8), -1), (dict(K=0), -1), (dict(act=4), -1), (dict(act=-1), -1),
                     (dict(N=20), -2), (dict(K=12), -2), (dict(x=24), -2), (dict(M=1 << 29), -2)):
        assert fwd(**kw) == code, kw
        assert bwd(**kw) == code, kw
    for kw, code in ((dict(y=None), -1), (dict(bias=24), -2), (dict(res=8), -2), (dict(z=8), -2)):
        assert fwd(**kw) == code, kw
    for kw, code in ((dict(dy=None), -1), (dict(dx=None, dw=None, db=None), -1), (dict(z=16), -1), (dict(act=1), -1), (dict(dt=2), -1), (dict(db=8), -2)):
        assert bwd(**kw) == code, kw


def test_linear_scratch():
    # one wave of tiles or more, or few rows: none; a split sum: parts x outputs in fp32
    assert T.topk_linear_workspace_bytes(32768, 768, 768) == 0
    assert T.topk_linear_workspace_bytes(4, 4096, 1024) == 0
    ws = T.topk_linear_workspace_bytes(64, 512, 4096)
    assert ws > 0 and ws % (64 * 512 * 4) == 0 and ws <= 160 * 64 * 512 * 4
    assert T.topk_linear_workspace_bytes(64, 510, 4096) == 0
    assert T.topk_linear_bwd_workspace_bytes(8192, 4096, 1024, "relu") >= 8192 * 4096 * 2
    assert T.topk_linear_bwd_workspace_bytes(8192, 4096, 1024, "relu") <= 2 * 8192 * 4096 * 2


def test_linear_binding():
    x, w = torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(8, 16, dtype=torch.bfloat16)
    for bad in (dict(act="tanh"), dict(bias=torch.zeros(8)), dict(residual=torch.zeros(4, 7, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            T.linear(x, w, **bad)
    with pytest.raises(ValueError):
        T.linear(x.float(), w)
    with pytest.raises(ValueError):
        T.linear_bwd(x, x, w)
