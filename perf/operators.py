"""Measured cases of the operators around the attention: the norms of queries and keys with the position
rotation, the linear layer with bias, activation and residual, and the AdamW step over many tensors.

``run`` computes a case in its plain form (elementary torch operations in 32 bits), or, where ``own`` is
true, by the calls that a user makes of this package.
"""
import math

import torch

own = False

BF16, F32, F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
DTYPES = {"bf16": BF16, "f32": F32}
BLOCK = 256  # elements that share the scale of an 8-bit state
EPS = 1e-6  # of the norms
BETAS, ADAM_EPS, LR, DECAY, SEED, STEP0 = (0.9, 0.999), 1e-8, 1e-3, 0.01, 1234, 10
LAYERS = {  # decoder stacks by their widths: (layers, d_model, d_ff)
    "tiny": (2, 256, 512),
    "base": (12, 768, 2048),
    "large": (18, 1280, 4096),
}


def listed():
    return [
        # one new token for each of 4 sequences, written into their caches (12 heads of 64, as decode_65k)
        dict(name="qk_token", op="qk_fwd", B=4, L=1, Hq=12, Hkv=12, d=64, rot=64, axes=1, pairs="half", dtype="bf16", cap=8192),
        # the long sequence of the paper's benchmark: 65,536 tokens, 12 heads of 64
        dict(name="qk_long", op="qk_fwd", B=1, L=65536, Hq=12, Hkv=12, d=64, rot=64, axes=1, pairs="half", dtype="bf16", cap=0),
        # image and video tokens: three axes, shared key heads, an odd length
        dict(name="qk_video", op="qk_fwd", B=2, L=4099, Hq=32, Hkv=8, d=128, rot=128, axes=3, pairs="half", dtype="bf16", cap=0),
        # the gradients of the causal decoder layer with 16 heads of 128, as attention's backward pass hands them over (fp32)
        dict(name="qk_grad", op="qk_bwd", B=2, L=16384, Hq=16, Hkv=16, d=128, rot=128, axes=1, pairs="half", dtype="bf16", grad="f32"),
        # shared key heads, a partial rotation of neighbouring pairs, a short odd batch in fp32
        dict(name="qk_grad_odd", op="qk_bwd", B=3, L=333, Hq=10, Hkv=2, d=64, rot=32, axes=2, pairs="neighbours", dtype="f32", grad="f32"),
        # a few tokens being decoded through the up projection
        dict(name="lin_token", op="lin_fwd", M=4, K=1024, N=4096, act="gelu", bias=True, res=False, keep=False),
        # the attention's output projection with the residual, 32,768 tokens of the 12-layer decoder
        dict(name="lin_proj", op="lin_fwd", M=32768, K=768, N=768, act="none", bias=False, res=True, keep=False),
        # a training forward pass of a wide feed-forward layer, its pre-activations kept
        dict(name="lin_wide", op="lin_fwd", M=16384, K=2048, N=8192, act="silu", bias=True, res=False, keep=True),
        # the gradients of a feed-forward layer over an odd number of tokens
        dict(name="lin_grad", op="lin_bwd", M=8197, K=1024, N=4096, act="relu", bias=True),
        # a small model's many small tensors: latency
        dict(name="adamw_tiny", op="adamw", stack="tiny", bits=32, param="f32", grad="f32", master=False),
        # the 12-layer decoder in bf16 with 32-bit states and 32-bit masters
        dict(name="adamw_base", op="adamw", stack="base", bits=32, param="bf16", grad="bf16", master=True),
        # a larger model with states in 8 bits
        dict(name="adamw_8bit", op="adamw", stack="large", bits=8, param="bf16", grad="bf16", master=False),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    top = {"qk_fwd": 6.2e8, "qk_bwd": 1.4e9, "lin_fwd": 5e11, "lin_bwd": 5e11, "adamw": 3e9}
    op = rng.choice(["qk_fwd", "qk_fwd", "qk_bwd", "lin_fwd", "lin_fwd", "lin_bwd", "adamw"])
    while True:
        if op in ("qk_fwd", "qk_bwd"):
            d = rng.choice([64, 128])
            hkv = rng.choice([2, 4, 8, 12, 16])
            hq = hkv * rng.choice([1, 1, 2, 4])
            c = dict(op=op, B=rng.choice([1, 2, 3, 4, 8]), L=_log(rng, 1, 65536), Hq=hq, Hkv=hkv, d=d, rot=rng.choice([d, d, d // 2]),
                     axes=rng.choice([1, 1, 2, 3]), pairs=rng.choice(["half", "neighbours"]), dtype=rng.choice(["bf16", "bf16", "f32"]))
            if op == "qk_fwd":
                c["cap"] = 4096 if c["L"] <= 512 and rng.random() < 0.7 else 0
            else:
                c["grad"] = "f32" if c["dtype"] == "f32" else rng.choice(["bf16", "f32"])
            cost = work(c)["bytes"]
        elif op in ("lin_fwd", "lin_bwd"):
            c = dict(op=op, M=_log(rng, 1, 32768), K=_log(rng, 256, 8192, 8), N=_log(rng, 256, 8192, 8), act=rng.choice(["none", "relu", "gelu", "silu"]),
                     bias=rng.random() < 0.5)
            if op == "lin_fwd":
                c.update(res=rng.random() < 0.4, keep=c["act"] != "none" and rng.random() < 0.5)
            cost = work(c)["flops"]
        else:
            param = rng.choice(["f32", "bf16"])
            c = dict(op=op, layers=rng.randint(1, 16), d_model=_log(rng, 64, 1024, 8), d_ff=_log(rng, 128, 4096, 8), bits=rng.choice([8, 32]), param=param,
                        grad=rng.choice(["f32", param]), master=param == "bf16" and rng.random() < 0.5)
            cost = work(c)["bytes"]
        if cost <= top[op] and 3072 not in (c.get("M"), c.get("K"), c.get("N"), c.get("d_ff"), 3 * c.get("d_model", 0)):
            return c


# ------------------------------------------------------------------ inputs


def _sections(c):
    """The pairs of each axis: time first, the others share what is left."""
    half, a = c["rot"] // 2, c["axes"]
    rest = half // a
    return [half - rest * (a - 1)] + [rest] * (a - 1)


def _shapes(c):
    n, dm, dff = LAYERS[c["stack"]] if "stack" in c else (c["layers"], c["d_model"], c["d_ff"])
    layer = [(dm,)] * 4 + [(3 * dm, dm), (dm, dm), (dff, dm), (dff, dm)]
    return layer * n + [(dm,)] * 2


def _spans(c):
    """(elements, start) of each tensor in the flat states: every tensor starts a block of its own."""
    at, spans = 0, []
    for shape in _shapes(c):
        n = math.prod(shape)
        spans.append((n, at))
        at += -(-n // BLOCK) * BLOCK
    return spans, at


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s, dtype=F32: torch.randn(*s, generator=g, device="cuda", dtype=F32).to(dtype)  # noqa: E731
    if c["op"] in ("qk_fwd", "qk_bwd"):
        dt, B, L, Hq, Hkv, d = DTYPES[c["dtype"]], c["B"], c["L"], c["Hq"], c["Hkv"], c["d"]
        qkv = rand(B, L, Hq + 2 * Hkv, d, dtype=dt)  # the projection's output
        s = dict(c, q=qkv[:, :, :Hq], k=qkv[:, :, Hq:Hq + Hkv], v=qkv[:, :, Hq + Hkv:], sections=_sections(c),
                 qw=1 + 0.1 * rand(d), kw=1 + 0.1 * rand(d), scale=d ** -0.5)
        s["qw"], s["kw"] = s["qw"].to(dt), s["kw"].to(dt)
        rows = max(c.get("cap", 0), L)
        angle = torch.arange(rows, dtype=torch.float64, device="cuda")[:, None] * 10000.0 ** (
            -torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda") * 2 / c["rot"])
        s["cos"], s["sin"] = angle.cos().float(), angle.sin().float()
        s["start"] = None
        if c.get("cap"):
            s["start"] = torch.randint(0, c["cap"] - L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["kc"], s["vc"] = (rand(B, Hkv, c["cap"], d, dtype=dt) for _ in range(2))
        t = torch.arange(L, device="cuda", dtype=torch.int32)
        first = t.expand(B, L) if s["start"] is None else t + s["start"][:, None]
        side = max(1, math.isqrt(L))  # an image's rows and columns
        s["pos"] = torch.stack(([first] + [(t // side).expand(B, L), (t % side).expand(B, L)])[: c["axes"]]).contiguous()
        if c["op"] == "qk_bwd":
            gt = DTYPES[c["grad"]]
            s["dq"], s["dk"], s["dv"] = (rand(B, h, L, d, dtype=gt) for h in (Hq, Hkv, Hkv))
        return s
    if c["op"] in ("lin_fwd", "lin_bwd"):
        M, K, N = c["M"], c["K"], c["N"]
        s = dict(c, x=rand(M, K, dtype=BF16), w=(rand(N, K) * K ** -0.5).to(BF16))
        s["b"] = (0.1 * rand(N)).to(BF16) if c["bias"] else None
        if c["op"] == "lin_fwd":
            s["r"] = rand(M, N, dtype=BF16) if c["res"] else None
        else:
            s["z"] = None if c["act"] == "none" else rand(M, N, dtype=BF16)
            s["dy"] = rand(M, N, dtype=BF16)
        return s
    spans, total = _spans(c)
    pt, gt = DTYPES[c["param"]], DTYPES[c["grad"]]
    s = dict(c, spans=spans, total=total, steps=STEP0, opt=None)
    full = 0.02 * rand(total)
    s["p"], s["g"] = full.to(pt), (1e-3 * rand(total)).to(gt)
    s["master"] = full if c["master"] else None
    m, r = 1e-3 * rand(total), (1e-3 * rand(total)).abs() + 1e-5
    pad = torch.ones(total, dtype=torch.bool, device="cuda")
    for n, at in spans:
        pad[at:at + n] = False
    m, r = m.masked_fill(pad, 0), r.masked_fill(pad, 0)
    if c["bits"] == 32:
        s["m"], s["v"] = m, r * r
    else:
        for name, x in (("m", m), ("v", r)):
            scale = x.view(-1, BLOCK).abs().amax(1) * (1 / 448)
            s[name], s[name + "s"] = (x.view(-1, BLOCK) / scale[:, None]).to(F8).view(-1), scale
    s["ps"], s["gs"] = ([s[k][at:at + n].view(shape) for (n, at), shape in zip(spans, _shapes(c))] for k in ("p", "g"))
    s["masters"] = [s["master"][at:at + n] for n, at in spans] if c["master"] else None
    return s


# ------------------------------------------------------------------ one pass


def run(s):
    return {"qk_fwd": _qk_fwd, "qk_bwd": _qk_bwd, "lin_fwd": _lin_fwd, "lin_bwd": _lin_bwd, "adamw": _adamw}[s["op"]](s)


def _rope_args(s):
    return dict(positions=s["pos"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS, q_scale=s["scale"], sections=s["sections"], interleaved=s["pairs"] != "half")


def _angles(s):
    """cos and sin of each token and pair, [B, L, 1, rot/2]."""
    axis = torch.repeat_interleave(torch.arange(len(s["sections"]), device="cuda"), torch.tensor(s["sections"], device="cuda"), output_size=s["rot"] // 2)
    p = s["pos"].long()[axis].permute(1, 2, 0)
    i = torch.arange(s["rot"] // 2, device="cuda")
    return s["cos"][p, i][:, :, None], s["sin"][p, i][:, :, None]


def _split(x, s):
    x, rest = x[..., : s["rot"]], x[..., s["rot"]:]
    return (*(x.chunk(2, -1) if s["pairs"] == "half" else (x[..., 0::2], x[..., 1::2])), rest)


def _join(a, b, rest, s):
    x = torch.cat((a, b), -1) if s["pairs"] == "half" else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((x, rest), -1)


def _qk_fwd(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        cache = (s["kc"], s["vc"]) if s["cap"] else None
        return T.qk_norm_rope(s["q"], s["k"], s["v"], s["cos"], s["sin"], cache=cache, cache_start=s["start"], **_rope_args(s))
    cos, sin = _angles(s)

    def one(x, w, scale):
        x = x.float()
        n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
        a, b, rest = _split(n, s)
        return (_join(a * cos - b * sin, b * cos + a * sin, rest, s) * scale).to(s["q"].dtype)

    q, k, v = one(s["q"], s["qw"], s["scale"]), one(s["k"], s["kw"], 1.0), s["v"]
    q = q.transpose(1, 2).contiguous()
    if not s["cap"]:
        return q, k.transpose(1, 2).contiguous(), v.transpose(1, 2).contiguous()
    rows = s["start"][:, None].long() + torch.arange(s["L"], device="cuda")
    at = torch.arange(s["B"], device="cuda")[:, None]
    s["kc"][at, :, rows], s["vc"][at, :, rows] = k, v
    return q, s["kc"], s["vc"]


def _qk_bwd(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.qk_norm_rope_bwd(s["dq"], s["dk"], s["dv"], s["q"], s["k"], s["cos"], s["sin"], **_rope_args(s))
    cos, sin = _angles(s)

    def one(dy, x, w, scale):
        dy, x, w = dy.float().transpose(1, 2) * scale, x.float(), w.float()
        a, b, rest = _split(dy, s)
        g = _join(a * cos + b * sin, b * cos - a * sin, rest, s)
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        u = g * w
        dx = u * r - x * (r * r * r) * (u * x).mean(-1, keepdim=True)
        return dx.to(s["q"].dtype), (g * x * r).sum((0, 1, 2))

    dq, dqw = one(s["dq"], s["q"], s["qw"], s["scale"])
    dk, dkw = one(s["dk"], s["k"], s["kw"], 1.0)
    return torch.cat((dq, dk, s["dv"].transpose(1, 2).to(s["q"].dtype)), 2), dqw, dkw


def _act(z, act):
    if act == "relu":
        return z.clamp_min(0)
    if act == "gelu":
        return z * 0.5 * (1 + torch.erf(z * 0.5 ** 0.5))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _lin_fwd(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.linear(s["x"], s["w"], bias=s["b"], act=s["act"], residual=s["r"], return_preact=s["keep"])
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z, s["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return (y.to(BF16), z.to(BF16)) if s["keep"] else y.to(BF16)


def _lin_bwd(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.linear_bwd(s["dy"], s["x"], s["w"], preact=s["z"], act=s["act"], bias=s["bias"])
    dz = s["dy"].float()
    if s["act"] == "relu":
        dz = dz * (s["z"] > 0)
    elif s["act"] == "gelu":
        z = s["z"].float()
        dz = dz * (0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5)
    elif s["act"] == "silu":
        z = s["z"].float()
        sig = 1 / (1 + torch.exp(-z))
        dz = dz * (sig * (1 + z * (1 - sig)))
    dx, dw = dz @ s["w"].float(), dz.t() @ s["x"].float()
    return dx.to(BF16), dw.to(BF16), (dz.sum(0).to(BF16) if s["bias"] else None)


# The random bits of an element at a step: a hash of both, so that a step can be repeated.
_MASK = 0xFFFFFFFF


def _mix(x):
    """The hash of whole numbers below 2^32 (int64 tensors, or one number)."""
    x = (x ^ (x >> 16)) & _MASK
    x = (x * 0x7FEB352D) & _MASK
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & _MASK
    return x ^ (x >> 16)


def _bits_of(index, step):
    return _mix((index * 0x9E3779B1 + _mix((SEED + step * 0x9E3779B9) & _MASK)) & _MASK)


def _to8(x, rnd):
    """8-bit floats and a scale for each block; `rnd`: 10 random bits for each value."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1) * (1 / 448)
    scale = torch.where(scale < 2.0 ** -100, 0.0, scale)
    inv = torch.where(scale == 0, 0.0, 1 / scale)
    y = x.abs() * inv[:, None]
    code = ((y * 2.0 ** -120).view(torch.int32) + (rnd.view(-1, BLOCK).to(torch.int32) << 10) + 512) >> 20
    code = code.clamp_max(0x7E) | torch.where(x < 0, 0x80, 0).to(torch.int32)
    return code.to(torch.uint8).view(F8).view(-1), scale


def _adamw(s):
    s["steps"] += 1
    if own:
        if s["opt"] is None:
            from paper_2106_06899_gb300 import optim

            state = {"exp_avg": s["m"], "exp_avg_sq": s["v"]} if s["bits"] == 32 else {"exp_avg": s["m"], "exp_avg_scale": s["ms"], "exp_avg_root": s["v"], "exp_avg_root_scale": s["vs"]}
            s["opt"] = optim.AdamW(s["ps"], lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, state_bits=s["bits"], seed=SEED, masters=s["masters"],
                                   state={**state, "step": s["steps"] - 1})
        s["opt"].step(s["gs"])
    else:
        t, (b1, b2) = s["steps"], BETAS
        isb2, size = 1 / math.sqrt(1 - b2 ** t), LR / (1 - b1 ** t)
        for k, (n, at) in enumerate(s["spans"]):  # one tensor after the other
            here, padded = slice(at, at + n), slice(at, at + -(-n // BLOCK) * BLOCK)
            g = s["gs"][k].view(-1).float()
            if s["bits"] == 32:
                m, v = s["m"][here], s["v"][here]
            else:
                m, v = ((s[name][padded].float().view(-1, BLOCK) * s[name + "s"][at // BLOCK:padded.stop // BLOCK, None]).view(-1)[:n] for name in ("m", "v"))
                v = v * v
            m = m * b1 + g * (1 - b1)
            v = v * b2 + (g * g) * (1 - b2)
            root = v.sqrt()
            p = (s["p"] if s["master"] is None else s["master"])[here].float()
            p = p * (1 - LR * DECAY) - (m / (root * isb2 + ADAM_EPS)) * size
            rnd = None
            if s["bits"] == 8 or (s["master"] is None and s["param"] == "bf16"):
                rnd = _bits_of(torch.arange(padded.start, padded.stop, device="cuda"), t)
            if s["master"] is not None:
                s["master"][here] = p
                s["p"][here] = p.to(s["p"].dtype)
            elif s["param"] == "bf16":
                s["p"][here] = ((p.view(torch.int32) + (rnd[:n] >> 20 << 4).to(torch.int32) + 8) & -65536).view(F32).to(BF16)
            else:
                s["p"][here] = p
            if s["bits"] == 32:
                s["m"][here], s["v"][here] = m, v
            else:
                tail = padded.stop - at - n
                for name, x, bits in (("m", m, rnd & 1023), ("v", root, rnd >> 10 & 1023)):
                    code, scale = _to8(torch.nn.functional.pad(x, (0, tail)), bits)
                    s[name].view(torch.uint8)[padded] = code.view(torch.uint8)
                    s[name + "s"][at // BLOCK:padded.stop // BLOCK] = scale
    out = [s["p"], s["m"], s["v"]] + ([s["ms"], s["vs"]] if s["bits"] == 8 else [])
    return out if s["master"] is None else out + [s["master"]]


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    c = case
    if c["op"] in ("qk_fwd", "qk_bwd"):
        e, rows = (2 if c["dtype"] == "bf16" else 4), c["B"] * c["L"]
        heads = c["Hq"] + 2 * c["Hkv"]
        tables = min(rows * c["axes"], max(c.get("cap", 0), c["L"])) * c["rot"] // 2 * 8 + rows * c["axes"] * 4
        if c["op"] == "qk_fwd":
            return {"bytes": 2 * rows * heads * c["d"] * e + tables, "flops": 10 * rows * heads * c["d"]}
        ge = 2 if c["grad"] == "bf16" else 4
        return {"bytes": rows * c["d"] * (heads * (e + ge) + (c["Hq"] + c["Hkv"]) * e) + tables, "flops": 20 * rows * heads * c["d"]}
    if c["op"] in ("lin_fwd", "lin_bwd"):
        M, K, N = c["M"], c["K"], c["N"]
        if c["op"] == "lin_fwd":
            return {"bytes": 2 * (M * K + N * K + M * N * (1 + c["res"] + c["keep"]) + N * c["bias"]), "flops": 2 * M * N * K}
        return {"bytes": 2 * (2 * M * K + 2 * N * K + M * N * (1 + (c["act"] != "none")) + N * c["bias"]), "flops": 4 * M * N * K}
    n = sum(math.prod(x) for x in _shapes(c))
    p, g = (2 if c["param"] == "bf16" else 4), (2 if c["grad"] == "bf16" else 4)
    per = (g + p + 8) if c["master"] else (g + 2 * p)
    return {"bytes": int(n * (per + (16 if c["bits"] == 32 else 4 + 16 / BLOCK))), "flops": 16 * n}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s, F64 = prepare(case, seed), torch.float64
    if s["op"] in ("qk_fwd", "qk_bwd"):
        # the rotation as a matrix of 2 x 2 blocks would turn it: complex numbers, one for each pair
        where = [a for a, n in enumerate(s["sections"]) for _ in range(n)]
        table = torch.complex(s["cos"].to(F64), s["sin"].to(F64))
        turn = torch.stack([table[s["pos"][a].long(), i] for i, a in enumerate(where)], -1)[:, :, None]
        half = s["rot"] // 2
        first = torch.arange(half, device="cuda") * (1 if s["pairs"] == "half" else 2)
        second = first + (half if s["pairs"] == "half" else 1)

        def rotate(x, by):
            y, z = x.clone(), torch.complex(x[..., first], x[..., second]) * by
            y[..., first], y[..., second] = z.real, z.imag
            return y

        def norm(x):
            return (x.pow(2).sum(-1, keepdim=True) / s["d"] + EPS).pow(-0.5)

        if s["op"] == "qk_fwd":
            q, k = (rotate(x.to(F64) * norm(x.to(F64)) * w.to(F64), turn) for x, w in ((s["q"], s["qw"]), (s["k"], s["kw"])))
            q, k, v = (q * s["scale"]).permute(0, 2, 1, 3), k.permute(0, 2, 1, 3), s["v"].permute(0, 2, 1, 3)
            if not s["cap"]:
                return q, k, v
            for b, t in enumerate(s["start"].tolist()):
                s["vc"][b, :, t:t + s["L"]] = v[b]
            kc = s["kc"].to(F64)
            for b, t in enumerate(s["start"].tolist()):
                kc[b, :, t:t + s["L"]] = k[b]
            return q, kc, s["vc"]
        packed, weights = [], []
        for dy, x, w, scale in ((s["dq"], s["q"], s["qw"], s["scale"]), (s["dk"], s["k"], s["kw"], 1.0)):
            g = rotate(dy.permute(0, 2, 1, 3).to(F64), turn.conj()) * scale
            x, r = x.to(F64), norm(x.to(F64))
            hat = x * r
            u = g * w.to(F64)
            packed.append(r * (u - hat * (u * hat).sum(-1, keepdim=True) / s["d"]))
            weights.append(torch.einsum("blhd,blhd->d", g, hat))
        return torch.cat(packed + [s["dv"].permute(0, 2, 1, 3).to(F64)], 2), *weights
    if s["op"] in ("lin_fwd", "lin_bwd"):
        x, w = s["x"].to(F64), s["w"].to(F64)
        normal = torch.distributions.Normal(torch.tensor(0.0, dtype=F64, device="cuda"), 1.0)
        if s["op"] == "lin_fwd":
            z = torch.einsum("mk,nk->mn", x, w) + (0 if s["b"] is None else s["b"].to(F64))
            y = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0), "gelu": lambda: z * normal.cdf(z), "silu": lambda: z * torch.sigmoid(z)}[s["act"]]()
            y = y if s["r"] is None else y + s["r"].to(F64)
            return (y, z) if s["keep"] else y
        dy, z = s["dy"].to(F64), None if s["z"] is None else s["z"].to(F64)
        slope = {"none": lambda: 1.0, "relu": lambda: torch.sign(z).clamp(0, 1), "gelu": lambda: normal.cdf(z) + z * normal.log_prob(z).exp(),
                 "silu": lambda: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)}[s["act"]]()
        dz = dy * slope
        return torch.einsum("mn,nk->mk", dz, w), torch.einsum("mn,mk->nk", dz, x), (torch.einsum("mn->n", dz) if s["bias"] else None)
    # AdamW over the flat buffers; the tensors' padding is left as it is
    t, (b1, b2) = s["steps"] + 1, BETAS
    real = torch.zeros(s["total"], dtype=torch.bool, device="cuda")
    for n, at in s["spans"]:
        real[at:at + n] = True
    g = torch.where(real, s["g"].to(F64), 0)
    if s["bits"] == 32:
        m, v = s["m"].to(F64), s["v"].to(F64)
    else:
        m, v = (s[k].to(F64) * s[k + "s"].to(F64).repeat_interleave(BLOCK) for k in ("m", "v"))
        v = v.pow(2)
    m, v = torch.lerp(g, m, b1), torch.lerp(g.pow(2), v, b2)
    old = (s["p"] if s["master"] is None else s["master"]).to(F64)
    step = LR * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + ADAM_EPS)
    p = torch.where(real, old - LR * DECAY * old - step, old)
    rnd = _bits_of(torch.arange(s["total"], device="cuda"), t).to(F64)
    stored = p
    if s["master"] is None and s["param"] == "bf16":  # stochastic: down to a multiple of the last place after adding a part of it
        ulp = torch.exp2(torch.floor(torch.log2(p.abs().clamp_min(1e-300))) - 7)
        part = (torch.floor(rnd / 2 ** 20) * 16 + 8) / 65536
        stored = torch.where(real, torch.sign(p) * ulp * torch.floor(p.abs() / ulp + part), old)
    out = [stored]
    if s["bits"] == 32:
        out += [torch.where(real, m, s["m"].to(F64)), torch.where(real, v, s["v"].to(F64))]
    else:
        scales = []
        for x, shift in ((m, 0), (v.sqrt(), 10)):
            scale = x.view(-1, BLOCK).abs().amax(1) / 448
            y = (x.view(-1, BLOCK).abs() / scale[:, None].clamp_min(1e-300)).view(-1)
            place = torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** -6))) - 3)  # of an 8-bit float with 3 bits after the point
            part = (torch.floor(rnd / 2 ** shift).remainder(1024) * 1024 + 512) / 2 ** 20
            out.append(torch.sign(x) * (place * torch.floor(y / place + part)).clamp_max(448))
            scales.append(scale)
        out += scales
    return out if s["master"] is None else out + [p]
