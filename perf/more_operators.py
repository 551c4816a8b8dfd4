"""Measured cases of the operators at a language model's two ends and of its serving attention: the embedding lookup
with its gradient, log probabilities of tokens with their gradient, attention over packed prompts, and attention of
drafted tokens (a tree of them, or a single one) over key/value caches.

``run`` computes a case in its plain form (elementary torch operations in 32 bits), or, where ``own`` is
true, by the calls that a user makes of this package.
"""
import math

import numpy as np
import torch

own = False

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
DTYPES = {"bf16": BF16, "f32": F32}


def listed():
    return [
        # the next tokens of 8 sequences on their way into the decoder
        dict(name="embed_token", op="embed", N=8, V=32768, D=768, dtype="bf16", scale=True, pad=False),
        # a long batch into a wide model, a large vocabulary, padded ends
        dict(name="embed_batch", op="embed", N=65536, V=131072, D=1280, dtype="bf16", scale=True, pad=True),
        # the gradient of the 12-layer decoder's embedding, 32,768 tokens, most of them of a few common words
        dict(name="embed_grad", op="embed_bwd", N=32768, V=32768, D=768, dtype="bf16", grad="bf16", into=False, pad=False),
        # tied weights: added to the 32-bit gradient that the output projection left; odd sizes
        dict(name="embed_grad_tied", op="embed_bwd", N=8191, V=50001, D=1000, dtype="bf16", grad="f32", into=True, pad=True),
        # a decoding step's 4 rows of logits, with 20 alternatives for each
        dict(name="logprob_token", op="logprob", N=4, V=131072, top=20, dtype="bf16", target=True, masked=0, hot=0.8),
        # scoring given texts: an odd vocabulary, its last entries masked, 8 alternatives
        dict(name="logprob_score", op="logprob", N=4099, V=50001, top=8, dtype="bf16", target=True, masked=47, hot=1.0),
        # the gradient of a training loss with an entropy term
        dict(name="logprob_grad", op="logprob_bwd", N=8192, V=32768, top=0, dtype="bf16", entropy=True, masked=0, hot=1.0),
        # a few short prompts: latency
        dict(name="prompt_short", op="prompt", B=4, longest=61, Hq=12, Hkv=12, d=64, past=0, causal=True),
        # a serving batch: prompts of many lengths, shared key heads
        dict(name="prompt_batch", op="prompt", B=12, longest=4093, Hq=32, Hkv=8, d=128, past=0, causal=True),
        # one long prompt, 16 heads of 128
        dict(name="prompt_long", op="prompt", B=1, longest=16384, Hq=16, Hkv=4, d=128, past=0, causal=True),
        # single tokens of 4 sequences against their caches, 12 heads of 64
        dict(name="tree_token", op="tree", B=4, T=1, cap=8192, Hq=12, Hkv=12, d=64),
        # 16 drafted tokens for each of 16 sequences against long caches, shared key heads
        dict(name="tree_draft", op="tree", B=16, T=16, cap=32768, Hq=32, Hkv=8, d=128),
    ]


def _log(rng, lo, hi, step=1):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))


def draw(rng):
    """Sizes over the listed ranges; no case costs more than the largest listed one of its operator."""
    largest = {}
    for c in listed():
        w = work(c)
        largest[c["op"]] = max(largest.get(c["op"], 0), w["flops"] if c["op"] == "prompt" else w["bytes"])
    op = rng.choice(["embed", "embed_bwd", "logprob", "logprob", "logprob_bwd", "prompt", "prompt", "tree", "tree"])
    while True:
        if op in ("embed", "embed_bwd"):
            dtype = rng.choice(["bf16", "bf16", "f32"])
            c = dict(op=op, N=_log(rng, 1, 65536), V=_log(rng, 1000, 131072), D=_log(rng, 64, 2048, rng.choice([1, 8, 64])), dtype=dtype, pad=rng.random() < 0.5)
            c.update(dict(scale=rng.random() < 0.5) if op == "embed" else dict(grad=rng.choice(["f32", dtype]), into=rng.random() < 0.4))
        elif op in ("logprob", "logprob_bwd"):
            c = dict(op=op, N=_log(rng, 1, 16384), V=_log(rng, 1000, 131072), top=rng.choice([0, 1, 5, 20, 64]), dtype=rng.choice(["bf16", "bf16", "f32"]),
                     masked=rng.choice([0, 0, 13]), hot=rng.choice([1.0, 1.0, 0.7]))
            if op == "logprob":
                c["target"] = c["top"] == 0 or rng.random() < 0.7
            else:
                c["entropy"] = rng.random() < 0.5
        else:
            Hkv = rng.choice([1, 2, 4, 8, 12])
            c = dict(op=op, B=_log(rng, 1, 32), Hq=Hkv * rng.choice([1, 1, 2, 3, 4, 8]), Hkv=Hkv, d=rng.choice([64, 128]))
            if op == "prompt":
                c.update(longest=_log(rng, 1, 16384), past=rng.choice([0, 0, 0, 100, 1000]), causal=rng.random() < 0.85)
                # what the plain form holds at once
                if c["B"] * c["Hq"] * c["longest"] * (c["longest"] + c["past"]) > 7e9:
                    continue
            else:
                c.update(T=_log(rng, 1, 64), cap=_log(rng, 128, 65536))
                if c["B"] * c["Hq"] * c["T"] * c["cap"] > 3e9:
                    continue
        w = work(c)
        if (w["flops"] if op == "prompt" else w["bytes"]) <= largest[op]:
            return c


# ------------------------------------------------------------------ inputs


def _spread(n):
    """n numbers in (0, 1], spread evenly, the first of them 1."""
    return [1 - (0.6180339887 * b) % 1 for b in range(n)]


def _lengths(c):
    """(queries, keys) of each packed sequence."""
    lq = [max(1, round(c["longest"] * x)) for x in _spread(c["B"])]
    return lq, [n + (c["past"] + 37 * b if c["past"] else 0) for b, n in enumerate(lq)]


def _cached(c):
    """Keys in each sequence's cache before the drafted ones."""
    room = c["cap"] - c["T"]
    return [round(room * (0.125 + 0.875 * x)) for x in _spread(c["B"])]


def _words(c, g):
    """Token ids: the r-th most common of them about 1/r as often as the first; some -1, where a batch is padded."""
    u = torch.rand(c["N"], generator=g, device="cuda", dtype=F64)
    rank = torch.exp(u * math.log(c["V"] + 1)).long().clamp(1, c["V"]) - 1
    ids = torch.randperm(c["V"], generator=g, device="cuda")[rank]
    if c["pad"]:
        ids[torch.arange(c["N"], device="cuda") % 16 == 15] = -1
    return ids


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s, dtype=F32: torch.randn(*s, generator=g, device="cuda", dtype=F32).to(dtype)  # noqa: E731
    if c["op"] in ("embed", "embed_bwd"):
        dt = DTYPES[c["dtype"]]
        s = dict(c, ids=_words(c, g), factor=math.sqrt(c["D"]))
        if c["op"] == "embed":
            s["w"] = rand(c["V"], c["D"], dtype=dt)
            s["factor"] = s["factor"] if c["scale"] else 1.0
        else:
            s["dy"] = (1e-3 * rand(c["N"], c["D"])).to(dt)
            s["sum"] = (1e-2 * rand(c["V"], c["D"])).to(DTYPES[c["grad"]]) if c["into"] else None
        return s
    if c["op"] in ("logprob", "logprob_bwd"):
        N, V = c["N"], c["V"]
        common = torch.log1p(torch.arange(V, device="cuda", dtype=F32)) * -0.5  # common tokens have low numbers
        x = 2 * rand(N, V) + common
        if c["masked"]:
            x[:, V - c["masked"]:] = -math.inf
        s = dict(c, x=x.to(DTYPES[c["dtype"]]))
        t = torch.exp(torch.rand(N, generator=g, device="cuda") * math.log(V - c["masked"])).long().clamp(1, V - c["masked"]) - 1
        t[torch.arange(N, device="cuda") % 32 == 31] = -100  # padded ends
        s["t"] = t
        if c["op"] == "logprob_bwd":
            z = s["x"].double() * c["hot"]
            lse = torch.logsumexp(z, 1)
            logp = z - lse[:, None]
            s["lse"], s["H"] = lse.float(), -torch.where(logp == -math.inf, 0.0, logp.exp() * logp).sum(1).float()
            s["g"] = -torch.rand(N, generator=g, device="cuda") / N
            s["gH"] = 0.01 * rand(N) / N if c["entropy"] else None
            s["ids"], s["gtop"] = None, None
            if c["top"]:
                s["ids"], s["gtop"] = _best(s["x"], c["top"])[1], rand(N, c["top"]) / N
        else:
            s["t"] = t if c["target"] else None
        return s
    dt, Hq, Hkv, d = BF16, c["Hq"], c["Hkv"], c["d"]
    if c["op"] == "prompt":
        lq, lk = _lengths(c)
        edges = lambda n: torch.tensor([0, *np.cumsum(n).tolist()], device="cuda", dtype=torch.int32)  # noqa: E731
        s = dict(c, lq=lq, lk=lk, qs=edges(lq), ks=edges(lk) if c["past"] else None)
        s["q"] = (rand(sum(lq), Hq, d) * d ** -0.5 * 1.5).to(dt)  # the temperature is in q
        kv = rand(sum(lk), 2 * Hkv, d, dtype=dt)  # the projection's output
        s["k"], s["v"] = kv[:, :Hkv], kv[:, Hkv:]
        return s
    n = _cached(c)
    s = dict(c, n=torch.tensor(n, device="cuda", dtype=torch.int32), longest=max(n) + c["T"])
    s["q"] = (rand(c["B"], Hq, c["T"], d) * d ** -0.5 * 1.5).to(dt)
    s["keys"], s["values"] = (rand(c["B"], Hkv, c["cap"], d, dtype=dt) for _ in range(2))
    # drafted trees: a token's parent is one of the tokens before it (or it starts a branch: -1)
    up = (torch.rand(c["B"], c["T"], generator=g, device="cuda") * (torch.arange(c["T"], device="cuda") + 1)).long().cpu() - 1
    rows = []
    for b in range(c["B"]):
        seen = []
        for i, p in enumerate(up[b].tolist()):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows.append([w - (1 << 64) if w >> 63 else w for w in seen])
    s["tree"] = torch.tensor(rows, dtype=torch.int64, device="cuda") if c["T"] > 1 else None
    return s


# ------------------------------------------------------------------ one pass


def run(s):
    return {"embed": _embed, "embed_bwd": _embed_bwd, "logprob": _logprob, "logprob_bwd": _logprob_bwd, "prompt": _prompt, "tree": _tree}[s["op"]](s)


def _embed(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.embedding(s["ids"], s["w"], scale=s["factor"])
    rows = s["w"][s["ids"].clamp_min(0)].float() * s["factor"]
    return torch.where((s["ids"] >= 0)[:, None], rows, 0.0).to(s["w"].dtype)


def _embed_bwd(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.embedding_bwd(s["dy"], s["ids"], s["V"], scale=s["factor"], grad_dtype=DTYPES[s["grad"]], into=s["sum"])
    total = torch.zeros(s["V"] + 1, s["D"], device="cuda")
    total.index_add_(0, torch.where(s["ids"] < 0, s["V"], s["ids"]), s["dy"].float())
    total = total[:-1] * s["factor"]
    if s["into"]:
        s["sum"].copy_(s["sum"].float() + total)
        return s["sum"]
    return total.to(DTYPES[s["grad"]])


def _best(x, top):
    """The `top` largest of each row, the lower index first among equals: (values, indices); a masked entry is no alternative (index -1)."""
    bits = x.float().view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)  # as the values are ordered (-0 as 0)
    place = torch.arange(x.shape[1], device=x.device)
    at = (order * (1 << 24) - place).topk(min(top, x.shape[1]), 1)[1]
    best = x.gather(1, at).float()
    return best, torch.where(best == -math.inf, -1, at).int()


def _logprob(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        r = T.token_logprobs(s["x"], s["t"], top=s["top"], scale=s["hot"])
        return [r.logp, r.entropy, r.lse, r.top_logp, r.top_ids]
    x = s["x"].float() * s["hot"]
    m = x.amax(1, keepdim=True)
    e = torch.exp(x - m)
    total = e.sum(1, keepdim=True)
    lse = m + torch.log(total)
    entropy = torch.log(total) - torch.where(e == 0, 0.0, e * (x - m)).sum(1, keepdim=True) / total
    out = [None, entropy[:, 0], lse[:, 0], None, None]
    if s["t"] is not None:
        at = (x - m).gather(1, s["t"].clamp_min(0)[:, None]) - torch.log(total)
        out[0] = torch.where(s["t"] < 0, 0.0, at[:, 0])
    if s["top"]:
        best, out[4] = _best(s["x"], s["top"])
        out[3] = (best * s["hot"] - m) - torch.log(total)
    return out


def _logprob_bwd(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.token_logprobs_bwd(s["x"], s["lse"], targets=s["t"], dlogp=s["g"], entropy=s["H"], dentropy=s["gH"], top_ids=s["ids"], dtop=s["gtop"],
                                    scale=s["hot"])
    logp = s["x"].float() * s["hot"] - s["lse"][:, None]
    p = torch.exp(logp)
    g = torch.where(s["t"] < 0, 0.0, s["g"])[:, None]
    each = torch.zeros_like(p).scatter_add_(1, s["t"].clamp_min(0)[:, None], g)
    if s["top"]:
        h = torch.where(s["ids"] < 0, 0.0, s["gtop"])
        each.scatter_add_(1, s["ids"].long().clamp_min(0), h)
        g = g + h.sum(1, keepdim=True)
    each = each - p * g
    if s["gH"] is not None:
        each = each - s["gH"][:, None] * torch.where(p == 0, 0.0, p * (logp + s["H"][:, None]))
    return (each * s["hot"]).to(s["x"].dtype)


def _softmax(a, ok):
    """Rows of weights over the valid keys; zeros where a row has none."""
    a = torch.where(ok, a, -math.inf)
    a = torch.exp(a - a.amax(-1, keepdim=True).clamp_min(-3e38))
    return a / a.sum(-1, keepdim=True).clamp_min(1e-37)


def _prompt(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.prompt_attention(s["q"], s["k"], s["v"], s["qs"], k_starts=s["ks"], causal=s["causal"])
    B, Hkv, d, group = s["B"], s["Hkv"], s["d"], s["Hq"] // s["Hkv"]
    qs, ks = s["qs"].long(), (s["qs"] if s["ks"] is None else s["ks"]).long()
    i, j = torch.arange(max(s["lq"]), device="cuda"), torch.arange(max(s["lk"]), device="cuda")
    nq, nk = (qs[1:] - qs[:-1])[:, None], (ks[1:] - ks[:-1])[:, None]
    # every sequence in rows of its own
    q = s["q"][(qs[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)].float().view(B, -1, Hkv, group, d).permute(0, 2, 3, 1, 4)
    k, v = (x[(ks[:-1, None] + j).clamp_max(x.shape[0] - 1)].float().permute(0, 2, 1, 3)[:, :, None] for x in (s["k"], s["v"]))
    ok = (j < nk)[:, None, :]
    if s["causal"]:
        ok = ok & (j[None, None] <= (i + nk - nq)[:, :, None])
    a = _softmax(q @ k.transpose(-1, -2), ok[:, None, None])
    y = (a @ v).permute(0, 3, 1, 2, 4).reshape(B, -1, s["Hq"], d)
    return y[i < nq].to(BF16)


def _tree(s):
    if own:
        from paper_2106_06899_gb300 import topk as T

        return T.tree_attention(s["q"], s["keys"], s["values"], s["n"], tree=s["tree"])
    B, T, Hkv, d, n = s["B"], s["T"], s["Hkv"], s["d"], s["longest"]
    q = s["q"].float().view(B, Hkv, -1, T, d)
    k, v = (x[:, :, None, :n].float() for x in (s["keys"], s["values"]))
    j = torch.arange(n, device="cuda") - s["n"].long()[:, None]  # from the first drafted key on
    ok = (j < 0)[:, None].expand(B, T, n)
    if s["tree"] is None:
        ok = ok | (j == 0)[:, None]
    else:
        ok = ok | ((j >= 0) & (j < T))[:, None] & ((s["tree"][:, :, None] >> j.clamp(0, 63)[:, None]) & 1).bool()
    a = _softmax(q @ k.transpose(-1, -2), ok[:, None, None])
    return (a @ v).reshape(B, s["Hq"], T, d).to(BF16)


# ------------------------------------------------------------------ what a pass cannot do without


def _distinct(N, V):
    """How many different ids N draws of _words have, on average."""
    r = np.arange(1, V + 1, dtype=np.float64)
    return float((1 - np.exp(N * np.log1p(-np.log1p(1 / r) / math.log(V + 1)))).sum())


def work(case):
    c = case
    if c["op"] in ("embed", "embed_bwd"):
        e, N, D = (2 if c["dtype"] == "bf16" else 4), c["N"], c["D"]
        rows = _distinct(N, c["V"])
        if c["op"] == "embed":
            return {"bytes": int((N + min(N, rows)) * D * e + 8 * N), "flops": N * D}
        ge = 2 if c["grad"] == "bf16" else 4
        return {"bytes": int(N * D * e + 8 * N + (2 * rows if c["into"] else c["V"]) * D * ge), "flops": N * D}
    if c["op"] in ("logprob", "logprob_bwd"):
        e, cells = (2 if c["dtype"] == "bf16" else 4), c["N"] * c["V"]
        if c["op"] == "logprob":
            return {"bytes": cells * e + c["N"] * (20 + 8 * c["top"]), "flops": 8 * cells}
        return {"bytes": 2 * cells * e + c["N"] * (24 + 8 * c["top"]), "flops": 10 * cells}
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    if c["op"] == "prompt":
        lq, lk = _lengths(c)
        pairs = sum(a * b - (a * (a - 1) // 2 if c["causal"] else 0) for a, b in zip(lq, lk))
        return {"bytes": 4 * d * (Hq * sum(lq) + Hkv * sum(lk)), "flops": 4 * d * Hq * pairs}
    keys = sum(n + c["T"] for n in _cached(c))
    return {"bytes": 4 * d * (Hkv * keys + c["B"] * Hq * c["T"]), "flops": 4 * d * Hq * c["T"] * keys}


# ------------------------------------------------------------------ the definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    return {"embed": _exact_embed, "embed_bwd": _exact_embed_bwd, "logprob": _exact_logprob, "logprob_bwd": _exact_logprob_bwd, "prompt": _exact_prompt,
            "tree": _exact_tree}[s["op"]](s)


def _exact_embed(s):
    y = torch.zeros(s["N"], s["D"], dtype=F64, device="cuda")
    real = s["ids"] >= 0
    y[real] = torch.index_select(s["w"], 0, s["ids"][real]).to(F64) * s["factor"]
    return y


def _exact_embed_bwd(s):
    # the tokens in the order of their ids; a row's sum is the difference of two running sums, one block of columns after the other
    V = s["V"]
    order = torch.argsort(s["ids"], stable=True)
    edge = torch.searchsorted(s["ids"][order], torch.arange(V + 1, device="cuda"))
    out = torch.empty(V, s["D"], dtype=F64, device="cuda")
    for at in range(0, s["D"], 256):
        running = torch.cumsum(s["dy"][order, at:at + 256].to(F64), 0)
        running = torch.cat((torch.zeros_like(running[:1]), running))
        out[:, at:at + 256] = (running[edge[1:]] - running[edge[:-1]]) * s["factor"]
    return out + s["sum"].to(F64) if s["into"] else out


def _exact_logprob(s):
    parts = []
    for x in s["x"].split(max(1, (1 << 27) // s["V"])):
        z = x.to(F64) * s["hot"]
        lse = torch.logsumexp(z, 1, keepdim=True)
        parts.append([lse[:, 0], torch.special.entr(torch.exp(z - lse)).sum(1)])
        if s["top"]:
            parts[-1].append((torch.topk(x, s["top"], 1)[0].to(F64) * s["hot"]) - lse)
    lse, entropy, *best = (torch.cat(p) for p in zip(*parts))
    logp = None
    if s["t"] is not None:
        logp = torch.zeros_like(lse)
        for n, t in enumerate(s["t"].tolist()):
            if t >= 0:
                logp[n] = s["x"][n, t].to(F64) * s["hot"] - lse[n]
    return [logp, entropy, lse, best[0] if best else None, None]


def _exact_logprob_bwd(s):
    # the gradient of each output in turn: that of a log probability is a unit vector less p, that of the entropy -p (log p + H)
    out = torch.empty(s["N"], s["V"], dtype=F64, device="cuda")
    for n in range(0, s["N"], max(1, (1 << 26) // s["V"])):
        rows = slice(n, n + max(1, (1 << 26) // s["V"]))
        z = s["x"][rows].to(F64) * s["hot"]
        logp = torch.log_softmax(z, 1)
        p = torch.exp(logp)
        d = torch.zeros_like(p)
        pairs = [(s["t"][rows], s["g"][rows])] + ([(s["ids"][rows, m], s["gtop"][rows, m]) for m in range(s["ids"].shape[1])] if s["top"] else [])
        for t, g in pairs:
            r = torch.nonzero(t >= 0)[:, 0]
            d[r] -= p[r] * g[r, None].to(F64)
            d[r, t[r].long()] += g[r].to(F64)
        if s["gH"] is not None:
            H = torch.special.entr(p).sum(1, keepdim=True)
            d += s["gH"][rows, None].to(F64) * (torch.special.entr(p) - p * H)
        out[rows] = d * s["hot"]
    return out


def _attend(q, k, v, ok):
    """One head: q [n, d], k and v [m, d], ok [n, m]."""
    a = torch.einsum("nd,md->nm", q.to(F64), k.to(F64)).masked_fill_(~ok, -math.inf)
    return torch.einsum("nm,md->nd", torch.nan_to_num_(torch.softmax(a, 1), 0.0), v.to(F64))


def _exact_prompt(s):
    if work({k: s[k] for k in ("op", "B", "longest", "Hq", "Hkv", "d", "past", "causal")})["flops"] > 2e12:
        return None
    out = torch.empty(s["q"].shape, dtype=F64, device="cuda")
    group, at, bt = s["Hq"] // s["Hkv"], 0, 0
    for n, m in zip(s["lq"], s["lk"]):
        for first in range(0, n, 4096):  # of the queries
            rows = slice(first, min(n, first + 4096))
            ok = torch.ones(rows.stop - first, m, dtype=torch.bool, device="cuda")
            ok = ok.tril(m - n + first) if s["causal"] else ok
            for h in range(s["Hq"]):
                out[at + rows.start:at + rows.stop, h] = _attend(s["q"][at + rows.start:at + rows.stop, h], s["k"][bt:bt + m, h // group], s["v"][bt:bt + m, h // group], ok)
        at, bt = at + n, bt + m
    return out


def _exact_tree(s):
    out = torch.empty(s["q"].shape, dtype=F64, device="cuda")
    group, T = s["Hq"] // s["Hkv"], s["T"]
    for b, n in enumerate(s["n"].tolist()):
        ok = torch.ones(T, n + T, dtype=torch.bool, device="cuda")
        if s["tree"] is not None:
            seen = [[w >> j & 1 for j in range(T)] for w in s["tree"][b].tolist()]
            ok[:, n:] = torch.tensor(seen, device="cuda").bool()
        for h in range(s["Hkv"]):
            q = s["q"][b, h * group:(h + 1) * group].reshape(group * T, -1)
            y = _attend(q, s["keys"][b, h, :n + T], s["values"][b, h, :n + T], ok.repeat(group, 1))
            out[b, h * group:(h + 1) * group] = y.view(group, T, -1)
    return out
