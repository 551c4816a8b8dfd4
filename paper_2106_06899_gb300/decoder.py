"""A decoder stack composed of the library's calls: the 12-layer decoder of the paper's
benchmarks (Sec. 3, "12-layer decoder"), trained end to end.

Every layer is pre-LayerNorm causal self-attention followed by a feed-forward layer, each with
a residual connection.  The attention is top-k attention (Eq. 4) through the C ABI, forward with
the kept (index, score) cache and backward from that cache (Sec. 2.2); the feed-forward layer is
either the top-k FF layer (Eq. 3 with top-k) through the C ABI, forward and backward, or the
dense layer.  The projections, LayerNorms and the dense FF layer are ordinary PyTorch operations:
they are the model around the method, not part of it.  The temperature of Eq. 1 is folded into Q
(footnote to Eq. 1).

With fused=True (bf16) those, but for the LayerNorms, are the library's operators too: the projections with
their activation and residual (topk_linear_fwd / _bwd), and between the q/k/v projection and the attention
the norms of queries and keys with a rotation by position (topk_qk_norm_rope_fwd / _bwd).  The fused
decoder also generates, a token a step, against key/value caches (Decoder.step), after it has read packed prompts into
them (Decoder.prefill), or several drafted tokens a step (Decoder.step_tree).  With vocab=V it works on token ids: an
embedding before the first layer (topk_embedding_fwd / _bwd), the same weights behind the last norm, and
log probabilities with their gradient (topk_token_logprobs_fwd / _bwd).

The library's gradients have no gradients of their own: a second differentiation through one of these functions is
an error, and so is a forward-mode one.
A training step may be captured into a CUDA graph while no earlier eager graph of the same parameters is alive (drop the
losses of warm-up steps first, and run them on the capturing stream): PyTorch adds up a leaf's gradient on the stream where
its first graph was made, which ends a capture on another one.
"""
from __future__ import annotations

import itertools

import torch
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import topk as T


def _tangents(tensors) -> bool:
    """Whether one of the tensors (or None) has a forward-mode tangent, which the library's calls would drop."""
    if getattr(forward_ad, "_current_level", 0) < 0:  # outside of every dual level: 0.1 us in place of 0.3 for each tensor
        return False
    return any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


def _derived(*tensors) -> bool:
    """Whether a derivative by one of the tensors (or None) is wanted: a gradient, or a tangent, which the functions below refuse."""
    return (torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)) or _tangents(tensors)


class TopKAttentionFunction(torch.autograd.Function):
    """Top-k attention with the paper's caching: the forward pass keeps q, k, v and the kept
    (index, score) lists, O(L k) per head, and the backward pass recomputes only the activation."""

    @staticmethod
    def forward(ctx, q, k, v, topk: int, causal: bool):
        out, idx, score = T.attention(q, k, v, topk, causal=causal, return_indices=True)
        ctx.save_for_backward(q, k, v, idx, score)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        q, k, v, idx, score = ctx.saved_tensors
        dq, dk, dv = T.attention_bwd(q, k, v, dout.to(q.dtype).contiguous(), idx, score)
        return dq.to(q.dtype), dk.to(k.dtype), dv.to(v.dtype), None, None


class TopKFFNFunction(torch.autograd.Function):
    """The top-k FF layer with the same caching: x [N, d_model], W1/W2 [d_ff, d_model] (bf16)."""

    @staticmethod
    def forward(ctx, x, w1, w2, topk: int):
        out, idx, score = T.ffn(x, w1, w2, topk, return_indices=True)
        ctx.save_for_backward(x, w1, w2, idx, score)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        x, w1, w2, idx, score = ctx.saved_tensors
        dx, d1, d2 = T.ffn_bwd(x, w1, w2, dout.float().contiguous(), idx, score)
        return dx.to(x.dtype), d1.to(w1.dtype), d2.to(w2.dtype), None


class LinearFunction(torch.autograd.Function):
    """act(x w^T) + residual for x [M, K], w [N, K] (bf16).  The backward pass needs the pre-activations, but for
    ReLU, whose slope is the sign of its output, only where a residual was added to that."""

    @staticmethod
    def forward(ctx, x, w, act: str, residual):
        if act == "none" or (act == "relu" and residual is None):
            y = T.linear(x, w, act=act, residual=residual)
            z = None if act == "none" else y
        else:
            y, z = T.linear(x, w, act=act, residual=residual, return_preact=True)
        ctx.save_for_backward(x, w, z)
        ctx.act, ctx.has_residual = act, residual is not None
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, w, z = ctx.saved_tensors
        dy = dy.contiguous()
        dx = dw = None
        if any(ctx.needs_input_grad[:2]):
            dx, dw, _ = T.linear_bwd(dy, x, w, z, ctx.act, need_dx=ctx.needs_input_grad[0], need_dw=ctx.needs_input_grad[1])
        return dx, dw, None, dy if ctx.has_residual else None


def linear(x, w, act: str = "none", residual=None):
    """LinearFunction where a derivative is wanted, else the library's call, which then keeps nothing."""
    if _derived(x, w, residual):
        return LinearFunction.apply(x, w, act, residual)
    return T.linear(x, w, act=act, residual=residual)


class RotaryAttentionFunction(torch.autograd.Function):
    """Norms, rotation and causal attention of a packed projection qkv [B, L, 3 H, d] (q's heads, k's, v's): top-k
    attention, whose fp32 gradients go straight into the rotation's backward pass.  Of the projection and what attention
    reads only the projection is kept: the backward pass turns it again (twelve layers of 768, 32,768 tokens: 1.8 GB less)."""

    @staticmethod
    def turned(qkv, q_weight, k_weight, cos, sin):
        H = qkv.shape[2] // 3
        return T.qk_norm_rope(qkv[:, :, :H], qkv[:, :, H:2 * H], qkv[:, :, 2 * H:], cos, sin, q_weight=q_weight, k_weight=k_weight,
                              q_scale=qkv.shape[3] ** -0.5)

    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, cos, sin, topk: int):
        q, k, v = RotaryAttentionFunction.turned(qkv, q_weight, k_weight, cos, sin)
        out, idx, score = T.attention(q, k, v, topk, causal=True, return_indices=True)
        ctx.save_for_backward(qkv, q_weight, k_weight, cos, sin, idx, score)
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dout):
        qkv, q_weight, k_weight, cos, sin, idx, score = ctx.saved_tensors
        H = qkv.shape[2] // 3
        q, k, v = RotaryAttentionFunction.turned(qkv, q_weight, k_weight, cos, sin)
        dq, dk, dv = T.attention_bwd(q, k, v, dout.to(q.dtype).contiguous(), idx, score)
        dqkv, dqw, dkw = T.qk_norm_rope_bwd(dq, dk, dv, qkv[:, :, :H], qkv[:, :, H:2 * H], cos, sin, q_weight=q_weight, k_weight=k_weight,
                                            q_scale=qkv.shape[3] ** -0.5)
        return dqkv, dqw.to(q_weight.dtype), dkw.to(k_weight.dtype), None, None, None


class QKNormRopeFunction(torch.autograd.Function):
    """Norms and rotation alone: qkv [B, L, 3 H, d] to q, k, v [B, H, L, d]."""

    @staticmethod
    def forward(ctx, qkv, q_weight, k_weight, cos, sin):
        H = qkv.shape[2] // 3
        ctx.save_for_backward(qkv, q_weight, k_weight, cos, sin)
        return T.qk_norm_rope(qkv[:, :, :H], qkv[:, :, H:2 * H], qkv[:, :, 2 * H:], cos, sin, q_weight=q_weight, k_weight=k_weight,
                              q_scale=qkv.shape[3] ** -0.5)

    @staticmethod
    @once_differentiable
    def backward(ctx, dq, dk, dv):
        qkv, q_weight, k_weight, cos, sin = ctx.saved_tensors
        H = qkv.shape[2] // 3
        dqkv, dqw, dkw = T.qk_norm_rope_bwd(dq.contiguous(), dk.contiguous(), dv.contiguous(), qkv[:, :, :H], qkv[:, :, H:2 * H], cos, sin,
                                            q_weight=q_weight, k_weight=k_weight, q_scale=qkv.shape[3] ** -0.5)
        return dqkv, dqw.to(q_weight.dtype), dkw.to(k_weight.dtype), None, None


class EmbeddingFunction(torch.autograd.Function):
    """scale weight[ids]; ids below 0 are padding."""

    @staticmethod
    def forward(ctx, ids, weight, scale: float):
        ctx.save_for_backward(ids)
        ctx.rows, ctx.dtype, ctx.scale = weight.shape[0], weight.dtype, scale
        return T.embedding(ids, weight, scale=scale)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        (ids,) = ctx.saved_tensors
        return None, T.embedding_bwd(dy.contiguous(), ids, ctx.rows, scale=ctx.scale, grad_dtype=ctx.dtype), None


class TokenLogProbsFunction(torch.autograd.Function):
    """T.token_logprobs of logits [N, V]; logp, entropy and top_logp have gradients, lse and top_ids none."""

    @staticmethod
    def forward(ctx, logits, targets, top: int, scale: float):
        r = T.token_logprobs(logits, targets, top=top, scale=scale)
        ctx.save_for_backward(logits, targets, r.lse, r.entropy, r.top_ids)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        ctx.mark_non_differentiable(*(t for t in (r.lse, r.top_ids) if t is not None))
        return tuple(r)

    @staticmethod
    @once_differentiable
    def backward(ctx, dlogp, dentropy, _lse, dtop, _ids):
        logits, targets, lse, entropy, ids = ctx.saved_tensors
        if dlogp is None and dentropy is None and dtop is None:
            return None, None, None, None
        dlogp, dentropy, dtop = (None if g is None else g.contiguous() for g in (dlogp, dentropy, dtop))
        return T.token_logprobs_bwd(logits, lse, targets=targets, dlogp=dlogp, entropy=entropy, dentropy=dentropy, top_ids=ids, dtop=dtop,
                                    scale=ctx.scale), None, None, None


class WithoutGradientFunction(torch.autograd.Function):
    """x as it is, for a user who looks at it; in a loss of `of` it is an error, where a part of the gradient would be missing."""

    @staticmethod
    def forward(ctx, x, of, name: str):
        ctx.name = name
        return x.view_as(x)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError(f"{ctx.name} has no gradient: detach it, or leave it out of the loss")


class DecoderLayer(torch.nn.Module):
    def __init__(self, d_model: int, heads: int, d_ff: int, topk: int | None, ffn_topk: int | None,
                 dtype=torch.bfloat16, device="cuda", fused: bool = False):
        super().__init__()
        self.h, self.dh = heads, d_model // heads
        self.topk, self.ffn_topk, self.fused = topk, ffn_topk, fused
        if fused and dtype != torch.bfloat16:
            raise ValueError("the fused decoder is bfloat16")
        kw = dict(dtype=dtype, device=device)
        self.ln1 = torch.nn.LayerNorm(d_model, **kw)
        self.ln2 = torch.nn.LayerNorm(d_model, **kw)
        self.qkv = torch.nn.Linear(d_model, 3 * d_model, bias=False, **kw)
        self.proj = torch.nn.Linear(d_model, d_model, bias=False, **kw)
        # FF keys and values are the rows of W1 and W2 (Sec. 2.1)
        self.w1 = torch.nn.Parameter(torch.randn(d_ff, d_model, **kw) * d_model ** -0.5)
        self.w2 = torch.nn.Parameter(torch.randn(d_ff, d_model, **kw) * d_ff ** -0.5)
        if fused:
            self.q_norm, self.k_norm = (torch.nn.Parameter(torch.ones(self.dh, **kw)) for _ in range(2))
            if ffn_topk is None:  # the dense layer's second product takes W2 as a linear layer's weight
                self.w2 = torch.nn.Parameter(self.w2.detach().t().contiguous())

    def attention(self, q, k, v):
        if self.topk is None:  # plain causal attention (PyTorch), the comparison
            return torch.nn.functional.scaled_dot_product_attention(q, k, v, is_causal=True, scale=1.0)
        return TopKAttentionFunction.apply(q, k, v, self.topk, True)

    def feed_forward(self, h):
        if self.ffn_topk is None:
            return torch.relu(h @ self.w1.t()) @ self.w2
        return TopKFFNFunction.apply(h.contiguous(), self.w1, self.w2, self.ffn_topk).to(h.dtype)

    def _fused_tail(self, a, x):
        """Output projection and feed-forward layer, each with its residual: a (attention, [M, D]), x [M, D]."""
        x = linear(a, self.proj.weight, residual=x)
        h = self.ln2(x)
        if self.ffn_topk is None:
            return linear(linear(h, self.w1, "relu"), self.w2, residual=x)
        return x + TopKFFNFunction.apply(h.contiguous(), self.w1, self.w2, self.ffn_topk).to(h.dtype)

    def forward_fused(self, x, tables):
        B, L, D = x.shape
        x = x.reshape(B * L, D)
        qkv = linear(self.ln1(x), self.qkv.weight).view(B, L, 3 * self.h, self.dh)
        if self.topk is None:
            a = self.attention(*QKNormRopeFunction.apply(qkv, self.q_norm, self.k_norm, *tables))
        else:
            a = RotaryAttentionFunction.apply(qkv, self.q_norm, self.k_norm, *tables, min(self.topk, L))
        return self._fused_tail(a.transpose(1, 2).reshape(B * L, D), x).view(B, L, D)

    def _cached(self, x, cache, start, positions, tables):
        """Queries [B, H, T, d] of x [B, T, D], whose keys and values go into the caches at rows start[b] on."""
        B, T_, D = x.shape
        qkv = T.linear(self.ln1(x).view(B * T_, D), self.qkv.weight).view(B, T_, 3 * self.h, self.dh)
        return T.qk_norm_rope(qkv[:, :, :self.h], qkv[:, :, self.h:2 * self.h], qkv[:, :, 2 * self.h:], *tables, cache=cache, cache_start=start,
                              positions=positions, q_weight=self.q_norm, k_weight=self.k_norm, q_scale=self.dh ** -0.5)[0]

    def step(self, x, cache, start, positions, tables):
        """One token for each of B sequences, x [B, D]: keys and values go into the caches [B, H, cap, d] at rows
        start [B], and attention reads the rows up to them."""
        B, D = x.shape
        keys, values = cache
        q = self._cached(x.view(B, 1, D), cache, start, positions, tables)
        if self.topk is None:
            a = T.vanilla_attention(q, keys, values, kv_len=start + 1)
        else:
            a = T.attention(q, keys, values, min(self.topk, keys.shape[2]), kv_len=start + 1)
        return self._fused_tail(a.view(B, D), x)

    def step_tree(self, x, cache, start, positions, tables, tree, mask):
        """T drafted tokens of each of B sequences, x [B, T, D], behind the start[b] rows that the caches hold.  They read by tree,
        or, with top-k attention, by mask [B, 1, T, cap]."""
        B, T_, D = x.shape
        q = self._cached(x, cache, start, positions, tables)
        if self.topk is None:
            a = T.tree_attention(q, *cache, start, tree=tree)
        else:
            a = T.attention(q, *cache, min(self.topk, mask.shape[3]), mask=mask)
        return self._fused_tail(a.transpose(1, 2).reshape(B * T_, D), x.view(B * T_, D)).view(B, T_, D)

    def prefill(self, x, cache, starts, token, positions, rows, tables):
        """Packed prompts x [T, D] with plain attention; the keys and values of tokens token [T] go to rows positions of the caches of
        sequences rows."""
        n, D = x.shape
        qkv = T.linear(self.ln1(x), self.qkv.weight).view(1, n, 3 * self.h, self.dh)
        q, k, v = (t[0].transpose(0, 1) for t in T.qk_norm_rope(
            qkv[:, :, :self.h], qkv[:, :, self.h:2 * self.h], qkv[:, :, 2 * self.h:], *tables, positions=positions.view(1, 1, n),
            q_weight=self.q_norm, k_weight=self.k_norm, q_scale=self.dh ** -0.5))
        for c, t in zip(cache, (k, v)):
            c[rows, :, positions[token]] = t[token]
        return self._fused_tail(T.prompt_attention(q, k, v, starts).view(n, D), x)

    def forward(self, x):
        B, L, D = x.shape
        qkv = self.qkv(self.ln1(x)).view(B, L, 3, self.h, self.dh).permute(2, 0, 3, 1, 4)
        q = (qkv[0] * self.dh ** -0.5).contiguous()  # Eq. 1's temperature folded into Q
        k, v = qkv[1].contiguous(), qkv[2].contiguous()
        a = self.attention(q, k, v)
        x = x + self.proj(a.transpose(1, 2).reshape(B, L, D))
        f = self.feed_forward(self.ln2(x).reshape(B * L, D))
        return x + f.view(B, L, D)


class Decoder(torch.nn.Module):
    """n_layers decoder layers over d_model features; topk / ffn_topk None selects the plain
    attention / the dense FF layer.  fused: the library's linear layers, and queries and keys normalised and
    rotated by their positions, of which there are max_positions.  vocab (fused; a multiple of 8): token ids in the place of
    features, by an embedding that is also the output projection; ids below 0 are padding."""

    def __init__(self, n_layers=12, d_model=768, heads=12, d_ff=3072, topk: int | None = 64,
                 ffn_topk: int | None = None, dtype=torch.bfloat16, device="cuda", fused: bool = False,
                 max_positions: int = 65536, vocab: int | None = None):
        super().__init__()
        if vocab is not None and (not fused or vocab % 8):
            raise ValueError("a vocabulary needs a fused decoder and a multiple of 8")
        self.layers = torch.nn.ModuleList(
            DecoderLayer(d_model, heads, d_ff, topk, ffn_topk, dtype, device, fused) for _ in range(n_layers))
        self.norm = torch.nn.LayerNorm(d_model, dtype=dtype, device=device)
        self.fused = fused
        self.tables = T.rope_tables(max_positions, d_model // heads, device=device) if fused else None
        self.vocab = vocab
        if vocab is not None:
            self.embedding = torch.nn.Parameter(torch.randn(vocab, d_model, dtype=dtype, device=device) * d_model ** -0.5)

    def _apply(self, fn, recurse=True):
        super()._apply(fn, recurse)
        # the tables go where the parameters go, but stay in 32 bits and out of the state_dict
        device = self.norm.weight.device
        if self.tables is not None and self.tables[0].device != device:
            rows, half = self.tables[0].shape
            self.tables = T.rope_tables(rows, 2 * half, device=device)
        return self

    def _features(self, x):
        """Features of token ids (int32 or int64, any shape), or x as it is."""
        if self.vocab is None or x.is_floating_point():
            return x
        x, scale = x.contiguous(), self.embedding.shape[1] ** 0.5
        if _derived(self.embedding):
            return EmbeddingFunction.apply(x, self.embedding, scale)
        return T.embedding(x, self.embedding, scale=scale)

    def _served(self, x):
        """_features for calls that have no derivatives."""
        if _tangents(itertools.chain((x,), self.parameters())):
            raise NotImplementedError("generation has no forward-mode derivative")
        return self._features(x).contiguous()

    def forward(self, x):
        x = self._features(x)
        for layer in self.layers:
            x = layer.forward_fused(x, self.tables) if self.fused else layer(x)
        return self.norm(x)

    def logprobs(self, features, targets=None, top: int = 0, scale: float = 1.0) -> T.TokenLogProbs:
        """What features [.., d_model] (of forward, step, ..) say of the next tokens: T.token_logprobs of their logits, one row for
        each of them, with targets [..] or None.  Differentiable where gradients are on, but for lse, which a loss may hold only detached."""
        if self.vocab is None:
            raise ValueError("logprobs() needs a vocabulary")
        # reshape leaves views such as the last tokens' features[:, -1] as they are
        logits = linear(features.reshape(-1, features.shape[-1]).contiguous(), self.embedding)
        targets = None if targets is None else targets.reshape(-1).contiguous()
        if _derived(logits):
            r = T.TokenLogProbs(*TokenLogProbsFunction.apply(logits, targets, top, scale))
            return r._replace(lse=WithoutGradientFunction.apply(r.lse, logits, "lse"))
        return T.token_logprobs(logits, targets, top=top, scale=scale)

    def new_cache(self, batch: int, capacity: int):
        """Key/value caches of every layer, [batch, heads, capacity, d] each, for step()."""
        w = self.norm.weight
        return [tuple(torch.zeros(batch, layer.h, capacity, layer.dh, dtype=w.dtype, device=w.device) for _ in range(2))
                for layer in self.layers]

    @torch.no_grad()
    def step(self, x, caches, start):
        """The next token of each of B sequences (fused only): x [B, d_model] (or ids [B]) at positions start [B] (int32), the
        caches (new_cache) holding the tokens before; returns [B, d_model] and leaves the token in the caches."""
        if not self.fused:
            raise ValueError("step() needs a fused decoder")
        x = self._served(x)
        positions = start.view(1, -1, 1)
        for layer, cache in zip(self.layers, caches):
            x = layer.step(x, cache, start, positions, self.tables)
        return self.norm(x)

    @torch.no_grad()
    def prefill(self, x, starts, caches):
        """Reads packed prompts (fused, plain attention) into empty caches: x [T, d_model] (or ids [T]), sequence b's in rows
        starts[b] to starts[b + 1] - 1 ([B + 1] int32, from 0 to T); returns [T, d_model]."""
        if not self.fused or any(layer.topk is not None for layer in self.layers):
            raise ValueError("prefill() needs a fused decoder with plain attention (topk=None)")
        n, cap, ends = x.shape[0], caches[0][0].shape[2], starts.long()
        if not 2 <= starts.shape[0] <= caches[0][0].shape[0] + 1:
            raise ValueError("starts must have from one to the caches' number of sequences, and an end")
        if n > cap and int((ends[1:] - ends[:-1]).max()) > cap:  # the host waits for the lengths only where they could be too long
            raise ValueError("the caches have no room for the longest prompt")
        x = self._served(x)
        # rows of no sequence write what the nearest token of one does
        token = torch.minimum(torch.maximum(torch.arange(n, device=x.device), ends[0]), (ends[-1] - 1).clamp_min(0)).clamp(0, n - 1)
        rows = torch.searchsorted(ends[1:], token, right=True).clamp_max(ends.shape[0] - 2)
        at = (token - ends[rows]).clamp(0, cap - 1)
        positions = torch.zeros(n, dtype=torch.int64, device=x.device).index_put_((token,), at)
        for layer, cache in zip(self.layers, caches):
            x = layer.prefill(x, cache, starts, token, positions.int(), rows, self.tables)
        return self.norm(x)

    @torch.no_grad()
    def step_tree(self, x, caches, start, tree=None):
        """T drafted tokens of each of B sequences at once (fused only): x [B, T, d_model] (or ids [B, T]) behind the start [B]
        (int32) tokens that the caches hold.  tree [B, T] (T.tree_mask): which drafted tokens each one reads, its ancestors and itself;
        None: a chain.  Returns [B, T, d_model] and leaves the tokens in rows start[b] on; keep() makes a path of them the sequence's."""
        if not self.fused:
            raise ValueError("step_tree() needs a fused decoder")
        x = self._served(x)
        B, n, _ = x.shape
        i = torch.arange(n, device=x.device)
        reads = (i <= i[:, None]).expand(B, n, n) if tree is None else (tree.expand(B, n)[..., None] >> i & 1).bool()
        positions = (start[:, None] + reads.sum(-1) - 1).int()[None].contiguous()
        mask = None
        if any(layer.topk is not None for layer in self.layers):
            j = torch.arange(caches[0][0].shape[2], device=x.device) - start[:, None].long()  # from the first drafted row on
            drafted = reads.gather(2, j.clamp(0, n - 1)[:, None].expand(B, n, j.shape[1])) & ((j >= 0) & (j < n))[:, None]
            mask = ((j < 0)[:, None] | drafted)[:, None]
        for layer, cache in zip(self.layers, caches):
            x = layer.step_tree(x, cache, start, positions, self.tables, tree, mask)
        return self.norm(x)

    @torch.no_grad()
    def keep(self, caches, start, path):
        """Moves the drafted tokens path [B, n] (indices into step_tree's, a token and its descendants in order) to rows start[b] to
        start[b] + n - 1 of the caches; an index that repeats fills up a shorter path.  Rows outside the caches are cut to them."""
        B, n = path.shape
        if B != start.shape[0] or B > caches[0][0].shape[0]:
            raise ValueError("path must have a row for each of start's sequences, which the caches hold")
        b = torch.arange(B, device=path.device)[:, None]
        last = caches[0][0].shape[2] - 1
        to, of = ((start.long()[:, None] + i).clamp(0, last) for i in (torch.arange(n, device=path.device), path.long()))
        for cache in caches:
            for c in cache:
                c[b, :, to] = c[b, :, of]
