/*
 * topk_attention.h -- C ABI of libtopk.so: top-k attention and the top-k
 * feed-forward layer (Gupta et al., "Memory-efficient Transformers via Top-k
 * Attention", arXiv 2106.06899) on NVIDIA GB300 (sm_103a).
 *
 * Operations
 *   topk_attn_fwd  -- Eq. 4 (Sec. 2.2):  out = softmax(top-k(Q K^T)) V, row by
 *                     row, the softmax taken over the k kept entries only.
 *                     The temperature of Eq. 1 is folded into Q by the caller
 *                     (footnote to Eq. 1).  Optional causal mask, Eq. 2: the
 *                     queries are the last Lq of the Lk positions (Lq <= Lk;
 *                     Lq < Lk is decoding against a key/value cache), and key
 *                     j is valid for query i iff j <= i + Lk - Lq.
 *   topk_attn_fwd_masked -- the same under Eq. 2's general mask B in {0, -inf}:
 *                     per-batch key counts and an arbitrary bit mask as well.
 *   topk_ffn_fwd   -- Eq. 3 with top-k (Sec. 2.1 "Feed-forward as attention"):
 *                     out = sum over the k largest s_j = x . W1_j of
 *                     ReLU(s_j) * W2_j.  Keys and values are the ROWS of W1
 *                     and W2.
 *   topk_attn_bwd  -- the backward pass of Eq. 4 for the kept set the forward
 *   topk_ffn_bwd      pass cached (Sec. 2.2 "Improving efficiency through
 *                     top-k attention"): gradients of q, k, v (x, W1, W2)
 *                     from dout, the kept indices and their scores, with the
 *                     activation recomputed from the cached scores.
 * Query chunking (Sec. 2.2 "Query chunking") bounds scheduling only: results
 * never depend on `chunk`, and no [chunk x L_K] score matrix is ever stored
 * in device memory.
 *
 * Selection rule: each row keeps the first k entries of the total order
 * (score descending, key index ascending) among its valid keys, i.e. ties go
 * to the lower key index.  A row with fewer than k valid keys keeps all of
 * them; a row with none outputs zeros (its indices are all -1).
 *
 * Conventions shared by every call
 *   - Tensor pointers are DEVICE pointers (except the *_host entry points),
 *     owned by the caller, contiguous, row-major, 16-byte aligned.
 *     (topk_qk_norm_rope_fwd takes strided q, k and v.)
 *   - Shapes: q, out [B, H, Lq, d]; k, v [B, H, Lk, d];
 *             x [N, d_model]; W1, W2 [d_ff, d_model]; ffn out [N, d_model].
 *   - dtype: TOPK_F32 (fp32 in/out, fp32 FMA scores, never TF32) or
 *            TOPK_BF16 (bf16 in/out, fp32 accumulation).  The feed-forward
 *            call takes bf16 inputs and writes fp32 output.
 *   - `stream` is a cudaStream_t (NULL = legacy default stream).  Calls
 *     enqueue work and return without synchronising.
 *   - Every argument is validated before anything is launched, so an error
 *     return never leaves a partial write.
 *   - Scratch, where a call needs it, is taken on `stream` from a
 *     stream-ordered memory pool that the library owns (one per device) and
 *     returned to it on `stream`; its size is reported by the
 *     *_workspace_bytes queries and is never proportional to Lq * Lk: a
 *     fixed amount per SM for attention (plus, when a grid of few query
 *     tiles is split into key parts, each part's kept list per row), linear
 *     in the tokens for the feed-forward layer and in the cache for the
 *     backward calls.  The pool keeps returned memory
 *     reserved for later calls (up to the largest amount in use at once),
 *     so that repeated calls do not map device memory again each time, until
 *     topk_pool_trim() hands it back or the process exits;
 *     topk_pool_usage() reports it.
 *
 * Return codes: 0 on success, else one of the negative TOPK_ERR_* values;
 * topk_error_string() describes them.
 */
#ifndef TOPK_ATTENTION_H
#define TOPK_ATTENTION_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { TOPK_F32 = 0, TOPK_BF16 = 1 } topk_dtype;

enum {
  TOPK_OK = 0,
  TOPK_ERR_INVALID_ARG = -1, /* null pointer, non-positive size, topk < 1 or > keys, chunk < 1,
                                causal with Lq > Lk, negative mask stride, unknown dtype */
  TOPK_ERR_UNSUPPORTED = -2, /* valid but not implemented: head size, topk above the
                                kernel's limit, pointer not 16-byte aligned */
  TOPK_ERR_CUDA = -3,        /* a CUDA runtime/driver call or a launch failed */
  TOPK_ERR_TIMEOUT = -4,     /* a device pipeline wait ran out its time limit; the
                                kernel stopped early and its outputs are invalid */
  TOPK_ERR_WORKSPACE = -5,   /* an internal consistency check of the selection
                                failed (no input is known to cause it; candidate
                                lists are compacted exactly rather than overflow);
                                outputs invalid */
  TOPK_ERR_NO_DEVICE = -6,   /* no usable sm_103 device */
  TOPK_ERR_SCRATCH_LIMIT = -7, /* the problem needs more scratch than the fixed buffer of
                                 topk_ffn_fwd_noalloc holds */
  TOPK_ERR_RANGE = -8        /* a position outside the rotation tables (its nearest row was used) or
                                a row outside the cache (not written); reported by topk_check() */
};

/*
 * Top-k attention forward, Eq. 4 (Sec. 2.2), optionally causal (Eq. 2).
 *   q, k, v, out : device pointers, layouts above, element type `dtype`.
 *   B, H         : batch and heads; every (b, h) is an independent problem.
 *   Lq, Lk       : query and key counts (causal requires Lq <= Lk).
 *   d            : head size.  TOPK_BF16: 64 or 128.  TOPK_F32: 16, 32, 64, 128.
 *   topk         : 1 <= topk <= Lk; the supported maximum is 512.
 *   chunk        : query-chunk size (Sec. 2.2), >= 1; a scheduling hint only.
 *   causal       : 0 or 1.
 *   Scratch: topk_attn_workspace_bytes() (a fixed amount per SM, or none;
 *            plus parts x B*H*Lq x (8 topk + 4) bytes where at most half the
 *            SMs would get a query tile and the key tiles are split into parts).
 * Errors: TOPK_ERR_INVALID_ARG / TOPK_ERR_UNSUPPORTED before any launch;
 *         TOPK_ERR_CUDA if a launch fails (or the scratch cannot be had).
 *         A device-side timeout is not returned by this call (it returns
 *         once the work is enqueued): topk_check() and the *_host calls
 *         report it, from the device's error word (see topk_check).
 */
int topk_attn_fwd(const void* q, const void* k, const void* v, void* out, int B, int H, int Lq, int Lk,
                  int d, int topk, int chunk, int causal, int dtype, void* stream);

/*
 * Same as topk_attn_fwd, and additionally writes, per query row, the kept
 * key indices and their fp32 scores in selection order (score descending,
 * index ascending).  idx [B, H, Lq, topk] int32, -1 padded; score same shape,
 * fp32, -inf padded.  Either may be NULL.  Used for parity checks.
 */
int topk_attn_fwd_indices(const void* q, const void* k, const void* v, void* out, int B, int H, int Lq,
                          int Lk, int d, int topk, int chunk, int causal, int dtype, int32_t* idx,
                          float* score, void* stream);

/*
 * Top-k attention under the general mask of Eq. 2 (Sec. 2.1): B_ij = -inf
 * removes key j from query i's candidates before the top-k.  Three masks
 * combine (a key must pass all of them):
 *   causal  : 0 or 1, as in topk_attn_fwd (key j valid iff j <= i + Lk - Lq).
 *   kv_len  : NULL, or [B] int32 device pointer: key j is valid for every query
 *             of batch b iff j < kv_len[b] (key padding; values are clamped to
 *             [0, Lk]).
 *   mask    : NULL, or a uint32 device bit array: key j is valid for query i of
 *             (b, h) iff bit (j % 32) of word
 *               b * mask_batch_stride + h * mask_head_stride + i * W + j / 32,
 *             W = ceil(Lk / 32), is 1.  A stride of 0 shares the mask across
 *             batches or heads.  4-byte aligned.
 * A row with fewer than k valid keys keeps all of them; a row with none writes
 * zeros.  Other arguments as topk_attn_fwd_indices (idx/score may be NULL).
 * With a bit mask the scores run on the CUDA cores (fp32 FMA of the exact
 * bf16/fp32 inputs); causal and kv_len alone keep the tensor-core kernel.
 * Errors: as topk_attn_fwd; a negative stride is TOPK_ERR_INVALID_ARG, a
 * misaligned mask or kv_len TOPK_ERR_UNSUPPORTED.
 */
int topk_attn_fwd_masked(const void* q, const void* k, const void* v, void* out, int B, int H, int Lq, int Lk,
                         int d, int topk, int chunk, int causal, const int32_t* kv_len, const uint32_t* mask,
                         long long mask_batch_stride, long long mask_head_stride, int dtype, int32_t* idx,
                         float* score, void* stream);

/*
 * Plain (vanilla) attention, Eq. 1 (Sec. 2.1), under Eq. 2's causal mask and
 * per-batch key counts: the softmax covers every valid key.  It is the path
 * the paper compares top-k attention with (Sec. 3; query chunking, Sec. 2.2,
 * bounds its memory there): here the score tile stays on chip, so no
 * [chunk x Lk] buffer exists and `chunk` is validated but has no effect.
 *   q, k, v, out, B, H, Lq, Lk, causal, kv_len: as topk_attn_fwd_masked.
 *   d      : 64 or 128.  dtype: TOPK_BF16 only (fp32 is TOPK_ERR_UNSUPPORTED).
 *   B * H  : at most 65535.
 *   Scratch: topk_vanilla_attn_workspace_bytes() (V transposed, B*H*d*Lk*2
 *   bytes rounded up), from the library's pool.  A row with no valid key
 *   writes zeros.  Errors as topk_attn_fwd.
 */
int topk_vanilla_attn_fwd(const void* q, const void* k, const void* v, void* out, int B, int H, int Lq, int Lk,
                          int d, int chunk, int causal, const int32_t* kv_len, int dtype, void* stream);
size_t topk_vanilla_attn_workspace_bytes(int B, int H, int Lq, int Lk, int d, int dtype);

/*
 * The dense feed-forward layer, Eq. 3 without top-k (Sec. 2.1): out =
 * ReLU(x W1^T) W2, the comparison path for topk_ffn_fwd (Sec. 3).  d_ff is
 * taken in slices of `chunk` keys (chunking bounds the memory, Sec. 2.2): per
 * slice the hidden activations [N, chunk] are formed in bf16, ReLU'd and
 * multiplied into the fp32 output.  The two products run in cuBLAS (plain
 * GEMMs, bf16 inputs, fp32 accumulation); ReLU in the library's own kernel.
 *   x, W1, W2, out, N, d_model, d_ff: as topk_ffn_fwd (d_model a multiple of 8).
 *   chunk  : keys per slice, >= 1; a multiple of 8 unless it covers all of d_ff.
 *   Scratch: topk_vanilla_ffn_workspace_bytes() = N * min(chunk, d_ff) * 2 bytes.
 */
int topk_vanilla_ffn_fwd(const void* x, const void* W1, const void* W2, void* out, int N, int d_model, int d_ff,
                         int chunk, void* stream);
size_t topk_vanilla_ffn_workspace_bytes(int N, int d_model, int d_ff, int chunk);

/*
 * Top-k feed-forward layer, Eq. 3 with the top-k of Eq. 4 and ReLU as the
 * activation (Sec. 2.1, Sec. 2.2).
 *   x  : [N, d_model] bf16 device pointer (the queries).
 *   W1 : [d_ff, d_model] bf16; row j is key j.
 *   W2 : [d_ff, d_model] bf16; row j is value j.
 *   out: [N, d_model] fp32 device pointer.
 *   d_model: a multiple of 64, at most 4096.  1 <= topk <= d_ff, topk <= 1024.
 *   Scratch: topk_ffn_workspace_bytes(); it grows linearly with N.
 * Top-k is taken over the signed scores; ReLU is applied after selection.
 */
int topk_ffn_fwd(const void* x, const void* W1, const void* W2, void* out, int N, int d_model, int d_ff,
                 int topk, void* stream);

/* topk_ffn_fwd plus the kept indices [N, topk] int32 and scores [N, topk] fp32. */
int topk_ffn_fwd_indices(const void* x, const void* W1, const void* W2, void* out, int N, int d_model,
                         int d_ff, int topk, int32_t* idx, float* score, void* stream);

/*
 * Backward pass of top-k attention (Sec. 2.2, "Improving efficiency through
 * top-k attention"): the forward pass caches, per query row, the kept key
 * indices and their scores (topk_attn_fwd_indices writes exactly that
 * cache), and the backward pass recomputes only the activation over them.
 * With L = sum over rows of dout_i . out_i and the kept set held fixed:
 *   a_t  = softmax over the row's kept scores,  da_t = dout_i . v_{j_t},
 *   ds_t = a_t (da_t - sum_u a_u da_u),
 *   dq_i = sum_t ds_t k_{j_t};  dk_j, dv_j = the sums of ds_t q_i and
 *   a_t dout_i over every (i, t) that kept key j of the same (b, h).
 *   q, k, v : the forward pass's inputs (device, `dtype`, layouts above).
 *   dout    : [B, H, Lq, d] device, `dtype` (the dtype of out).
 *   idx     : [B, H, Lq, topk] int32 device, the cached kept indices; an entry
 *             outside [0, Lk) (the forward pass pads with -1) is an empty slot.
 *   score   : [B, H, Lq, topk] fp32 device, the cached scores s_t = q_i . k_{j_t}.
 *   dq      : [B, H, Lq, d] fp32 device (written).
 *   dk, dv  : [B, H, Lk, d] fp32 device (written; keys no row kept get 0).
 *   d       : TOPK_BF16: 64 or 128.  TOPK_F32: 16, 32, 64 or 128.
 *   topk    : the cache's width, 1 <= topk <= 2048.  B*H*Lq*topk and B*H*Lk
 *             must stay below 2^31.
 *   Any order of the kept entries within a row gives the same result.  dk and
 *   dv add each key's terms in an order that depends on atomic ranks, so
 *   they can differ in the last bits from call to call.
 *   Scratch: topk_attn_bwd_workspace_bytes() (20 bytes per cache entry plus
 *   8 bytes per key), from the library's pool.  Errors as topk_attn_fwd.
 */
int topk_attn_bwd(const void* q, const void* k, const void* v, const void* dout, const int32_t* idx,
                  const float* score, float* dq, float* dk, float* dv, int B, int H, int Lq, int Lk, int d,
                  int topk, int dtype, void* stream);

/*
 * Backward pass of the top-k feed-forward layer (Eq. 3 with ReLU, Sec. 2.1
 * and Sec. 2.2) for the cache of topk_ffn_fwd_indices:
 *   a_t = ReLU(s_t),  ds_t = (dout_i . W2_{j_t}) if s_t > 0 else 0,
 *   dx_i = sum_t ds_t W1_{j_t};  dW1_j, dW2_j = the sums of ds_t x_i and
 *   a_t dout_i over every (i, t) that kept key j.
 *   x, W1, W2 : the forward pass's inputs (bf16 device, layouts above).
 *   dout      : [N, d_model] fp32 device (the dtype of the forward output).
 *   idx, score: [N, topk] int32 / fp32 device, the cache.
 *   dx        : [N, d_model] fp32; dW1, dW2: [d_ff, d_model] fp32 (written).
 *   d_model   : a multiple of 64, at most 2048.  1 <= topk <= d_ff.
 *   Scratch: topk_ffn_bwd_workspace_bytes() (20 bytes per cache entry, 4 more per
 *   cache entry and 256 columns of d_model, 8 per key).  Errors as topk_ffn_fwd.
 */
int topk_ffn_bwd(const void* x, const void* W1, const void* W2, const float* dout, const int32_t* idx,
                 const float* score, float* dx, float* dW1, float* dW2, int N, int d_model, int d_ff, int topk,
                 void* stream);

/*
 * Query/key norm with the position rotation: what stands between a layer's
 * q/k/v projection and its attention, in one pass.  For every token (b, t) and
 * head, with x the head's row of d elements:
 *   n = x (mean(x^2) + eps)^-1/2 w      if normalize (w = 1 where NULL), else n = x
 *   a' = a cos[p, i] - b sin[p, i], b' = b cos[p, i] + a sin[p, i]
 *                                       for pair i < rot / 2 of q and k, where
 *     (a, b) = (n[i], n[i + rot/2]), or (n[2i], n[2i+1]) if interleaved, and
 *     p = positions[axis(i)][b, t];  elements from rot on are not rotated
 *   q' is multiplied by q_scale (the temperature, footnote to Eq. 1); v is copied.
 * Pair i belongs to the first axis x with i < sections[0] + .. + sections[x]
 * (one axis for text; time, height and width for video).
 *   q, k, v  : q [B, L, Hq, d], k and v [B, L, Hkv, d], `dtype`, 16-byte aligned, with
 *              element strides {batch, token, head}, each a multiple of 4, and contiguous
 *              rows: views of one packed projection output, for instance.  Hkv need not
 *              equal Hq.  v may be NULL.
 *   q_weight, k_weight: [d], `dtype`, 16-byte aligned, or NULL.
 *   cos, sin : [table_rows, rot / 2] fp32 (NULL if rot is 0).  positions: [axes, B, L] int32, or NULL for
 *              p = t on every axis.  A position outside the tables takes the nearest row
 *              and is reported as TOPK_ERR_RANGE by topk_check().
 *   d        : a multiple of 8, at most 256.  rot: a multiple of 8, at most d (0: none).
 *   axes     : 1 to 4; their sections are >= 0 and sum to rot / 2.
 *   Hq, Hkv  : at most 65,536 each.  A launch holds 65,535 groups of q's, k's and v's heads; what makes more
 *              (in the worst case, axes of one or two pairs, 65,536 heads of over 128 elements together) is
 *              TOPK_ERR_UNSUPPORTED.
 * Sums are taken in fp32 and each result is rounded once, to nearest.
 */
typedef struct {
  const void *q, *k, *v;
  long long q_stride[3], k_stride[3], v_stride[3];
  const void *q_weight, *k_weight;
  const float *cos, *sin;
  const int32_t* positions;
  int table_rows, B, L, Hq, Hkv, d, rot, axes;
  int sections[4];
  int interleaved, normalize, dtype;
  float eps, q_scale;
} topk_qk_args;

/*
 * Forward.  q_out [B, Hq, L, d], k_out and v_out [B, Hkv, cap, d], contiguous.
 * Without cache_start (NULL) cap must equal L; with it ([B] int32, device) token t of
 * batch b is written to row cache_start[b] + t of k_out and v_out, whose other rows are
 * left alone (a key/value cache with room for cap rows); a row outside [0, cap) is not
 * written and is reported as TOPK_ERR_RANGE by topk_check().  v_out is NULL iff v is.
 */
int topk_qk_norm_rope_fwd(const topk_qk_args* args, void* q_out, void* k_out, void* v_out, int cap,
                          const int32_t* cache_start, void* stream);

/*
 * Backward, from the gradients of the forward pass's outputs (cap = L).  With R the
 * rotation: g = R^T dout (times q_scale for q), dw = sum over tokens and heads of g x r,
 * u = g w, dx = r u - x r^3 mean(u x), where r = (mean(x^2) + eps)^-1/2.
 *   args       : the forward pass's q, k, weights, tables and positions (args->v is not read).
 *   dq, dk, dv : contiguous [B, Hq, L, d], [B, Hkv, L, d] (x 2); grad_dtype TOPK_F32, or
 *                TOPK_BF16 where `dtype` is TOPK_BF16.  dv may be NULL.
 *   dqkv       : [B, L, Hq + 2 Hkv (Hq + Hkv without dv), d] of `dtype`: q's heads, k's, v's.
 *   dq_weight, dk_weight: [d] fp32 or NULL; written only if normalize.  Blocks add up in a
 *                fixed order: two runs give the same bits.
 *   Scratch: topk_qk_norm_rope_bwd_workspace_bytes(), at most d floats for each of eight blocks per
 *   SM and for each head, from the library's pool.
 */
int topk_qk_norm_rope_bwd(const topk_qk_args* args, const void* dq, const void* dk, const void* dv, int grad_dtype,
                          void* dqkv, float* dq_weight, float* dk_weight, void* stream);
size_t topk_qk_norm_rope_bwd_workspace_bytes(int B, int L, int Hq, int Hkv, int d);

/*
 * The linear layer with its epilogue: z = x w^T + bias, y = act(z) + residual.
 *   x        : [M, K].  w: [N, K] (row n: the weights of output n).  bias: [N] or NULL.
 *   residual : [M, N] or NULL.  y: [M, N].  preact: NULL, or [M, N], which receives z for
 *              the backward pass.  All bf16, contiguous, 16-byte aligned; y and preact overlap no
 *              input, but y may be the residual itself.
 *   act      : TOPK_ACT_*; GELU is z Phi(z) (the erf form), SILU z / (1 + e^-z).  Phi is within 6e-7;
 *              its relative error passes half a bf16 place (3.7e-3) below z = -6, where |y| < 1e-8.
 *   M >= 1; N and K multiples of 8.  Sums in fp32, every result rounded once, to nearest.
 *   Scratch: topk_linear_workspace_bytes(): 0, or fp32 partial sums (parts x M x N) where the
 *   outputs are too few tiles for the SMs and the sum is split; parts are added in order, so
 *   two runs give the same bits.  Errors as topk_attn_fwd.
 */
enum { TOPK_ACT_NONE = 0, TOPK_ACT_RELU = 1, TOPK_ACT_GELU = 2, TOPK_ACT_SILU = 3 };

int topk_linear_fwd(const void* x, const void* w, const void* bias, const void* residual, void* y, void* preact, int M,
                    int N, int K, int act, void* stream);
size_t topk_linear_workspace_bytes(int M, int N, int K);

/*
 * Backward: dz = dy act'(z) (ReLU's slope at 0 is 0), dx = dz w, dw = dz^T x, db = the column sums
 * of dz.  The residual's gradient is dy itself.
 *   dy, preact : [M, N] bf16; preact is z (NULL iff act is TOPK_ACT_NONE).
 *   dx         : [M, K] bf16 or NULL.  dw: [N, K], db: [N], of grad_dtype (TOPK_F32 or TOPK_BF16), or
 *                NULL; at least one of the three is asked for.
 *   Sums are fp32; with an activation dz is rounded to bf16 before the two products (the
 *   tensor cores' operand), not before db.  A dw of TOPK_F32 has that rounding's error too
 *   (1.7e-3 in the 2-norm; none for ReLU, whose dz is dy or 0).
 *   Scratch: topk_linear_bwd_workspace_bytes(): dz, the partial sums of db and of split products.
 */
int topk_linear_bwd(const void* dy, const void* x, const void* w, const void* preact, void* dx, void* dw, void* db, int M,
                    int N, int K, int act, int grad_dtype, void* stream);
size_t topk_linear_bwd_workspace_bytes(int M, int N, int K, int act);

/*
 * One AdamW step over many tensors, in place:
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2  (g: the gradient x *grad_scale)
 *   p = p (1 - lr wd) - lr / (1 - beta1^step)  m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * in fp32, each operation rounded by itself in the order written (lr / (..) last); with 8-bit
 * states the quotient is an approximation (2^-22) and the last difference fused.
 *   tensors    : `count` descriptions in HOST memory, read before the call returns.  Tensors may
 *                be of any length (0 is skipped) and alignment; 16-byte aligned ones (8-byte
 *                for 8-bit states) take vector accesses.  No two may overlap.
 *   param_dtype, grad_dtype: TOPK_F32 or TOPK_BF16, of all tensors.
 *   state_bits : 32: m and v fp32 [n].  8: m and v hold e4m3 floats [n], with one fp32 scale for
 *                every 256 elements in m_scale, v_scale [ceil(n / 256)] (value = float x scale,
 *                scale = largest magnitude / 448; a block whose scale is below 2^-100 is zero); v
 *                holds the ROOT of the second moment.  They are rounded stochastically; the
 *                update uses the values before rounding.  A root above zero is held as the
 *                smallest float (2^-9) at least: cut to zero, it would leave the m beside it, which
 *                may be rounded up to a whole float, without a denominator in the next step.
 *   master     : NULL, or (TOPK_BF16 parameters, all tensors or none) fp32 [n] that the step
 *                reads and updates; param is then its copy, rounded to nearest.  bf16
 *                parameters without a master are rounded stochastically.
 *   seed       : of the random bits, which are a hash of (seed, step, index + element): a
 *                repeated step gives the same bits.  `index` numbers the tensor's first element
 *                among all of the optimizer's.
 *   step       : 1 for the first step.  0 <= beta < 1, eps >= 0; lr, wd finite.
 *   grad_scale : NULL, or a device float that multiplies the gradients (loss unscaling,
 *                clipping); if it is not finite the step changes nothing, and is not to be
 *                counted in `step` of the next one.
 * A non-finite gradient spoils its element, and with 8-bit states its block's moments.
 * One launch for every 352 tensors; no scratch.  Errors as topk_attn_fwd.
 */
typedef struct {
  void* param;
  const void* grad;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  long long n, index;
  double lr, weight_decay;
} topk_adamw_tensor;

int topk_adamw_step(const topk_adamw_tensor* tensors, int count, int param_dtype, int grad_dtype, int state_bits,
                    double beta1, double beta2, double eps, long long step, const float* grad_scale, uint32_t seed,
                    void* stream);

/* Scratch bytes of the two backward calls for these arguments; 0 if invalid or unsupported. */
size_t topk_attn_bwd_workspace_bytes(int B, int H, int Lq, int Lk, int d, int topk, int dtype);
size_t topk_ffn_bwd_workspace_bytes(int N, int d_model, int d_ff, int topk);

/*
 * topk_ffn_fwd without any device allocation.  The paper has no counterpart:
 * this entry exists for callers that cannot allocate device memory when they
 * call -- for instance a host runtime that hands out all device memory from
 * its own arena and allows no other allocation, or a latency-bound serving
 * loop that must never wait on an allocator or fail on a fragmented pool.
 * Instead of taking scratch from the stream-ordered pool it uses one buffer
 * of TOPK_FFN_NOALLOC_SCRATCH_BYTES that is part of the library: every GPU
 * that loads libtopk.so holds it until the process exits.
 *   - Arguments, layouts and results are those of topk_ffn_fwd; the caller
 *     still passes (and owns) x, W1, W2 and out.
 *   - Returns TOPK_ERR_SCRATCH_LIMIT, before launching anything, when
 *     topk_ffn_workspace_bytes() of the arguments exceeds the buffer.
 *   - The first call on a device looks up the buffer's device address (one
 *     runtime query, no allocation); make that first call before any stream
 *     capture on that device.
 *   - All calls on a device share the one buffer, and each call re-clears
 *     the parts that must start at zero.  Calls whose work overlaps on the
 *     GPU (other streams, or other threads) race on the buffer: serialise
 *     them, e.g. by issuing them on one stream.
 * It calls no cudaMalloc, cudaFree or other allocating routine.
 */
#define TOPK_FFN_NOALLOC_SCRATCH_BYTES (32u << 20)
int topk_ffn_fwd_noalloc(const void* x, const void* W1, const void* W2, void* out, int N, int d_model,
                         int d_ff, int topk, void* stream);

/* Bytes of stream-ordered scratch the calls above take for these arguments
 * (0 if none).  Returns 0 as well when the arguments are invalid.
 *   - attention: the bf16 tensor-core kernel with split selection parks each
 *     work unit's kept keys for its epilogue warps: per CTA (one per SM, at
 *     most one per 128-query tile) 4 x 2 x topk x 32 keys of 8 bytes plus
 *     256 counts of 4 bytes, whatever Lq and Lk are.  Sized for the current
 *     device, or for 152 SMs (a GB300) when no device is visible.
 *   - feed-forward: linear in N (see topk_ffn_fwd). */
size_t topk_attn_workspace_bytes(int B, int H, int Lq, int Lk, int d, int topk, int chunk, int dtype);
size_t topk_ffn_workspace_bytes(int N, int d_model, int d_ff, int topk);

/*
 * End-to-end variants taking HOST pointers (pinned memory is fastest).  They
 * stage the inputs into device memory from the library's pool, run the call
 * above on `stream`, copy the result back and synchronise `stream` before
 * returning.  Sizes and dtypes as above.
 *   - topk_attn_fwd_host splits the B*H heads into up to 8 consecutive
 *     slices when there are enough query tiles (about 6 per SM per slice)
 *     and launches one call per slice, alternating between two compute
 *     streams of the library (ordered after `stream`); each slice's inputs
 *     are copied on a copy stream of the library and its output copied back
 *     on another.  The copies of neighbouring slices overlap the kernels,
 *     and a slice's kernel starts on the SMs the previous slice's last wave
 *     leaves idle.  The result is identical to one call over all heads.
 *   - topk_ffn_fwd_host copies x and W1 first and W2 on a copy stream while
 *     the score and selection kernels run; the W2 gather waits for it.
 *   The library's streams are shared by all host-buffer calls on a device;
 *   `stream` is synchronised, after it has waited for all of them.
 */
int topk_attn_fwd_host(const void* q, const void* k, const void* v, void* out, int B, int H, int Lq,
                       int Lk, int d, int topk, int chunk, int causal, int dtype, void* stream);
int topk_ffn_fwd_host(const void* x, const void* W1, const void* W2, void* out, int N, int d_model,
                      int d_ff, int topk, void* stream);

/* Synchronises `stream` and returns the device-side error recorded since the
 * last check (TOPK_ERR_TIMEOUT before TOPK_ERR_WORKSPACE), clearing it;
 * TOPK_ERR_CUDA if the stream itself reports an error; else TOPK_OK.
 * The error word is ONE per device, shared by every stream and host thread
 * that calls into the library on that device: an error raised by work on one
 * stream is reported to (and cleared by) whichever caller checks first, and
 * the *_host calls check it too.  Callers that share a device and need to
 * tell their errors apart must serialise their calls and checks. */
int topk_check(void* stream);

/* Human-readable text for a return code (static storage). */
const char* topk_error_string(int code);

/* Number of kernel launches the last successful call on this host thread
 * enqueued (for launch accounting in benchmarks). */
int topk_last_launch_count(void);

/* Testing hook: sets the device-side wait limit in microseconds for later
 * calls (0 restores the default of 2 s) and returns the previous value. */
long long topk_set_wait_limit_us(long long us);

/* Device memory of the library's own stream-ordered pool on the current
 * device (scratch of the device-pointer calls, staging buffers of the *_host
 * calls): *used_high = the most bytes in use at once since the last reset,
 * *reserved = bytes the pool holds now (in use or kept for later calls).
 * Either pointer may be NULL; reset_high != 0 restarts the high-water mark
 * after reading it.  Returns TOPK_ERR_NO_DEVICE without a usable device. */
int topk_pool_usage(size_t* used_high, size_t* reserved, int reset_high);

/* Hands the pool's reserved but unused memory back to the device.  Memory
 * freed by enqueued work is released only once that work has completed:
 * synchronise the streams that used the library first. */
int topk_pool_trim(void);

/* Testing hook: when `on` is non-zero, later tcgen05 attention launches
 * withhold their second key tile, so that the consumers' bounded waits run
 * out and the call reports TOPK_ERR_TIMEOUT through topk_check() without
 * hanging the device.  Returns the previous setting. */
int topk_debug_skip_arrive(int on);

#ifdef __cplusplus
}
#endif

#endif /* TOPK_ATTENTION_H */
