// norm_rope.cu -- the step between a layer's q/k/v projection and its
// attention, in one pass: RMS norm of every query and key head, the rotary
// position rotation, the temperature folded into q (footnote to Eq. 1), and
// the change from the projection's token-major rows [B, L, heads, d] to the
// head-major [B, H, L, d] that attention reads.  Values are copied along.
//
//   r = (mean_c x_c^2 + eps)^-1/2,  n = x r w                  (one head's row)
//   a' = a cos - b sin,  b' = b cos + a sin                    (pair i < rot / 2)
// with cos/sin from row pos[axis(i)][b, t] of fp32 tables; pair i is
// (n_i, n_{i + rot/2}), or (n_2i, n_2i+1) when interleaved.  Backward, from the
// gradient of the outputs (R orthogonal, so its transpose undoes it):
//   g = R^T dout,  dw += g x r,  u = g w,  dx = r u - x r^3 mean(u x).
//
// Every element is read once and written once and costs a few FMAs: the kernels
// are bound by HBM, so they are laid out for coalesced 128-byte rows and loads
// in flight.  G = d / 8 lanes (rounded up to a power of two) own a row, eight
// elements each, chosen so that both members of a pair sit in one lane: the
// rotation needs no exchange, and the norm one butterfly over the G lanes.  A
// warp takes one token and walks over its heads, so the token's cos and sin are
// loaded once into registers and serve every head; the warps of a block take
// neighbouring tokens, whose rows of a head are neighbours in the output.
#include <cuda_bf16.h>

#include "kernels.h"

namespace topk {

namespace {

constexpr int kWarps = 8;        // tokens per block
constexpr unsigned kFull = 0xffffffffu;
constexpr int kBwdBlocksPerSm = 3;

__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
  const float4 f = *reinterpret_cast<const float4*>(p);
  v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
}

__device__ __forceinline__ void load4(const __nv_bfloat16* p, float (&v)[4]) {
  const uint2 u = *reinterpret_cast<const uint2*>(p);
  v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
  v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
}

__device__ __forceinline__ void store4(float* p, const float (&v)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}

// the one rounding of a result to bf16, to nearest
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float (&v)[4]) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}

template <int G>
__device__ __forceinline__ float group_sum(float s) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) s += __shfl_xor_sync(kFull, s, o);
  return s;
}

// What a lane owns of every row: elements [a, a + 4) and [b, b + 4).  In the
// half layout the two are partners; elsewhere (interleaved pairs, the
// unrotated tail) they are neighbours.
struct Lane {
  int a, b;
  bool on, rotated;
};

__device__ __forceinline__ Lane lane_of(const QkArgs& p, int j) {
  Lane l;
  l.on = 8 * j < p.d;
  l.rotated = 8 * j < p.rot;
  const bool half = l.rotated && !p.interleaved;
  l.a = half ? 4 * j : 8 * j;
  l.b = half ? p.rot / 2 + 4 * j : 8 * j + 4;
  return l;
}

// cos and sin of the lane's four pairs 4j .. 4j + 3 for token (b, t); identity
// where the lane does not rotate.  A position outside the tables is reported
// and clamped.
__device__ __forceinline__ void load_angles(const QkArgs& p, const Lane& l, int j, int b, int t, const DevCtl& ctl,
                                            float (&c)[4], float (&s)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = 1.f, s[e] = 0.f;
  if (!l.rotated) return;
  const int half = p.rot / 2;
  int row[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    int axis = 0;
    for (int x = 0; x + 1 < p.axes; ++x) axis += 4 * j + e >= p.bound[x];
    int pos = p.positions ? __ldg(p.positions + (static_cast<size_t>(axis) * p.B + b) * p.L + t) : t;
    if (pos < 0 || pos >= p.table_rows) {
      atomicOr(ctl.error, kDevErrRange);
      pos = pos < 0 ? 0 : p.table_rows - 1;
    }
    row[e] = pos;
  }
  if (row[0] == row[3] && row[0] == row[1] && row[0] == row[2]) {
    load4(p.cos + static_cast<size_t>(row[0]) * half + 4 * j, c);
    load4(p.sin + static_cast<size_t>(row[0]) * half + 4 * j, s);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      c[e] = __ldg(p.cos + static_cast<size_t>(row[e]) * half + 4 * j + e);
      s[e] = __ldg(p.sin + static_cast<size_t>(row[e]) * half + 4 * j + e);
    }
  }
}

// Rotates the lane's eight values by (c, s) in place.
__device__ __forceinline__ void rotate(float (&a)[4], float (&b)[4], const float (&c)[4], const float (&s)[4],
                                       bool interleaved) {
  if (!interleaved) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = a[e], y = b[e];
      a[e] = x * c[e] - y * s[e];
      b[e] = y * c[e] + x * s[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float x = a[2 * e], y = a[2 * e + 1];
      a[2 * e] = x * c[e] - y * s[e];
      a[2 * e + 1] = y * c[e] + x * s[e];
      x = b[2 * e], y = b[2 * e + 1];
      b[2 * e] = x * c[e + 2] - y * s[e + 2];
      b[2 * e + 1] = y * c[e + 2] + x * s[e + 2];
    }
  }
}

template <typename T>
__device__ __forceinline__ void load_weight(const T* w, const Lane& l, float (&a)[4], float (&b)[4]) {
  if (w && l.on) {
    load4(w + l.a, a);
    load4(w + l.b, b);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = b[e] = 1.f;
  }
}

// A warp's share of a token: `rows` heads of one kind (q, k or v), U x R at most.
// The groups of a token are q's, then k's, then v's.
enum Kind { kQ, kK, kV };

struct Group {
  int kind, h0, rows;
};

__device__ __forceinline__ Group group_of(const QkArgs& p, int g, int size) {
  const int nq = (p.Hq + size - 1) / size, nk = (p.Hkv + size - 1) / size;
  Group o;
  o.kind = g < nq ? kQ : (g < nq + nk ? kK : kV);
  const int i = g - (o.kind == kQ ? 0 : (o.kind == kK ? nq : nq + nk));
  const int heads = o.kind == kQ ? p.Hq : p.Hkv;
  o.h0 = i * size;
  o.rows = min(size, heads - o.h0);
  return o;
}

// Loads as they lie in memory: a lane holds a row in four registers (bf16), and the loads of
// all its rows go out before the first is used.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  float4 u;
  __device__ __forceinline__ void load(const float* p) { u = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void zero() { u = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w; }
};
template <>
struct Raw<__nv_bfloat16> {
  uint2 u;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { u = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void zero() { u = make_uint2(0u, 0u); }
  __device__ __forceinline__ void get(float (&v)[4]) const {
    v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xffff0000u);
  }
};

template <typename T, int G, int U>
__global__ void __launch_bounds__(kWarps * 32, 4) qk_fwd_kernel(const __grid_constant__ QkArgs p, T* __restrict__ qo, T* __restrict__ ko,
                                                               T* __restrict__ vo, int cap, const int32_t* __restrict__ start, DevCtl ctl) {
  constexpr int R = 32 / G;  // rows (heads) of a warp at a time
  const int lane = threadIdx.x & 31, j = lane % G, sub = lane / G;
  const long long token = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (token >= static_cast<long long>(p.B) * p.L) return;
  const int b = static_cast<int>(token / p.L), t = static_cast<int>(token % p.L);
  const Group g = group_of(p, blockIdx.y, R * U);
  const Lane l = lane_of(p, j);
  const void* in = g.kind == kQ ? p.q : (g.kind == kK ? p.k : p.v);
  const long long* stride = g.kind == kQ ? p.q_stride : (g.kind == kK ? p.k_stride : p.v_stride);
  const T* src = static_cast<const T*>(in) + b * stride[0] + t * stride[1] + (g.h0 + sub) * stride[2];
  const long long step = R * stride[2];
  Raw<T> ra[U], rb[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (u * R + sub < g.rows && l.on) {
      ra[u].load(src + u * step + l.a);
      rb[u].load(src + u * step + l.b);
    } else {
      ra[u].zero();
      rb[u].zero();
    }
  }
  // the output row of the group's first head
  const int heads = g.kind == kQ ? p.Hq : p.Hkv, rows = g.kind == kQ ? p.L : cap;
  long long row = t;
  if (start && g.kind != kQ) {
    row += __ldg(start + b);
    if (row < 0 || row >= cap) {
      if (lane == 0) atomicOr(ctl.error, kDevErrRange);
      return;
    }
  }
  T* dst = (g.kind == kQ ? qo : (g.kind == kK ? ko : vo)) + ((static_cast<long long>(b) * heads + g.h0 + sub) * rows + row) * p.d;
  const long long out_step = static_cast<long long>(R) * rows * p.d;
  if (g.kind == kV) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * R + sub >= g.rows || !l.on) continue;
      *reinterpret_cast<Raw<T>*>(dst + u * out_step + l.a) = ra[u];
      *reinterpret_cast<Raw<T>*>(dst + u * out_step + l.b) = rb[u];
    }
    return;
  }
  float c[4], s[4], wa[4], wb[4];
  load_angles(p, l, j, b, t, ctl, c, s);
  load_weight(static_cast<const T*>(g.kind == kQ ? p.q_weight : p.k_weight), l, wa, wb);
  const float scale = g.kind == kQ ? p.q_scale : 1.f, inv_d = 1.f / p.d;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float xa[4], xb[4];
    ra[u].get(xa);
    rb[u].get(xb);
    if (p.normalize) {
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) ss += xa[e] * xa[e] + xb[e] * xb[e];
      const float r = rsqrtf(group_sum<G>(ss) * inv_d + p.eps);
#pragma unroll
      for (int e = 0; e < 4; ++e) xa[e] = xa[e] * r * wa[e], xb[e] = xb[e] * r * wb[e];
    }
    rotate(xa, xb, c, s, p.interleaved);
#pragma unroll
    for (int e = 0; e < 4; ++e) xa[e] *= scale, xb[e] *= scale;
    if (u * R + sub >= g.rows || !l.on) continue;
    store4(dst + u * out_step + l.a, xa);
    store4(dst + u * out_step + l.b, xb);
  }
}

// Backward.  A block keeps one group of heads and walks over tokens in strides of the grid, so
// that its lanes sum their eight elements' weight gradient in registers; at the end the
// block adds its lanes up in a fixed order and writes one partial row.
// qk_bwd_weights_kernel adds the partial rows: the result does not depend on the order in
// which blocks run.
template <typename T, typename GT, int G, int U>
__global__ void __launch_bounds__(kWarps * 32, kBwdBlocksPerSm)
    qk_bwd_kernel(const __grid_constant__ QkArgs p, const GT* __restrict__ dq, const GT* __restrict__ dk, const GT* __restrict__ dv,
                  T* __restrict__ dqkv, float* __restrict__ partial, DevCtl ctl) {
  constexpr int R = 32 / G;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane % G, sub = lane / G;
  const int all = p.Hq + (dv ? 2 : 1) * p.Hkv;
  const long long tokens = static_cast<long long>(p.B) * p.L;
  const Lane l = lane_of(p, j);
  const Group g = group_of(p, blockIdx.y, R * U);
  const int heads = g.kind == kQ ? p.Hq : p.Hkv;
  const GT* grad = g.kind == kQ ? dq : (g.kind == kK ? dk : dv);
  const T* in = static_cast<const T*>(g.kind == kQ ? p.q : p.k);
  const long long* stride = g.kind == kQ ? p.q_stride : p.k_stride;
  const bool norm = p.normalize && g.kind != kV;
  float wa[4], wb[4], ga[4] = {}, gb[4] = {};
  load_weight(static_cast<const T*>(g.kind == kQ ? p.q_weight : p.k_weight), l, wa, wb);
  const float scale = g.kind == kQ ? p.q_scale : 1.f, inv_d = 1.f / p.d;
  for (long long token = static_cast<long long>(blockIdx.x) * kWarps + warp; token < tokens;
       token += static_cast<long long>(gridDim.x) * kWarps) {
    const int b = static_cast<int>(token / p.L), t = static_cast<int>(token % p.L);
    const GT* gs = grad + ((static_cast<long long>(b) * heads + g.h0 + sub) * p.L + t) * p.d;
    const long long gstep = static_cast<long long>(R) * p.L * p.d;
    const T* xs = in + b * stride[0] + t * stride[1] + (g.h0 + sub) * stride[2];
    Raw<GT> qa[U], qb[U];
    Raw<T> ra[U], rb[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = u * R + sub < g.rows && l.on;
      if (on) {
        qa[u].load(gs + u * gstep + l.a);
        qb[u].load(gs + u * gstep + l.b);
      } else {
        qa[u].zero();
        qb[u].zero();
      }
      if (on && norm) {
        ra[u].load(xs + u * R * stride[2] + l.a);
        rb[u].load(xs + u * R * stride[2] + l.b);
      } else {
        ra[u].zero();
        rb[u].zero();
      }
    }
    T* dst = dqkv + (token * all + (g.kind == kQ ? 0 : (g.kind == kK ? p.Hq : p.Hq + p.Hkv)) + g.h0 + sub) * p.d;
    float c[4], s[4];
    if (g.kind != kV) load_angles(p, l, j, b, t, ctl, c, s);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float ya[4], yb[4];
      qa[u].get(ya);
      qb[u].get(yb);
      if (g.kind != kV) {
#pragma unroll
        for (int e = 0; e < 4; ++e) ya[e] *= scale, yb[e] *= scale;
        const float back[4] = {-s[0], -s[1], -s[2], -s[3]};  // the transpose turns the other way
        rotate(ya, yb, c, back, p.interleaved);
      }
      if (norm) {
        float xa[4], xb[4], ss = 0.f, dot = 0.f;
        ra[u].get(xa);
        rb[u].get(xb);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ss += xa[e] * xa[e] + xb[e] * xb[e];
          dot += ya[e] * wa[e] * xa[e] + yb[e] * wb[e] * xb[e];
        }
        const float r = rsqrtf(group_sum<G>(ss) * inv_d + p.eps), k3 = r * r * r * group_sum<G>(dot) * inv_d;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          ga[e] += ya[e] * xa[e] * r;
          gb[e] += yb[e] * xb[e] * r;
          ya[e] = r * (ya[e] * wa[e]) - xa[e] * k3;
          yb[e] = r * (yb[e] * wb[e]) - xb[e] * k3;
        }
      }
      if (u * R + sub >= g.rows || !l.on) continue;
      store4(dst + u * R * p.d + l.a, ya);
      store4(dst + u * R * p.d + l.b, yb);
    }
  }
  if (!partial || g.kind == kV) return;
  // lanes of one j, then warps, in a fixed order
  __shared__ float sums[kWarps][G][8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int o = G; o < 32; o <<= 1) {
      ga[e] += __shfl_xor_sync(kFull, ga[e], o);
      gb[e] += __shfl_xor_sync(kFull, gb[e], o);
    }
    if (sub == 0) sums[warp][j][e] = ga[e], sums[warp][j][e + 4] = gb[e];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < G * 8; i += kWarps * 32) {
    const int jj = i / 8, e = i % 8;
    const Lane o = lane_of(p, jj);
    if (!o.on) continue;
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) a += sums[w][jj][e];
    partial[(static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x) * p.d + (e < 4 ? o.a + e : o.b + e - 4)] = a;
  }
}

// dw[c] = sum of the partial rows of q's groups (blockIdx.y 0) or k's, in order: 32 columns a block,
// 32 threads each.
__global__ void __launch_bounds__(1024) qk_bwd_weights_kernel(const float* __restrict__ partial, int q_rows, int k_rows, int d,
                                                              float* __restrict__ dqw, float* __restrict__ dkw) {
  __shared__ float sums[32][33];
  const int c = blockIdx.x * 32 + threadIdx.x;
  const int first = blockIdx.y ? q_rows : 0, end = blockIdx.y ? q_rows + k_rows : q_rows;
  float a = 0.f;
  if (c < d) {
#pragma unroll 4
    for (int r = first + threadIdx.y; r < end; r += 32) a += partial[static_cast<size_t>(r) * d + c];
  }
  sums[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y == 0 && c < d) {
    for (int y = 1; y < 32; ++y) a += sums[y][threadIdx.x];
    float* out = blockIdx.y ? dkw : dqw;
    if (out) out[c] = a;
  }
}

int groups_of(int heads, int size) { return (heads + size - 1) / size; }

// Rows a lane holds at once: the fewest padded rows over q, k and v, and of those the most (more
// loads in flight, the token's angles loaded less often).
int rows_per_lane(const QkArgs& p, int R, int most) {
  int best = 1, least = 1 << 30;
  for (int u = 1; u <= most; ++u) {
    const int rows = (groups_of(p.Hq, R * u) + 2 * groups_of(p.Hkv, R * u)) * u;
    if (rows <= least) least = rows, best = u;
  }
  return best;
}

template <typename F>
int by_rows(int u, F f) {
  switch (u) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 3: return f(std::integral_constant<int, 3>());
    default: return f(std::integral_constant<int, 4>());
  }
}

template <typename T, int G>
int launch_fwd(const QkArgs& p, void* qo, void* ko, void* vo, int cap, const int32_t* start, int num_sms, const DevCtl& ctl,
               cudaStream_t st) {
  const long long tokens = static_cast<long long>(p.B) * p.L;
  constexpr int R = 32 / G;
  const long long blocks = (tokens + kWarps - 1) / kWarps;
  // few tokens: one row a lane, for more warps
  const int u = blocks < num_sms ? 1 : rows_per_lane(p, R, 4);
  return by_rows(u, [&](auto n) {
    constexpr int U = decltype(n)::value;
    const dim3 grid(static_cast<unsigned>(blocks), groups_of(p.Hq, R * U) + (p.v ? 2 : 1) * groups_of(p.Hkv, R * U));
    qk_fwd_kernel<T, G, U><<<grid, kWarps * 32, 0, st>>>(p, static_cast<T*>(qo), static_cast<T*>(ko), static_cast<T*>(vo), cap, start, ctl);
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
  });
}

// Blocks that walk over the tokens, for each group.
int bwd_blocks(int B, int L, int groups, int num_sms) {
  const long long want = (static_cast<long long>(B) * L + kWarps - 1) / kWarps;
  const long long most = (static_cast<long long>(num_sms) * kBwdBlocksPerSm + groups - 1) / groups;
  return static_cast<int>(want < most ? want : most);
}

template <typename T, typename GT, int G>
int launch_bwd(const QkArgs& p, const void* dq, const void* dk, const void* dv, void* dqkv, float* dqw, float* dkw,
               float* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  constexpr int R = 32 / G;
  const bool weights = p.normalize && (dqw || dkw);
  constexpr int kRows = sizeof(T) == 2 ? 2 : 1;  // what 80 registers hold of a row and its gradient
  return by_rows(rows_per_lane(p, R, kRows), [&](auto n) {
    constexpr int U = decltype(n)::value < kRows ? decltype(n)::value : kRows;
    const int nq = groups_of(p.Hq, R * U), nk = groups_of(p.Hkv, R * U), groups = nq + (dv ? 2 : 1) * nk;
    const int blocks = bwd_blocks(p.B, p.L, groups, num_sms);
    qk_bwd_kernel<T, GT, G, U><<<dim3(blocks, groups), kWarps * 32, 0, st>>>(p, static_cast<const GT*>(dq), static_cast<const GT*>(dk),
                                                                            static_cast<const GT*>(dv), static_cast<T*>(dqkv),
                                                                            weights ? workspace : nullptr, ctl);
    if (cudaGetLastError() != cudaSuccess) return -1;
    if (!weights) return 1;
    qk_bwd_weights_kernel<<<dim3((p.d + 31) / 32, 2), dim3(32, 32), 0, st>>>(workspace, nq * blocks, nk * blocks, p.d, dqw, dkw);
    return cudaGetLastError() == cudaSuccess ? 2 : -1;
  });
}

template <typename F>
int by_lanes(int d, F f) {
  const int lanes = (d + 7) / 8;
  if (lanes <= 2) return f(std::integral_constant<int, 2>());
  if (lanes <= 4) return f(std::integral_constant<int, 4>());
  if (lanes <= 8) return f(std::integral_constant<int, 8>());
  if (lanes <= 16) return f(std::integral_constant<int, 16>());
  return f(std::integral_constant<int, 32>());
}

}  // namespace

// Partial rows of weight gradients: at most one for each block of a full grid and one more for each
// group, or one for each eight tokens and head.
int qk_bwd_partial_rows(int B, int L, int Hq, int Hkv, int num_sms) {
  const long long heads = static_cast<long long>(Hq) + Hkv, full = static_cast<long long>(num_sms) * kBwdBlocksPerSm + heads;
  const long long few = (static_cast<long long>(B) * L + kWarps - 1) / kWarps * heads;
  return static_cast<int>(few < full ? few : full);
}

int qk_norm_rope_fwd(const QkArgs& p, void* qo, void* ko, void* vo, int cap, const int32_t* start, int num_sms, const DevCtl& ctl,
                     cudaStream_t st) {
  return by_lanes(p.d, [&](auto g) {
    constexpr int G = decltype(g)::value;
    return p.bf16 ? launch_fwd<__nv_bfloat16, G>(p, qo, ko, vo, cap, start, num_sms, ctl, st)
                  : launch_fwd<float, G>(p, qo, ko, vo, cap, start, num_sms, ctl, st);
  });
}

int qk_norm_rope_bwd(const QkArgs& p, const void* dq, const void* dk, const void* dv, bool grad_bf16, void* dqkv, float* dqw,
                     float* dkw, float* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  return by_lanes(p.d, [&](auto g) {
    constexpr int G = decltype(g)::value;
    if (!p.bf16)
      return grad_bf16 ? 0 : launch_bwd<float, float, G>(p, dq, dk, dv, dqkv, dqw, dkw, workspace, num_sms, ctl, st);
    return grad_bf16 ? launch_bwd<__nv_bfloat16, __nv_bfloat16, G>(p, dq, dk, dv, dqkv, dqw, dkw, workspace, num_sms, ctl, st)
                     : launch_bwd<__nv_bfloat16, float, G>(p, dq, dk, dv, dqkv, dqw, dkw, workspace, num_sms, ctl, st);
  });
}

}  // namespace topk
