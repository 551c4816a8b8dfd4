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
__device__ __forceinline__ void load_weight(const void* w, const Lane& l, float (&a)[4], float (&b)[4]) {
  if (w && l.on) {
    load4(static_cast<const T*>(w) + l.a, a);
    load4(static_cast<const T*>(w) + l.b, b);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = b[e] = 1.f;
  }
}

template <typename T, int G, int U>
__global__ void __launch_bounds__(kWarps * 32) qk_fwd_kernel(const __grid_constant__ QkArgs p, T* __restrict__ qo, T* __restrict__ ko,
                                                            T* __restrict__ vo, int cap, const int32_t* __restrict__ start,
                                                            int heads_per_item, DevCtl ctl) {
  constexpr int R = 32 / G;  // rows (heads) of a warp at a time
  const int lane = threadIdx.x & 31, j = lane % G, sub = lane / G;
  const long long token = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
  if (token >= static_cast<long long>(p.B) * p.L) return;
  const int b = static_cast<int>(token / p.L), t = static_cast<int>(token % p.L);
  const int heads = p.Hq + p.Hkv + (p.v ? p.Hkv : 0);
  const int h0 = blockIdx.y * heads_per_item, h1 = min(h0 + heads_per_item, heads);
  const Lane l = lane_of(p, j);
  float c[4], s[4], wqa[4], wqb[4], wka[4], wkb[4];
  load_angles(p, l, j, b, t, ctl, c, s);
  load_weight<T>(p.q_weight, l, wqa, wqb);
  load_weight<T>(p.k_weight, l, wka, wkb);
  // the token's row of the key and value caches
  long long row = t;
  if (start) {
    row += __ldg(start + b);
    if (row < 0 || row >= cap) {
      if (lane == 0) atomicOr(ctl.error, kDevErrRange);
      row = -1;
    }
  }
  const float inv_d = 1.f / p.d;
  for (int hb = h0; hb < h1; hb += R * U) {
    float xa[U][4], xb[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * R + sub;
      const T* src;
      if (h < p.Hq)
        src = static_cast<const T*>(p.q) + b * p.q_stride[0] + t * p.q_stride[1] + h * p.q_stride[2];
      else if (h < p.Hq + p.Hkv)
        src = static_cast<const T*>(p.k) + b * p.k_stride[0] + t * p.k_stride[1] + (h - p.Hq) * p.k_stride[2];
      else
        src = static_cast<const T*>(p.v) + b * p.v_stride[0] + t * p.v_stride[1] + (h - p.Hq - p.Hkv) * p.v_stride[2];
      if (h < h1 && l.on) {
        load4(src + l.a, xa[u]);
        load4(src + l.b, xb[u]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) xa[u][e] = xb[u][e] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int h = hb + u * R + sub;
      const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
      float ss = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) ss += xa[u][e] * xa[u][e] + xb[u][e] * xb[u][e];
      ss = group_sum<G>(ss);
      if (!is_v) {
        const float r = p.normalize ? rsqrtf(ss * inv_d + p.eps) : 1.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          xa[u][e] = xa[u][e] * r * (is_q ? wqa[e] : wka[e]);
          xb[u][e] = xb[u][e] * r * (is_q ? wqb[e] : wkb[e]);
        }
        rotate(xa[u], xb[u], c, s, p.interleaved);
        if (is_q) {
#pragma unroll
          for (int e = 0; e < 4; ++e) xa[u][e] *= p.q_scale, xb[u][e] *= p.q_scale;
        }
      }
      if (h >= h1 || !l.on) continue;
      T* dst;
      if (is_q)
        dst = qo + ((static_cast<size_t>(b) * p.Hq + h) * p.L + t) * p.d;
      else if (row < 0)
        continue;
      else if (!is_v)
        dst = ko + ((static_cast<size_t>(b) * p.Hkv + (h - p.Hq)) * cap + row) * p.d;
      else
        dst = vo + ((static_cast<size_t>(b) * p.Hkv + (h - p.Hq - p.Hkv)) * cap + row) * p.d;
      store4(dst + l.a, xa[u]);
      store4(dst + l.b, xb[u]);
    }
  }
}

// Backward.  Blocks take tokens in strides of the grid and keep the sums of
// both weight gradients in registers (eight elements of q's and of k's per
// lane); each block adds its lanes up in a fixed order and writes one partial
// row, and qk_bwd_weights_kernel adds the partial rows, so that the result does
// not depend on the order in which blocks run.
template <typename T, typename GT, int G, int U>
__global__ void __launch_bounds__(kWarps * 32) qk_bwd_kernel(const __grid_constant__ QkArgs p, const GT* __restrict__ dq,
                                                            const GT* __restrict__ dk, const GT* __restrict__ dv,
                                                            T* __restrict__ dqkv, float* __restrict__ partial, DevCtl ctl) {
  constexpr int R = 32 / G;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane % G, sub = lane / G;
  const int heads = p.Hq + p.Hkv + (dv ? p.Hkv : 0);
  const long long tokens = static_cast<long long>(p.B) * p.L;
  const Lane l = lane_of(p, j);
  float wqa[4], wqb[4], wka[4], wkb[4];
  load_weight<T>(p.q_weight, l, wqa, wqb);
  load_weight<T>(p.k_weight, l, wka, wkb);
  float gqa[4] = {}, gqb[4] = {}, gka[4] = {}, gkb[4] = {};
  const float inv_d = 1.f / p.d;
  for (long long token = static_cast<long long>(blockIdx.x) * kWarps + warp; token < tokens;
       token += static_cast<long long>(gridDim.x) * kWarps) {
    const int b = static_cast<int>(token / p.L), t = static_cast<int>(token % p.L);
    float c[4], s[4];
    load_angles(p, l, j, b, t, ctl, c, s);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] = -s[e];  // the transpose turns the other way
    for (int hb = 0; hb < heads; hb += R * U) {
      float ga[U][4], gb[U][4], xa[U][4], xb[U][4];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = hb + u * R + sub;
        const GT* gs;
        const T* xs = nullptr;
        if (h < p.Hq) {
          gs = dq + ((static_cast<size_t>(b) * p.Hq + h) * p.L + t) * p.d;
          xs = static_cast<const T*>(p.q) + b * p.q_stride[0] + t * p.q_stride[1] + h * p.q_stride[2];
        } else if (h < p.Hq + p.Hkv) {
          gs = dk + ((static_cast<size_t>(b) * p.Hkv + (h - p.Hq)) * p.L + t) * p.d;
          xs = static_cast<const T*>(p.k) + b * p.k_stride[0] + t * p.k_stride[1] + (h - p.Hq) * p.k_stride[2];
        } else {
          gs = dv + ((static_cast<size_t>(b) * p.Hkv + (h - p.Hq - p.Hkv)) * p.L + t) * p.d;
        }
        const bool on = h < heads && l.on;
#pragma unroll
        for (int e = 0; e < 4; ++e) ga[u][e] = gb[u][e] = xa[u][e] = xb[u][e] = 0.f;
        if (on) {
          load4(gs + l.a, ga[u]);
          load4(gs + l.b, gb[u]);
        }
        if (on && xs && p.normalize) {
          load4(xs + l.a, xa[u]);
          load4(xs + l.b, xb[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = hb + u * R + sub;
        const bool is_q = h < p.Hq, is_v = h >= p.Hq + p.Hkv;
        if (!is_v) {
          rotate(ga[u], gb[u], c, s, p.interleaved);
          if (is_q) {
#pragma unroll
            for (int e = 0; e < 4; ++e) ga[u][e] *= p.q_scale, gb[u][e] *= p.q_scale;
          }
        }
        if (p.normalize) {  // values have xa = xb = 0 here and keep their gradients
          float ss = 0.f, dot = 0.f, ua[4], ub[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ua[e] = ga[u][e] * (is_q ? wqa[e] : wka[e]);
            ub[e] = gb[u][e] * (is_q ? wqb[e] : wkb[e]);
            ss += xa[u][e] * xa[u][e] + xb[u][e] * xb[u][e];
            dot += ua[e] * xa[u][e] + ub[e] * xb[u][e];
          }
          ss = group_sum<G>(ss);
          dot = group_sum<G>(dot);
          const float r = rsqrtf(ss * inv_d + p.eps), k3 = r * r * r * dot * inv_d;
          if (!is_v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float da = ga[u][e] * xa[u][e] * r, db = gb[u][e] * xb[u][e] * r;
              gqa[e] += is_q ? da : 0.f, gqb[e] += is_q ? db : 0.f;
              gka[e] += is_q ? 0.f : da, gkb[e] += is_q ? 0.f : db;
              ga[u][e] = r * ua[e] - xa[u][e] * k3;
              gb[u][e] = r * ub[e] - xb[u][e] * k3;
            }
          }
        }
        if (h >= heads || !l.on) continue;
        T* dst = dqkv + (token * heads + h) * p.d;
        store4(dst + l.a, ga[u]);
        store4(dst + l.b, gb[u]);
      }
    }
  }
  if (!partial) return;
  // lanes of one j, then warps, in a fixed order
  __shared__ float sums[kWarps][2][G][8];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
#pragma unroll
    for (int o = G; o < 32; o <<= 1) {
      gqa[e] += __shfl_xor_sync(kFull, gqa[e], o);
      gqb[e] += __shfl_xor_sync(kFull, gqb[e], o);
      gka[e] += __shfl_xor_sync(kFull, gka[e], o);
      gkb[e] += __shfl_xor_sync(kFull, gkb[e], o);
    }
    if (sub == 0) {
      sums[warp][0][j][e] = gqa[e], sums[warp][0][j][e + 4] = gqb[e];
      sums[warp][1][j][e] = gka[e], sums[warp][1][j][e + 4] = gkb[e];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * G * 8; i += kWarps * 32) {
    const int which = i / (G * 8), jj = (i / 8) % G, e = i % 8;
    const Lane o = lane_of(p, jj);
    if (!o.on) continue;
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) a += sums[w][which][jj][e];
    partial[(static_cast<size_t>(blockIdx.x) * 2 + which) * p.d + (e < 4 ? o.a + e : o.b + e - 4)] = a;
  }
}

// dw[c] = sum of the blocks' partial rows; one block of 32 x 8 threads takes 32 columns.
__global__ void qk_bwd_weights_kernel(const float* __restrict__ partial, int blocks, int d, float* __restrict__ dqw,
                                      float* __restrict__ dkw) {
  __shared__ float sums[8][33];
  const int i = blockIdx.x * 32 + threadIdx.x;
  float a = 0.f;
  if (i < 2 * d)
    for (int b = threadIdx.y; b < blocks; b += 8) a += partial[static_cast<size_t>(b) * 2 * d + i];
  sums[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y == 0 && i < 2 * d) {
    for (int y = 1; y < 8; ++y) a += sums[y][threadIdx.x];
    float* out = i < d ? dqw : dkw;
    if (out) out[i < d ? i : i - d] = a;
  }
}

constexpr int kBwdBlocksPerSm = 2;

template <typename T, int G>
int launch_fwd(const QkArgs& p, void* qo, void* ko, void* vo, int cap, const int32_t* start, int num_sms, const DevCtl& ctl,
               cudaStream_t st) {
  const long long tokens = static_cast<long long>(p.B) * p.L;
  const int heads = p.Hq + p.Hkv + (p.v ? p.Hkv : 0);
  constexpr int R = 32 / G;
  const long long blocks = (tokens + kWarps - 1) / kWarps;
  // few tokens: their heads are shared out until every SM has some
  int per = heads;
  while (per > R && blocks * ((heads + per - 1) / per) < 2LL * num_sms) per = (per + 1) / 2;
  per = (per + R - 1) / R * R;
  const dim3 grid(static_cast<unsigned>(blocks), (heads + per - 1) / per);
  qk_fwd_kernel<T, G, 2><<<grid, kWarps * 32, 0, st>>>(p, static_cast<T*>(qo), static_cast<T*>(ko), static_cast<T*>(vo), cap,
                                                       start, per, ctl);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

template <typename T, typename GT, int G>
int launch_bwd(const QkArgs& p, const void* dq, const void* dk, const void* dv, void* dqkv, float* dqw, float* dkw,
               float* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  const int blocks = qk_bwd_blocks(p.B, p.L, num_sms);
  const bool weights = p.normalize && (dqw || dkw);
  qk_bwd_kernel<T, GT, G, 2><<<blocks, kWarps * 32, 0, st>>>(p, static_cast<const GT*>(dq), static_cast<const GT*>(dk),
                                                             static_cast<const GT*>(dv), static_cast<T*>(dqkv),
                                                             weights ? workspace : nullptr, ctl);
  if (cudaGetLastError() != cudaSuccess) return -1;
  if (!weights) return 1;
  qk_bwd_weights_kernel<<<(2 * p.d + 31) / 32, dim3(32, 8), 0, st>>>(workspace, blocks, p.d, dqw, dkw);
  return cudaGetLastError() == cudaSuccess ? 2 : -1;
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

int qk_bwd_blocks(int B, int L, int num_sms) {
  const long long want = (static_cast<long long>(B) * L + kWarps - 1) / kWarps, most = static_cast<long long>(num_sms) * kBwdBlocksPerSm;
  return static_cast<int>(want < most ? want : most);
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
