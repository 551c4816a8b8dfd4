// adamw.cu -- one AdamW step over many tensors: decoupled weight decay, the
// moments in 32 bits or in 8.
//
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t)  m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// Every element is read once and written once and costs a few dozen
// operations: the step is bound by HBM.  The tensors' addresses travel in the
// kernel's parameters, so that a launch needs no table in device memory and up to
// kMaxTensors tensors share it; a block takes kChunk elements of one tensor, found by
// bisection over the tensors' first blocks.  A lane takes eight neighbouring
// elements and a warp 256, which is one block of the 8-bit states: its two maxima
// are one warp reduction each.
//
// 8-bit states: block of 256 elements, values = e4m3 float x the block's fp32 scale
// (largest magnitude / 448).  The second moment is held as its root: the update
// needs the root, and the root's range is half as wide in the exponent, so that e4m3's
// 2^-9 .. 448 covers 2^35 in v.  Both are rounded stochastically: with b2 = 0.999
// a step moves v by a thousandth, far below half a place of a 4-bit significand, and to
// the nearest the moments would never move.  bf16 parameters without a 32-bit master
// are rounded stochastically for the same reason; a copy beside a master, which nothing
// is added to, to the nearest.  The random bits are a hash of (seed, step, element): a step
// gives the same bits whenever it is repeated.  States and roundings depend on the last
// bit of the sums before them, so the sums use separately rounded products (no
// fused multiply-add) and a test can state them exactly.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>

#include "kernels.h"

namespace topk {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                          // neighbouring elements of a lane
constexpr int kRound = kThreads * kPer;          // elements of a block at a time
constexpr unsigned kFull = 0xffffffffu;
constexpr float kTop = 448.f;                    // largest e4m3 value

struct Entry {
  void* param;
  const void* grad;
  float* master;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  long long n, index;
  float decay, size;  // 1 - lr wd, lr / (1 - b1^t)
  int first;          // first block of the tensor
  int vec;            // every pointer allows a lane's vector accesses
};

constexpr int kMaxTensors = 352;

struct Table {
  Entry e[kMaxTensors];
  const float* grad_scale;
  float b1, c1, b2, c2, isb2, eps;  // c = 1 - b, isb2 = 1 / sqrt(1 - b2^t)
  uint32_t key;
  int n_tensors, rounds;
};
static_assert(sizeof(Table) <= 32764, "kernel parameters");

__host__ __device__ inline uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7feb352du;
  x ^= x >> 15;
  x *= 0x846ca68bu;
  return x ^ (x >> 16);
}

__device__ __forceinline__ void load8(const float* p, float (&v)[8], bool vec, int count) {
  if (vec && count == 8) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count ? p[e] : 0.f;
  }
}

__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&v)[8], bool vec, int count) {
  if (vec && count == 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(w[e] << 16), v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < count ? __bfloat162float(p[e]) : 0.f;
  }
}

__device__ __forceinline__ void store8(float* p, const float (&v)[8], bool vec, int count) {
  if (vec && count == 8) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) p[e] = v[e];
  }
}

// eight 16-bit patterns (bf16)
__device__ __forceinline__ void store8_16(__nv_bfloat16* p, const uint32_t (&h)[8], bool vec, int count) {
  if (vec && count == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) p[e] = __ushort_as_bfloat16(static_cast<unsigned short>(h[e]));
  }
}

__device__ __forceinline__ uint2 load_codes(const uint8_t* p, bool vec, int count) {
  if (vec && count == 8) return *reinterpret_cast<const uint2*>(p);
  uint2 u = make_uint2(0, 0);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < count) (e < 4 ? u.x : u.y) |= static_cast<uint32_t>(p[e]) << (8 * (e & 3));
  return u;
}

__device__ __forceinline__ void store_codes(uint8_t* p, uint2 u, bool vec, int count) {
  if (vec && count == 8) {
    *reinterpret_cast<uint2*>(p) = u;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) p[e] = static_cast<uint8_t>((e < 4 ? u.x : u.y) >> (8 * (e & 3)));
  }
}

__device__ __forceinline__ void decode8(uint2 u, float scale, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = e < 2 ? u.x : u.y;
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * (e & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    v[2 * e] = __fmul_rn(f.x, scale);
    v[2 * e + 1] = __fmul_rn(f.y, scale);
  }
}

// e4m3 codes of x / scale, stochastically: y = |x| / scale <= 448 has the bit
// pattern of an e4m3 float 20 places up once its exponent is rebased by
// 2^-120, subnormals included; ten random bits and half of their last place are
// added below the last place kept, and the rest is cut off.
template <int kShift>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float inv, const uint32_t (&rnd)[8]) {
  uint2 u = make_uint2(0, 0);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float y = __fmul_rn(fabsf(x[e]), inv);
    uint32_t c = (__float_as_uint(__fmul_rn(y, 0x1p-120f)) + (((rnd[e] >> kShift) & 1023u) << 10) + 512u) >> 20;
    c = y == y ? min(c, 0x7eu) : 0x7fu;  // rounding in y can pass the largest value; NaN stays NaN
    c |= x[e] < 0.f ? 0x80u : 0u;
    (e < 4 ? u.x : u.y) |= c << (8 * (e & 3));
  }
  return u;
}

// The block's scale from its lanes' largest magnitudes, and its reciprocal; blocks
// below 2^-100 are held as zeros.
__device__ __forceinline__ float block_scale(const float (&x)[8], float* inv) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(fabsf(x[e])));
  float s = __fmul_rn(__uint_as_float(__reduce_max_sync(kFull, top)), 1.f / kTop);
  if (s < 0x1p-100f) s = 0.f;
  *inv = s == 0.f ? 0.f : __frcp_rn(s);
  return s;
}

template <typename P, typename G, bool k8>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table t) {
  float gs = 1.f;
  if (t.grad_scale) {
    gs = __ldg(t.grad_scale);
    if (!isfinite(gs)) return;  // an overflowed step changes nothing
  }
  int lo = 0, hi = t.n_tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first <= static_cast<int>(blockIdx.x))
      lo = mid;
    else
      hi = mid - 1;
  }
  const Entry& en = t.e[lo];
  const bool vec = en.vec, has_master = en.master != nullptr;
  const long long n = en.n;
  long long i = static_cast<long long>(static_cast<int>(blockIdx.x) - en.first) * t.rounds * kRound + threadIdx.x * kPer;
  for (int r = 0; r < t.rounds; ++r, i += kRound) {
    if (i - (threadIdx.x & 31) * kPer >= n) return;  // the warp's block of 256 is past the end
    const int count = i >= n ? 0 : (n - i < kPer ? static_cast<int>(n - i) : kPer);
    P* param = static_cast<P*>(en.param) + i;
    float p[8], g[8], m[8], v[8];
    load8(static_cast<const G*>(en.grad) + i, g, vec, count);
    if (has_master)
      load8(en.master + i, p, vec, count);
    else
      load8(param, p, vec, count);
    const long long block = i / 256;
    if constexpr (k8) {
      decode8(load_codes(static_cast<const uint8_t*>(en.m) + i, vec, count), en.m_scale[block], m);
      decode8(load_codes(static_cast<const uint8_t*>(en.v) + i, vec, count), en.v_scale[block], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], v[e]);
    } else {
      load8(static_cast<const float*>(en.m) + i, m, vec, count);
      load8(static_cast<const float*>(en.v) + i, v, vec, count);
    }
    float root[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = t.grad_scale ? __fmul_rn(g[e], gs) : g[e];
      m[e] = __fadd_rn(__fmul_rn(m[e], t.b1), __fmul_rn(x, t.c1));
      v[e] = __fadd_rn(__fmul_rn(v[e], t.b2), __fmul_rn(__fmul_rn(x, x), t.c2));
      root[e] = __fsqrt_rn(v[e]);
      const float u = __fdiv_rn(m[e], __fadd_rn(__fmul_rn(root[e], t.isb2), t.eps));
      p[e] = __fsub_rn(__fmul_rn(p[e], en.decay), __fmul_rn(u, en.size));
    }
    uint32_t rnd[8];
    if (k8 || (sizeof(P) == 2 && !has_master)) {
      const uint32_t first = static_cast<uint32_t>(en.index + i);
#pragma unroll
      for (int e = 0; e < 8; ++e) rnd[e] = mix32((first + e) * 0x9e3779b1u + t.key);
    }
    if constexpr (sizeof(P) == 4) {
      store8(param, p, vec, count);
    } else {
      uint32_t h[8];
      if (has_master) {
        store8(en.master + i, p, vec, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = __bfloat16_as_ushort(__float2bfloat16_rn(p[e]));
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t b = __float_as_uint(p[e]);
          h[e] = (isfinite(p[e]) ? b + ((rnd[e] >> 20) << 4) + 8u : b) >> 16;
        }
      }
      store8_16(param, h, vec, count);
    }
    if constexpr (k8) {
      float inv;
      const float ms = block_scale(m, &inv);
      store_codes(static_cast<uint8_t*>(en.m) + i, encode8<0>(m, inv, rnd), vec, count);
      const float vs = block_scale(root, &inv);
      store_codes(static_cast<uint8_t*>(en.v) + i, encode8<10>(root, inv, rnd), vec, count);
      if ((threadIdx.x & 31) == 0) en.m_scale[block] = ms, en.v_scale[block] = vs;
    } else {
      store8(static_cast<float*>(en.m) + i, m, vec, count);
      store8(static_cast<float*>(en.v) + i, v, vec, count);
    }
  }
}

template <typename P, typename G>
int launch_adamw(const Table& t, int blocks, bool k8, cudaStream_t st) {
  if (k8)
    adamw_kernel<P, G, true><<<blocks, kThreads, 0, st>>>(t);
  else
    adamw_kernel<P, G, false><<<blocks, kThreads, 0, st>>>(t);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

int adamw_step(const AdamwArgs& a, int num_sms, cudaStream_t st) {
  const double c1 = 1.0 - std::pow(a.beta1, static_cast<double>(a.step)), c2 = 1.0 - std::pow(a.beta2, static_cast<double>(a.step));
  Table t;
  t.grad_scale = a.grad_scale;
  t.b1 = static_cast<float>(a.beta1), t.c1 = static_cast<float>(1.0 - a.beta1);
  t.b2 = static_cast<float>(a.beta2), t.c2 = static_cast<float>(1.0 - a.beta2);
  t.isb2 = static_cast<float>(1.0 / std::sqrt(c2)), t.eps = static_cast<float>(a.eps);
  t.key = mix32(a.seed + static_cast<uint32_t>(a.step) * 0x9e3779b9u);
  long long total = 0;
  for (int k = 0; k < a.count; ++k) total += a.tensors[k].n;
  t.rounds = total >= 16LL * kRound * num_sms ? 4 : 1;
  int launches = 0;
  for (int k = 0; k < a.count;) {
    t.n_tensors = 0;
    long long blocks = 0;
    for (; k < a.count && t.n_tensors < kMaxTensors && blocks < (1 << 30); ++k) {
      const topk_adamw_tensor& x = a.tensors[k];
      if (x.n == 0) continue;
      Entry& e = t.e[t.n_tensors];
      e = {x.param, x.grad, x.master, x.m, x.v, x.m_scale, x.v_scale, x.n, x.index,
           static_cast<float>(1.0 - x.lr * x.weight_decay), static_cast<float>(x.lr / c1), static_cast<int>(blocks), 0};
      e.vec = aligned(x.param, 16) && aligned(x.grad, 16) && aligned(x.master, 16) && aligned(x.m, a.bits8 ? 8 : 16) &&
              aligned(x.v, a.bits8 ? 8 : 16);
      ++t.n_tensors;
      blocks += (x.n + static_cast<long long>(t.rounds) * kRound - 1) / (static_cast<long long>(t.rounds) * kRound);
    }
    if (t.n_tensors == 0) break;
    int n;
    if (!a.param_bf16)
      n = a.grad_bf16 ? launch_adamw<float, __nv_bfloat16>(t, static_cast<int>(blocks), a.bits8, st)
                      : launch_adamw<float, float>(t, static_cast<int>(blocks), a.bits8, st);
    else
      n = a.grad_bf16 ? launch_adamw<__nv_bfloat16, __nv_bfloat16>(t, static_cast<int>(blocks), a.bits8, st)
                      : launch_adamw<__nv_bfloat16, float>(t, static_cast<int>(blocks), a.bits8, st);
    if (n < 0) return -1;
    launches += n;
  }
  return launches;
}

}  // namespace topk
