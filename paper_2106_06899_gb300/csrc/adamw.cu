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
// gives the same bits whenever it is repeated.
//
// With 8-bit states the memory time of an element (10 bytes with bf16 parameters and
// gradients) is that of some 54 instructions: the scales take up b1, b2 and the
// gradient's factors, roots and reciprocals are the hardware's approximations (2^-22; the
// root's code is rounded to 2^-4 of it), the codes are cut out of fp32 patterns with byte
// permutations and the blocks' maxima are three-input ones.
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

constexpr int kMaxTensors = 352, kFewTensors = 32;

template <int MAX>
struct Table {
  Entry e[MAX];
  const float* grad_scale;
  float b1, c1, b2, c2, rb2, rc2, isb2, eps;  // c = 1 - b, rb2 and rc2 the roots of b2 and c2, isb2 = 1 / sqrt(1 - b2^t)
  uint32_t key;
  int n_tensors, rounds;
};
static_assert(sizeof(Table<kMaxTensors>) <= 32764, "kernel parameters");

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

// eight bf16 patterns, each in the upper half of a word
__device__ __forceinline__ void store8_16(__nv_bfloat16* p, const uint32_t (&h)[8], bool vec, int count) {
  if (vec && count == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(__byte_perm(h[0], h[1], 0x7632), __byte_perm(h[2], h[3], 0x7632),
                                              __byte_perm(h[4], h[5], 0x7632), __byte_perm(h[6], h[7], 0x7632));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < count) p[e] = __ushort_as_bfloat16(static_cast<unsigned short>(h[e] >> 16));
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

// Codes as floats, without the scale.
__device__ __forceinline__ void decode8(uint2 u, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t w = e < 2 ? u.x : u.y;
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w >> (16 * (e & 1))), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    v[2 * e] = f.x;
    v[2 * e + 1] = f.y;
  }
}

// e4m3 codes of x / scale, stochastically: y = |x| / scale <= 448 has the bit pattern of an e4m3 float 20
// places up once its exponent is rebased by 2^-120, subnormals included; ten random bits and half of
// their last place are added below the last place kept, and the rest is cut off.  At y = 448 the sum
// stays below the next code by 511 units, more than y's rounding: no clamp.  Where y is not a number the
// scale is not either, and the code does not matter.
template <int kShift, bool kSigned>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float inv, const uint32_t (&rnd)[8]) {
  uint32_t c[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t r = kShift == 0 ? ((rnd[e] << 10) & 0xffc00u) | 512u : (rnd[e] & 0xffc00u) | 512u;
    static_assert(kShift == 0 || kShift == 10, "the ten bits' place");
    const float y = __fmul_rn(__fmul_rn(fabsf(x[e]), inv), 0x1p-120f);
    c[e] = (__float_as_uint(y) + r) << 4;  // the code in the top byte
    if (kSigned) c[e] = (c[e] & 0x7fffffffu) | (__float_as_uint(x[e]) & 0x80000000u);
  }
  uint2 u;
  u.x = __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
  u.y = __byte_perm(__byte_perm(c[4], c[5], 0x0073), __byte_perm(c[6], c[7], 0x0073), 0x5410);
  return u;
}

// max(a, b, c); a NaN wins
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// The block's scale from its lanes' largest magnitudes, and its reciprocal; blocks below 2^-100 are held
// as zeros.  Bit patterns of magnitudes order as the magnitudes do, a NaN above all.
__device__ __forceinline__ float block_scale(const float (&x)[8], float* inv) {
  const float a = max3_nan(fabsf(x[0]), fabsf(x[1]), fabsf(x[2])), b = max3_nan(fabsf(x[3]), fabsf(x[4]), fabsf(x[5]));
  const float top = max3_nan(max3_nan(a, b, fabsf(x[6])), fabsf(x[7]), 0.f);
  float s = __fmul_rn(__uint_as_float(__reduce_max_sync(kFull, __float_as_uint(top))), 1.f / kTop);
  if (s < 0x1p-100f) s = 0.f;
  *inv = s == 0.f ? 0.f : __frcp_rn(s);
  return s;
}

__device__ __forceinline__ float sqrt_fast(float x) {
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

template <typename P, typename G, bool k8, int MAX>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<MAX> t) {
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
    float root[8];
    if constexpr (k8) {
      // b1 and the root of b2 go into the blocks' scales: v = (code scale sqrt(b2))^2 + (g sqrt(1 - b2))^2
      decode8(load_codes(static_cast<const uint8_t*>(en.m) + i, vec, count), m);
      decode8(load_codes(static_cast<const uint8_t*>(en.v) + i, vec, count), v);
      const float ms = en.m_scale[block] * t.b1, vs = en.v_scale[block] * t.rb2, gc1 = gs * t.c1, gc2 = gs * t.rc2;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] = fmaf(m[e], ms, g[e] * gc1);
        const float r0 = v[e] * vs, r1 = g[e] * gc2;
        root[e] = sqrt_fast(fmaf(r0, r0, r1 * r1));
        const float u = m[e] * rcp_fast(fmaf(root[e], t.isb2, t.eps));
        p[e] = fmaf(p[e], en.decay, -en.size * u);
      }
    } else {
      load8(static_cast<const float*>(en.m) + i, m, vec, count);
      load8(static_cast<const float*>(en.v) + i, v, vec, count);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = g[e] * gs;
        m[e] = __fadd_rn(__fmul_rn(m[e], t.b1), __fmul_rn(x, t.c1));
        v[e] = __fadd_rn(__fmul_rn(v[e], t.b2), __fmul_rn(__fmul_rn(x, x), t.c2));
        const float u = __fdiv_rn(m[e], __fadd_rn(__fmul_rn(__fsqrt_rn(v[e]), t.isb2), t.eps));
        p[e] = __fsub_rn(__fmul_rn(p[e], en.decay), __fmul_rn(u, en.size));
      }
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
        for (int e = 0; e < 8; ++e) h[e] = static_cast<uint32_t>(__bfloat16_as_ushort(__float2bfloat16_rn(p[e]))) << 16;
      } else {
        // a NaN's pattern must not be added to: 0 p is NaN for one, and for an infinity
        float odd = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          odd = fmaf(p[e], 0.f, odd);
          h[e] = __float_as_uint(p[e]) + (((rnd[e] >> 16) & 0xfff0u) | 8u);
        }
        if (odd != odd) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (!isfinite(p[e])) h[e] = __float_as_uint(p[e]);
        }
      }
      store8_16(param, h, vec, count);
    }
    if constexpr (k8) {
      float inv;
      const float ms = block_scale(m, &inv);
      store_codes(static_cast<uint8_t*>(en.m) + i, encode8<0, true>(m, inv, rnd), vec, count);
      const float vs = block_scale(root, &inv);
      store_codes(static_cast<uint8_t*>(en.v) + i, encode8<10, false>(root, inv, rnd), vec, count);
      if ((threadIdx.x & 31) == 0) en.m_scale[block] = ms, en.v_scale[block] = vs;
    } else {
      store8(static_cast<float*>(en.m) + i, m, vec, count);
      store8(static_cast<float*>(en.v) + i, v, vec, count);
    }
  }
}

template <typename P, typename G, int MAX>
int launch_adamw(const Table<MAX>& t, int blocks, bool k8, cudaStream_t st) {
  if (k8)
    adamw_kernel<P, G, true, MAX><<<blocks, kThreads, 0, st>>>(t);
  else
    adamw_kernel<P, G, false, MAX><<<blocks, kThreads, 0, st>>>(t);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <int MAX>
int step(const AdamwArgs& a, int num_sms, cudaStream_t st) {
  const double c1 = 1.0 - std::pow(a.beta1, static_cast<double>(a.step)), c2 = 1.0 - std::pow(a.beta2, static_cast<double>(a.step));
  Table<MAX> t;
  t.grad_scale = a.grad_scale;
  t.b1 = static_cast<float>(a.beta1), t.c1 = static_cast<float>(1.0 - a.beta1);
  t.b2 = static_cast<float>(a.beta2), t.c2 = static_cast<float>(1.0 - a.beta2);
  t.rb2 = static_cast<float>(std::sqrt(a.beta2)), t.rc2 = static_cast<float>(std::sqrt(1.0 - a.beta2));
  t.isb2 = static_cast<float>(1.0 / std::sqrt(c2)), t.eps = static_cast<float>(a.eps);
  t.key = mix32(a.seed + static_cast<uint32_t>(a.step) * 0x9e3779b9u);
  long long total = 0;
  for (int k = 0; k < a.count; ++k) total += a.tensors[k].n;
  // a block's start (the search for its tensor) is shared by four rounds where there are blocks enough
  t.rounds = total >= 16LL * kRound * num_sms ? 4 : 1;
  const long long chunk = static_cast<long long>(t.rounds) * kRound;
  int launches = 0;
  for (int k = 0; k < a.count;) {
    t.n_tensors = 0;
    long long blocks = 0;
    for (; k < a.count && t.n_tensors < MAX; ++k) {
      const topk_adamw_tensor& x = a.tensors[k];
      if (x.n == 0) continue;
      const long long more = (x.n + chunk - 1) / chunk;
      if (blocks + more > (1ll << 30)) break;
      Entry& e = t.e[t.n_tensors++];
      e = {x.param, x.grad, x.master, x.m, x.v, x.m_scale, x.v_scale, x.n, x.index,
           static_cast<float>(1.0 - x.lr * x.weight_decay), static_cast<float>(x.lr / c1), static_cast<int>(blocks), 0};
      e.vec = aligned(x.param, 16) && aligned(x.grad, 16) && aligned(x.master, 16) && aligned(x.m, a.bits8 ? 8 : 16) &&
              aligned(x.v, a.bits8 ? 8 : 16);
      blocks += more;
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

}  // namespace

int adamw_step(const AdamwArgs& a, int num_sms, cudaStream_t st) {
  // the parameters of a launch are copied whole: a short table where it does
  return a.count <= kFewTensors ? step<kFewTensors>(a, num_sms, st) : step<kMaxTensors>(a, num_sms, st);
}

}  // namespace topk
