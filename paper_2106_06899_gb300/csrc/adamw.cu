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
// gradients) is that of some 54 instructions, of which half at most on the integer pipe:
// shifts are products where the multipliers are free, the codes are cut out of fp32
// patterns with byte permutations, the blocks' maxima are three-input ones, and the
// quotient, which no state depends on, is the hardware's approximation.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace topk {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                          // neighbouring elements of a lane
constexpr int kRound = kThreads * kPer;          // elements of a block at a time
constexpr unsigned kFull = 0xffffffffu;
constexpr float kTop = 448.f;                    // largest e4m3 value
// 307 M bf16 parameters with 8-bit states: 832 us (3.7 TB/s, 55 % of a copy's rate) with three blocks per SM, 32 rounds
// a block and the next round's loads in flight (two blocks per SM, or four, with their spills, are slower).  Four fifths
// of all issue slots are taken: instructions bound it.  Of these the floor under the roots (encode8) costs 39 us, and
// exact roots and separate sums 8: approximate ones put 331 of one step's 614 M codes on the other side of their random
// threshold, and the step would differ from its formula by a place there.
constexpr int kBlocks8 = 3, kRounds8 = 32;

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

// Powers of two that the compiler does not know: a product by one is issued to the multipliers, where it would
// write a shift to the integer pipe, which is the 8-bit step's bottleneck.
struct Powers {
  uint32_t p0, p4, p14, p16;
};

template <int MAX>
struct Table {
  Entry e[MAX];
  const float* grad_scale;
  float b1, c1, b2, c2, isb2, eps;  // c = 1 - b, isb2 = 1 / sqrt(1 - b2^t)
  uint32_t key;
  Powers k;
  int n_tensors, rounds;
};
static_assert(sizeof(Table<kMaxTensors>) <= 32764, "kernel parameters");

// Mixes all bits of x: shifts and two multipliers published by C. Wellons ("Prospecting for Hash Functions", 2018).
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
// A root (not kSigned) above zero gets the smallest code at least.  Cut to zero, it would leave the next update's
// denominator to the next gradient alone, while the first moment, rounded by itself, may have grown to a whole code: a
// step of any length.  Held, the smallest codes' quotient is max|m| / max root of the block, which Adam's moments bound.
template <int kShift, bool kSigned>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float inv, const uint32_t (&rnd)[8], const Powers& k) {
  static_assert(kShift == 0 || kShift == 10, "the ten bits' place");
  uint32_t c[8];
  // a root is zero or above 2^-75 (it is that of an fp32 number): the smaller of it and 2^-125 has code 1's pattern
  const float least = !kSigned && inv > 0.f ? 0x1p-125f : 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t y = __float_as_uint(__fmul_rn(__fmul_rn(fabsf(x[e]), inv), 0x1p-120f));
    const uint32_t r = kShift == 0 ? (rnd[e] & 0x3ffu) * k.p14 + 8192u : (rnd[e] & 0xffc00u) * k.p4 + 8192u;
    c[e] = y * k.p4 + r;  // 16 (y + 1024 random + 512): the code in the top byte
    if (kSigned)
      c[e] = (c[e] & 0x7fffffffu) | (__float_as_uint(x[e]) & 0x80000000u);
    else
      c[e] = max(c[e], __float_as_uint(fminf(x[e], least)));
  }
  uint2 u;
  u.x = __byte_perm(__byte_perm(c[0], c[1], 0x0073), __byte_perm(c[2], c[3], 0x0073), 0x5410);
  u.y = __byte_perm(__byte_perm(c[4], c[5], 0x0073), __byte_perm(c[6], c[7], 0x0073), 0x5410);
  return u;
}

__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
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

// Eight values as they lie in memory.
template <typename T>
struct Raw8 {
  static constexpr int kWords = sizeof(T) * 2;  // 32-bit words
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p, bool vec, int count) {
    if (vec && count == 8) {
#pragma unroll
      for (int i = 0; i < kWords / 4; ++i) {
        const uint4 u = reinterpret_cast<const uint4*>(p)[i];
        w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
      }
    } else {
      float v[8];
      load8(p, v, false, count);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4)
          w[i] = __float_as_uint(v[i]);
        else
          w[i / 2] = i & 1 ? w[i / 2] | __float_as_uint(v[i]) : __float_as_uint(v[i]) >> 16;
      }
    }
  }
  __device__ __forceinline__ void get(float (&v)[8], const Powers& k) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (sizeof(T) == 4)
        v[e] = __uint_as_float(w[e]);
      else
        v[e] = __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] * k.p16);
    }
  }
};

// Stores parameters that no master stands behind: fp32 as they are, bf16 stochastically.
__device__ __forceinline__ void store_param(float* param, const float (&p)[8], const uint32_t (&)[8], const Powers&, bool vec, int count) {
  store8(param, p, vec, count);
}
__device__ __forceinline__ void store_param(__nv_bfloat16* param, const float (&p)[8], const uint32_t (&rnd)[8], const Powers& k, bool vec,
                                            int count) {
  uint32_t h[8];
  // a NaN's pattern must not be added to: 0 p is NaN for one, and for an infinity
  float odd = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    odd = fmaf(p[e], 0.f, odd);
    h[e] = __float_as_uint(p[e]) * k.p0 + ((rnd[e] >> 20) * k.p4 + 8u);
  }
  if (odd != odd) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!isfinite(p[e])) h[e] = __float_as_uint(p[e]);
  }
  store8_16(param, h, vec, count);
}

__device__ __forceinline__ void store_master(float* master, float*, const float (&p)[8], bool vec, int count) {
  store8(master, p, vec, count);
}
__device__ __forceinline__ void store_master(float* master, __nv_bfloat16* param, const float (&p)[8], bool vec, int count) {
  store8(master, p, vec, count);
  uint32_t h[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = static_cast<uint32_t>(__bfloat16_as_ushort(__float2bfloat16_rn(p[e]))) << 16;
  store8_16(param, h, vec, count);
}

__device__ __forceinline__ void random8(uint32_t first, uint32_t key, uint32_t (&rnd)[8]) {
  const uint32_t base = first * 0x9e3779b1u + key;
#pragma unroll
  for (int e = 0; e < 8; ++e) rnd[e] = mix32(base + e * 0x9e3779b1u);
}

// The tensor of a block: the last whose first block is not after it.
template <int MAX>
__device__ __forceinline__ const Entry& entry_of(const Table<MAX>& t) {
  int lo = 0, hi = t.n_tensors - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.e[mid].first <= static_cast<int>(blockIdx.x))
      lo = mid;
    else
      hi = mid - 1;
  }
  return t.e[lo];
}

template <int MAX>
__device__ __forceinline__ bool grad_scale_of(const Table<MAX>& t, float& gs) {
  gs = t.grad_scale ? __ldg(t.grad_scale) : 1.f;
  return isfinite(gs);  // an overflowed step changes nothing
}

// 32-bit states.
template <typename P, typename G, int MAX>
__global__ void __launch_bounds__(kThreads) adamw_kernel(const __grid_constant__ Table<MAX> t) {
  float gs;
  if (!grad_scale_of(t, gs)) return;
  const Entry& en = entry_of(t);
  const bool vec = en.vec, has_master = en.master != nullptr;
  const long long n = en.n;
  long long i = static_cast<long long>(static_cast<int>(blockIdx.x) - en.first) * t.rounds * kRound + threadIdx.x * kPer;
  for (int r = 0; r < t.rounds && i < n; ++r, i += kRound) {
    const int count = n - i < kPer ? static_cast<int>(n - i) : kPer;
    P* param = static_cast<P*>(en.param) + i;
    float p[8], g[8], m[8], v[8];
    load8(static_cast<const G*>(en.grad) + i, g, vec, count);
    if (has_master)
      load8(en.master + i, p, vec, count);
    else
      load8(param, p, vec, count);
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
    if (has_master) {
      store_master(en.master + i, param, p, vec, count);
    } else {
      uint32_t rnd[8];
      if constexpr (sizeof(P) == 2) random8(static_cast<uint32_t>(en.index + i), t.key, rnd);
      store_param(param, p, rnd, t.k, vec, count);
    }
    store8(static_cast<float*>(en.m) + i, m, vec, count);
    store8(static_cast<float*>(en.v) + i, v, vec, count);
  }
}

// 8-bit states.
template <typename S, typename G>
struct Held8 {  // a lane's eight elements as they lie in memory
  Raw8<S> p;
  Raw8<G> g;
  uint2 m, v;
  float ms, vs;
};

// Eight elements at offset `at` of the block's chunk: the update, then the block's new scales and codes.
// FULL: a whole, aligned chunk; else `count` elements, one access each where `vec` is false.
template <bool FULL, typename P, typename G, bool MASTER, int MAX>
struct Step8 {
  using S = std::conditional_t<MASTER, float, P>;  // what the parameters are read from
  const Table<MAX>& t;
  const Entry& en;
  const float gs;
  // the chunk's addresses, the same for all threads
  P* const param;
  const G* const grad;
  float* const master;
  uint8_t *const m8, *const v8;
  float *const m_scale, *const v_scale;
  const uint32_t index;
  const int left;
  const bool vec;

  __device__ __forceinline__ Step8(const Table<MAX>& t_, const Entry& e, float gs_, long long start, int left_)
      : t(t_), en(e), gs(gs_), param(static_cast<P*>(e.param) + start), grad(static_cast<const G*>(e.grad) + start),
        master(e.master + start), m8(static_cast<uint8_t*>(e.m) + start), v8(static_cast<uint8_t*>(e.v) + start),
        m_scale(e.m_scale + start / 256), v_scale(e.v_scale + start / 256), index(static_cast<uint32_t>(e.index + start)), left(left_), vec(e.vec) {}

  __device__ __forceinline__ int count(unsigned at) const {
    return FULL ? kPer : max(0, min(kPer, left - static_cast<int>(at)));
  }
  __device__ __forceinline__ void load(unsigned at, Held8<S, G>& h) const {
    const int n = count(at);
    const bool wide = FULL || vec;
    h.g.load(grad + at, wide, n);
    if constexpr (MASTER)
      h.p.load(master + at, wide, n);
    else
      h.p.load(param + at, wide, n);
    h.m = load_codes(m8 + at, wide, n);
    h.v = load_codes(v8 + at, wide, n);
    h.ms = m_scale[at / 256], h.vs = v_scale[at / 256];
  }
  __device__ __forceinline__ void work(unsigned at, const Held8<S, G>& h) const {
    const int n = count(at);
    const bool wide = FULL || vec;
    float p[8], g[8], m[8], v[8];
    h.g.get(g, t.k);
    h.p.get(p, t.k);
    decode8(h.m, m);
    decode8(h.v, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = g[e] * gs, r0 = __fmul_rn(v[e], h.vs);
      m[e] = __fadd_rn(__fmul_rn(__fmul_rn(m[e], h.ms), t.b1), __fmul_rn(x, t.c1));
      v[e] = __fsqrt_rn(__fadd_rn(__fmul_rn(__fmul_rn(r0, r0), t.b2), __fmul_rn(__fmul_rn(x, x), t.c2)));
      const float u = m[e] * rcp_fast(fmaf(v[e], t.isb2, t.eps));
      p[e] = fmaf(p[e], en.decay, -en.size * u);
    }
    uint32_t rnd[8];
    random8(index + at, t.key, rnd);
    if constexpr (MASTER)
      store_master(master + at, param + at, p, wide, n);
    else
      store_param(param + at, p, rnd, t.k, wide, n);
    float inv;
    const float ms1 = block_scale(m, &inv);
    store_codes(m8 + at, encode8<0, true>(m, inv, rnd, t.k), wide, n);
    const float vs1 = block_scale(v, &inv);
    store_codes(v8 + at, encode8<10, false>(v, inv, rnd, t.k), wide, n);
    if ((threadIdx.x & 31) == 0) m_scale[at / 256] = ms1, v_scale[at / 256] = vs1;
  }
};

template <typename P, typename G, bool MASTER, int MAX>
__global__ void __launch_bounds__(kThreads, kBlocks8) adamw8_kernel(const __grid_constant__ Table<MAX> t) {
  float gs;
  if (!grad_scale_of(t, gs)) return;
  const Entry& en = entry_of(t);
  const long long start = static_cast<long long>(static_cast<int>(blockIdx.x) - en.first) * t.rounds * kRound;
  const int chunk = t.rounds * kRound, left = en.n - start < chunk ? static_cast<int>(en.n - start) : chunk;
  const unsigned at0 = threadIdx.x * kPer;
  if (en.vec && left == chunk) {
    const Step8<true, P, G, MASTER, MAX> s(t, en, gs, start, left);
    Held8<typename Step8<true, P, G, MASTER, MAX>::S, G> a, b;
    s.load(at0, a);
#pragma unroll 1
    for (int at = 0;; at += 2 * kRound) {
      const bool second = at + kRound < chunk;
      if (second) s.load(at0 + at + kRound, b);
      s.work(at0 + at, a);
      if (!second) return;
      const bool third = at + 2 * kRound < chunk;
      if (third) s.load(at0 + at + 2 * kRound, a);
      s.work(at0 + at + kRound, b);
      if (!third) return;
    }
    return;
  }
  const Step8<false, P, G, MASTER, MAX> s(t, en, gs, start, left);
#pragma unroll 1
  for (int at = 0; at + static_cast<int>(at0 & ~255u) < left; at += kRound) {  // while the warp's block of 256 has elements
    Held8<typename Step8<false, P, G, MASTER, MAX>::S, G> h;
    s.load(at0 + at, h);
    s.work(at0 + at, h);
  }
}

template <typename P, typename G, int MAX>
int launch_adamw(const Table<MAX>& t, int blocks, bool k8, cudaStream_t st) {
  if (!k8) {
    adamw_kernel<P, G, MAX><<<blocks, kThreads, 0, st>>>(t);
  } else if constexpr (sizeof(P) == 2) {
    if (t.e[0].master)
      adamw8_kernel<P, G, true, MAX><<<blocks, kThreads, 0, st>>>(t);
    else
      adamw8_kernel<P, G, false, MAX><<<blocks, kThreads, 0, st>>>(t);
  } else {
    adamw8_kernel<P, G, false, MAX><<<blocks, kThreads, 0, st>>>(t);
  }
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

template <int MAX>
int step(const AdamwArgs& a, int num_sms, cudaStream_t st) {
  const double c1 = 1.0 - std::pow(a.beta1, static_cast<double>(a.step)), c2 = 1.0 - std::pow(a.beta2, static_cast<double>(a.step));
  Table<MAX> t;
  t.grad_scale = a.grad_scale;
  t.k = {1u, 1u << 4, 1u << 14, 1u << 16};
  t.b1 = static_cast<float>(a.beta1), t.c1 = static_cast<float>(1.0 - a.beta1);
  t.b2 = static_cast<float>(a.beta2), t.c2 = static_cast<float>(1.0 - a.beta2);
  t.isb2 = static_cast<float>(1.0 / std::sqrt(c2)), t.eps = static_cast<float>(a.eps);
  t.key = mix32(a.seed + static_cast<uint32_t>(a.step) * 0x9e3779b9u);
  long long total = 0;
  for (int k = 0; k < a.count; ++k) total += a.tensors[k].n;
  // the rounds of a block share its start (the search for its tensor), as many as leave every SM a dozen blocks
  const long long most = a.bits8 ? kRounds8 : 4, fair = total / (12LL * kRound * num_sms);
  t.rounds = static_cast<int>(fair < 1 ? 1 : (fair < most ? fair : most));
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
