// logprob.cu -- log probabilities of tokens from their logits: the target's, the entropy, the largest
// alternatives, and the gradient.
//
// Forward, one pass over a row: with a reference r near the maximum and d = c (x - r), c = scale log2 e, the sums S of 2^d and
// T of 2^d d give lse = scale r + ln S and the entropy ln S - ln 2 T / S.  A thread keeps its own reference and raises it
// only where an element exceeds it by more than kRaise; references are brought together at the end.
// Alternatives: after a block's first tile the top-th largest of 64 to 256 groups' maxima is a value that at least `top` elements
// of the tile reach, and 1.1 to 1.4 times as many, in each tile after it too where likely tokens lie anywhere.  The pass notes which vectors reach it; these few are
// looked at once more, an element a thread, and what reaches it is ranked (taken out of the vector as it passes, by the
// lane that holds it, a candidate holds up its whole warp: 110 us in place of 100).  A row with more candidates
// than the buffers hold is read a second time with a threshold that is raised whenever the buffer fills: values that rise along the row, thousands
// of equal ones, a first tile of masked tokens, and many alternatives of a vocabulary of many tiles without its likely tokens in the first one.  That
// takes up to eleven times as long: 4,096 rows of 131,072 fp32 with 64 alternatives 3.2 ms, and 0.43 ms with the likely tokens first.
//
// A block takes a row, or a cluster of up to eight blocks a share of it each where there are few rows (a decoding step): the
// first block then collects the others' sums and alternatives from their shared memory.
//
// Backward: elementwise from lse and the entropy, the row's few targets and alternatives patched in by the block
// that wrote the row's piece.  Both are bound by memory.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "kernels.h"

namespace cg = cooperative_groups;

namespace topk {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kRaise = 6.f;  // in powers of two
constexpr int kThreads = 256;
constexpr int kKept = 2048;    // alternatives' candidates of a block
constexpr int kMostBlocks = 8; // of a row: the portable size of a cluster

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }

// 2^x (ex2.approx, 2^-22); 2^-inf = 0, and NaN stays
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ long long target_at(const LogprobArgs& a, int n) {
  if (!a.targets) return -1;
  return a.targets64 ? __ldg(static_cast<const long long*>(a.targets) + n) : __ldg(static_cast<const int*>(a.targets) + n);
}

// Larger values first, then lower indices, as one number (0: none); -0 as 0.
__device__ __forceinline__ unsigned long long key_of(float v, int j) {
  const unsigned b = __float_as_uint(v + 0.f), o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return static_cast<unsigned long long>(o) << 32 | ~static_cast<unsigned>(j);
}
__device__ __forceinline__ float value_of(unsigned long long key) {
  const unsigned o = static_cast<unsigned>(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// Sixteen bytes of elements.
template <typename T>
struct Vec {
  static constexpr int N = 16 / sizeof(T);
  uint4 u;
  __device__ __forceinline__ void get(float (&x)[N]) const {
    if constexpr (sizeof(T) == 2) {
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(w[e] << 16), x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    } else {
      x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y), x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
    }
  }
  __device__ __forceinline__ void set(const float (&x)[N]) {
    if constexpr (sizeof(T) == 2) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&h);
      }
      u = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      u = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    }
  }
};

template <typename T>
__device__ __forceinline__ Vec<T> load_vec(const T* p) {
  Vec<T> v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.u.x), "=r"(v.u.y), "=r"(v.u.z), "=r"(v.u.w) : "l"(p));
  return v;
}

// What a set of elements says: S and T around a reference.  NaN or +inf among them shows in s.
struct Sums {
  float r, s, t;
  __device__ __forceinline__ void add(const Sums& o, float c) {
    const float to = fmaxf(r, o.r);
    if (to == -INFINITY) {  // nothing yet, but perhaps a NaN
      s += o.s;
      return;
    }
    // a side without an element has s = 0; one that is far below the other adds nothing to t
    const float d0 = fmaxf((r - to) * c, -300.f), d1 = fmaxf((o.r - to) * c, -300.f), f0 = exp2_fast(d0), f1 = exp2_fast(d1);
    t = f0 * (t + d0 * s) + f1 * (o.t + d1 * o.s);
    s = (r == -INFINITY ? s : f0 * s) + (o.r == -INFINITY ? o.s : f1 * o.s);
    r = to;
  }
  __device__ __forceinline__ void add_lane(int from, float c) {  // of the warp
    Sums o;
    o.r = __shfl_down_sync(0xffffffffu, r, from), o.s = __shfl_down_sync(0xffffffffu, s, from), o.t = __shfl_down_sync(0xffffffffu, t, from);
    add(o, c);
  }
};

// The largest of a vector's elements, NaN left out.
__device__ __forceinline__ float most_of(const Vec<__nv_bfloat16>& v) {
  const __nv_bfloat162* w = reinterpret_cast<const __nv_bfloat162*>(&v.u);
  const __nv_bfloat162 m = __hmax2(__hmax2(w[0], w[1]), __hmax2(w[2], w[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
__device__ __forceinline__ float most_of(const Vec<float>& v) {
  float x[4];
  v.get(x);
  return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
}

// Elements raised to `floor`; NaN stays.
__device__ __forceinline__ Vec<__nv_bfloat16> at_least(Vec<__nv_bfloat16> v, float floor) {
  __nv_bfloat162* w = reinterpret_cast<__nv_bfloat162*>(&v.u);
  const __nv_bfloat162 f = __float2bfloat162_rn(floor);
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] = __hmax2_nan(w[e], f);
  return v;
}
__device__ __forceinline__ Vec<float> at_least(Vec<float> v, float floor) {
  uint32_t* w = reinterpret_cast<uint32_t*>(&v.u);
#pragma unroll
  for (int e = 0; e < 4; ++e) asm("max.NaN.f32 %0, %1, %2;" : "=r"(w[e]) : "r"(w[e]), "f"(floor));
  return v;
}

// A thread's sums; t without the factor c.
struct Running {
  float r = -INFINITY, s = 0.f, t = 0.f;
  float floor = -INFINITY;  // elements below it are taken for it: their 2^d is 0, and 0 x d must not be NaN

  __device__ __forceinline__ void raise(float top, float c) {
    if ((top - r) * c > kRaise) {  // the first element too: r is -inf
      if (r > -INFINITY) {
        const float d = r - top, f = exp2_fast(d * c);
        t = f == 0.f ? 0.f : f * fmaf(d, s, t), s *= f;
      }
      r = top;
      // as a bf16, as at_least takes it (a finite one that rounds to -inf there would leave -inf elements, and 0 x -inf, in the sums); the last
      // part outlasts the rounding
      floor = __bfloat162float(__float2bfloat16_rn(top - 300.f / c - fabsf(top) * 0.03125f));
    }
  }
  // the vector's elements, `most` the largest of them
  template <typename T>
  __device__ __forceinline__ void take(const Vec<T>& v, float c, float most) {
    raise(most, c);
    float x[Vec<T>::N];
    if (floor == -INFINITY) {  // no element that counts yet, or none above the type's lowest values
      v.get(x);
#pragma unroll
      for (int e = 0; e < Vec<T>::N; ++e) add_one(x[e], c);
      return;
    }
    at_least(v, floor).get(x);
#pragma unroll
    for (int e = 0; e < Vec<T>::N; ++e) {
      const float d = x[e] - r, p = exp2_fast(d * c);
      s += p;
      t = fmaf(p, d, t);
    }
  }
  __device__ __forceinline__ void take_one(float x, float c) {
    raise(x, c);
    add_one(x, c);
  }
  __device__ __forceinline__ void add_one(float x, float c) {
    const float d = x - (r == -INFINITY ? 0.f : r), p = exp2_fast(d * c);
    s += p;
    t = p == 0.f ? t : fmaf(p, d, t);
  }
  __device__ __forceinline__ Sums sums(float c) const { return Sums{r, s, t * c}; }
};

// Sorts `n` (a power of two) keys, largest first; all threads.
__device__ void sort_keys(unsigned long long* k, int n) {
  for (int size = 2; size <= n; size *= 2)
    for (int step = size / 2; step; step /= 2) {
      for (int i = threadIdx.x; i < n / 2; i += kThreads) {
        const int lo = (i / step) * 2 * step + i % step, hi = lo + step;
        const unsigned long long a = k[lo], b = k[hi];
        if ((a < b) == ((lo & size) == 0)) k[lo] = b, k[hi] = a;
      }
      __syncthreads();
    }
}

struct Shared {
  alignas(16) unsigned long long kept[kKept];
  unsigned long long best[kMaxAlternatives];
  int hits[kKept];  // vectors with a candidate
  float groups[kThreads];
  Sums sums[kThreads / 32];
  Sums total;
  unsigned long long threshold;
  float bar;
  int vectors, count, have;  // with candidates, candidates, and the best among them
};

// The `top` best candidates in order; all threads.
__device__ void rank(Shared& sh, int top) {
  __syncthreads();
  const int n = min(sh.count, kKept);
  if (n <= 2 * kThreads) {
    if (threadIdx.x == 0 && n % 2) sh.kept[n] = 0;
    __syncthreads();
    for (int t = threadIdx.x; t < n; t += kThreads) {
      const unsigned long long k = sh.kept[t];
      int before = 0;
#pragma unroll 4
      for (int i = 0; i < n; i += 2) {  // kept has an even length, and 0 behind an odd number of candidates
        const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(sh.kept + i);
        before += (two.x > k) + (two.y > k);
      }
      if (before < top) sh.best[before] = k;
    }
  } else {
    for (int i = n + threadIdx.x; i < kKept; i += kThreads) sh.kept[i] = 0;
    __syncthreads();
    sort_keys(sh.kept, kKept);
    if (static_cast<int>(threadIdx.x) < top) sh.best[threadIdx.x] = sh.kept[threadIdx.x];
  }
  if (threadIdx.x == 0) sh.have = min(n, top);
  __syncthreads();
}

// Candidates of elements [e0, e1) and the row's ends once more, with a threshold that follows the `top` best so far.
template <typename T>
__device__ __noinline__ void rescan(Shared& sh, const T* x, int e0, int e1, int lead, int tail, int V, int top) {
  __syncthreads();
  if (threadIdx.x == 0) sh.count = 0, sh.threshold = 1;
  __syncthreads();
  const int n = e1 - e0 + lead + V - tail;
  for (int i0 = 0; i0 < n; i0 += kThreads) {
    if (sh.count + kThreads > kKept) {
      rank(sh, top);
      if (static_cast<int>(threadIdx.x) < sh.have) sh.kept[threadIdx.x] = sh.best[threadIdx.x];
      __syncthreads();
      if (threadIdx.x == 0) {
        sh.count = sh.have;
        sh.threshold = sh.have == top ? sh.best[top - 1] : 1;
      }
    }
    __syncthreads();
    const int i = i0 + threadIdx.x;
    if (i < n) {
      const int j = i < e1 - e0 ? e0 + i : i - (e1 - e0) < lead ? i - (e1 - e0) : tail + i - (e1 - e0) - lead;
      const float v = to_f(x[j]);
      const unsigned long long key = key_of(v, j);
      if (v > -INFINITY && key >= sh.threshold) sh.kept[atomicAdd(&sh.count, 1)] = key;
    }
    __syncthreads();
  }
}

// 4,099 rows of 50,001 bf16 logits with 8 alternatives: 100 us, 4.1 TB/s.  Without alternatives a warp issues 10.6 instructions an
// element (2^x alone takes the special units 44 us) and about 3,500 a row, whose ends, sums and threshold are the rest; a
// decoding step, 4 rows of 131,072 with 20 alternatives, takes 10 us, which is the latency of the same steps.  Products of two elements
// at a time (100 us), five or six blocks an SM with half the loads in flight (97, but 13 for the decoding step) and three
// (110) were measured.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads, 4)
    logprob_fwd_kernel(LogprobArgs a, float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, DevCtl ctl) {
  constexpr int N = Vec<T>::N, UNROLL = 4;
  __shared__ Shared sh;
  cg::cluster_group cluster = cg::this_cluster();
  const int blocks = static_cast<int>(cluster.num_blocks()), rank_here = static_cast<int>(cluster.block_rank());
  const int n = blockIdx.x / blocks;
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(n) * a.stride;
  const float c = a.scale * kLog2e;

  // the elements before the first 16-byte boundary and behind the last one go to the first block; whole vectors between
  const int lead = min(a.V, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T)));
  const int vecs = (a.V - lead) / N, tail = lead + vecs * N;
  const T* body = x + lead;
  const int each = (vecs + blocks - 1) / blocks, v0 = min(vecs, rank_here * each), v1 = min(vecs, v0 + each);
  int edge = -1;  // this thread's element of the ends
  if (rank_here == 0) {
    const int k = threadIdx.x;
    edge = k < lead ? k : k - lead < a.V - tail ? tail + k - lead : -1;
  }
  Running mine;
  float edge_x = -INFINITY;
  if (edge >= 0) {
    edge_x = to_f(x[edge]);
    mine.take_one(edge_x, c);
  }
  float bar = -INFINITY;
  const auto offer = [&](float v, int j) {
    if (v >= bar) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < kKept) sh.kept[at] = key_of(v, j);
    }
  };
  if (TOP && threadIdx.x == 0) sh.count = sh.vectors = 0;
  Vec<T> ahead[UNROLL];
  const auto fetch = [&](int v) {
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      const int at = v + i * kThreads + threadIdx.x;
      if (at < v1) ahead[i] = load_vec(body + static_cast<size_t>(at) * N);
    }
  };
  fetch(v0);
  for (int v = v0; v == v0 || v < v1; v += kThreads * UNROLL) {
    Vec<T> u[UNROLL];
    float most[UNROLL];
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) u[i] = ahead[i];
    fetch(v + kThreads * UNROLL);
#pragma unroll
    for (int i = 0; i < UNROLL; ++i) {
      most[i] = -INFINITY;
      if (v + i * kThreads + static_cast<int>(threadIdx.x) >= v1) continue;
      most[i] = most_of(u[i]);
      mine.take(u[i], c, most[i]);
    }
    if constexpr (TOP) {
      if (v == v0) {
        // 64 to 256 groups of neighbouring threads, twice as many as alternatives or more where there are
        const int lanes = a.top <= 32 ? 4 : a.top <= 64 ? 2 : 1, groups = kThreads / lanes;
        float high = fmaxf(edge_x, fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3])));
        for (int o = 1; o < lanes; o *= 2) high = fmaxf(high, __shfl_xor_sync(0xffffffffu, high, o));
        if (threadIdx.x % lanes == 0) sh.groups[threadIdx.x / lanes] = high;
        if (threadIdx.x == 0) sh.bar = -INFINITY;
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < groups) {
          const float g = sh.groups[threadIdx.x];
          int before = 0;
#pragma unroll 8
          for (int i = 0; i < groups; ++i) before += sh.groups[i] > g || (sh.groups[i] == g && i < static_cast<int>(threadIdx.x));
          if (before == a.top - 1) sh.bar = g;
        }
        __syncthreads();
        bar = fmaxf(sh.bar, -3.402823466e38f);  // -inf is no candidate
        if (edge >= 0) offer(edge_x, edge);
      }
#pragma unroll
      for (int i = 0; i < UNROLL; ++i) {
        if (most[i] >= bar) {
          const int at = atomicAdd(&sh.vectors, 1);
          if (at < kKept) sh.hits[at] = v + i * kThreads + threadIdx.x;
        }
      }
    }
  }
  if constexpr (TOP) {
    __syncthreads();
    // the few vectors that reach the bar once more, an element a thread
    for (int i = threadIdx.x, end = min(sh.vectors, kKept) * N; i < end; i += kThreads) {
      const int j = sh.hits[i / N] * N + i % N;
      offer(to_f(body[j]), lead + j);
    }
    __syncthreads();
    if (max(sh.count, sh.vectors) > kKept) rescan(sh, x, lead + v0 * N, lead + v1 * N, rank_here == 0 ? lead : 0, rank_here == 0 ? tail : a.V, a.V, a.top);
    rank(sh, a.top);
  }

  // sums: lanes, warps, blocks, in this order
  Sums all = mine.sums(c);
#pragma unroll
  for (int o = 16; o; o >>= 1) all.add_lane(o, c);
  if (threadIdx.x % 32 == 0) sh.sums[threadIdx.x / 32] = all;
  __syncthreads();
  if (threadIdx.x < 32) {
    all = threadIdx.x < kThreads / 32 ? sh.sums[threadIdx.x] : Sums{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int o = kThreads / 64; o; o >>= 1) all.add_lane(o, c);
    if (threadIdx.x == 0) sh.total = all, sh.count = 0;
  }
  if (blocks > 1) {
    cluster.sync();
    if (rank_here == 0) {
      // a warp for each block's alternatives, a lane for each one's sums: other blocks' memory is far away
      const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
      if (warp == 0) {
        all = lane < blocks ? *cluster.map_shared_rank(&sh.total, lane) : Sums{-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int o = kMostBlocks / 2; o; o >>= 1) all.add_lane(o, c);
      }
      if constexpr (TOP) {
        static_assert(kThreads / 32 >= kMostBlocks && kMostBlocks * kMaxAlternatives <= kKept, "a warp and a list for each block");
        if (warp < blocks) {
          const Shared* from = cluster.map_shared_rank(&sh, warp);
          const int have = from->have;
#pragma unroll
          for (int i = 0; i < kMaxAlternatives; i += 32)  // best holds anything from `have` on
            if (i + lane < a.top) {
              const unsigned long long k = from->best[i + lane];
              sh.kept[warp * kMaxAlternatives + i + lane] = i + lane < have ? k : 0;
            }
        }
        __syncthreads();
        // the lists are sorted: an element's rank is its place in its own and how many of each other one are larger
        for (int t = threadIdx.x; t < blocks * a.top; t += kThreads) {
          const int list = t / a.top, i = t % a.top;
          const unsigned long long k = sh.kept[list * kMaxAlternatives + i];
          int before = i;
          for (int o = 0; o < blocks && before < a.top; ++o) {
            if (o == list) continue;
            int lo = 0, hi = a.top;  // elements below lo are larger, from hi on they are not
            while (lo < hi) {
              const int mid = (lo + hi) / 2;
              if (sh.kept[o * kMaxAlternatives + mid] > k)
                lo = mid + 1;
              else
                hi = mid;
            }
            before += lo;
          }
          if (k && before < a.top) sh.best[before] = k;
          if (k && before < a.top) atomicAdd(&sh.count, 1);
        }
      }
      __syncthreads();
      if (threadIdx.x == 0) sh.total = all, sh.have = sh.count;
    }
    cluster.sync();  // no block leaves before its shared memory has been read
  }
  if (rank_here != 0) return;
  __syncthreads();
  all = sh.total;
  const bool bad = !(all.s < INFINITY), none = all.s == 0.f;
  const float ln_s = logf(all.s);
  const auto log_p = [&](float v) { return bad ? NAN : v == -INFINITY ? -INFINITY : fmaf(v - all.r, a.scale, -ln_s); };
  if (threadIdx.x == 0) {
    if (lse) lse[n] = bad ? NAN : none ? -INFINITY : fmaf(all.r, a.scale, ln_s);
    const float h = ln_s - kLn2 * all.t / all.s;
    if (entropy) entropy[n] = bad ? NAN : none || h < 0.f ? 0.f : h;  // a NaN stays one
    const long long target = target_at(a, n);
    if (target >= a.V) atomicOr(ctl.error, kDevErrRange);
    if (logp) logp[n] = target >= 0 && target < a.V ? log_p(to_f(x[target])) : 0.f;
  }
  if constexpr (TOP) {
    const int i = threadIdx.x;
    if (i < a.top) {
      const bool have = !bad && i < sh.have;
      top_ids[static_cast<size_t>(n) * a.top + i] = have ? static_cast<int>(~static_cast<unsigned>(sh.best[i])) : -1;
      top_logp[static_cast<size_t>(n) * a.top + i] = have ? log_p(value_of(sh.best[i])) : bad ? NAN : -INFINITY;
    }
  }
}

// ------------------------------------------------------------ backward
constexpr int kBwdThreads = 256, kBwdUnroll = 4;

struct BwdArgs {
  const float* lse;
  const float* dlogp;
  const float* entropy;
  const float* dentropy;
  const int32_t* top_ids;
  const float* dtop;
  long long out_stride;
  int pieces;  // blocks of a row
};

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Block (n, piece): a share of row n, and then the elements in it that are targets or alternatives.  8,192 rows of 32,768 bf16 with an
// entropy term: 161 us, 6.7 TB/s, a copy's rate; a row's logits are read and written once.
template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(kBwdThreads) logprob_bwd_kernel(LogprobArgs a, BwdArgs b, T* out) {
  constexpr int N = Vec<T>::N, LISTED = kMaxAlternatives + 1;
  __shared__ float grads[LISTED], values[LISTED];
  __shared__ int ids[LISTED];
  const int n = blockIdx.x / b.pieces, piece = blockIdx.x % b.pieces;
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(n) * a.stride;
  T* y = out + static_cast<size_t>(n) * b.out_stride;
  // whole vectors need rows that are aligned alike; the ends of the row are the first block's
  const bool alike = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
  const int lead = alike ? min(a.V, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / sizeof(T))) : 0;
  const int step = alike ? N : 1, groups = (a.V - lead) / step, tail = lead + groups * step;
  const int share = (groups + b.pieces - 1) / b.pieces, v0 = min(groups, piece * share), v1 = min(groups, v0 + share);
  const auto here = [&](int j) { return (j >= lead + v0 * step && j < lead + v1 * step) || (piece == 0 && (j < lead || j >= tail)); };

  for (int i = threadIdx.x; i <= a.top; i += kBwdThreads) {
    long long id = i < a.top ? b.top_ids[static_cast<size_t>(n) * a.top + i] : b.dlogp ? target_at(a, n) : -1;
    if (id < 0 || id >= a.V) id = -1;
    ids[i] = static_cast<int>(id);
    grads[i] = id < 0 ? 0.f : i < a.top ? b.dtop[static_cast<size_t>(n) * a.top + i] : b.dlogp[n];
    values[i] = id >= 0 && here(ids[i]) ? to_f(x[id]) : 0.f;  // before it is written: out may be the logits
  }
  __syncthreads();
  float total = 0.f;
  bool any = false;
  for (int i = 0; i <= a.top; ++i) total += grads[i], any |= grads[i] != 0.f;
  const float h = ENTROPY ? b.dentropy[n] : 0.f, H = ENTROPY && h != 0.f ? b.entropy[n] : 0.f, l = b.lse[n];
  const bool zero = !(any || h != 0.f) || l == -INFINITY;
  // scale (-p (total + h (log p + H))) = p (c0 + c1 log p)
  const float c0 = -a.scale * (total + h * H), c1 = -a.scale * h;
  const auto each = [&](float v) {
    const float lp = fmaf(v, a.scale, -l), p = exp2_fast(lp * kLog2e);
    return ENTROPY ? p * fmaf(c1, fmaxf(lp, -200.f), c0) : p * c0;  // p = 0 at -inf
  };

  if (piece == 0)
    for (int k = threadIdx.x; k < lead + a.V - tail; k += kBwdThreads) {
      const int j = k < lead ? k : tail + k - lead;
      put(y + j, zero ? 0.f : each(to_f(x[j])));
    }
  if (alike) {
    const T* from = x + lead;
    T* to = y + lead;
    for (int v = v0; v < v1; v += kBwdThreads * kBwdUnroll) {
      Vec<T> u[kBwdUnroll];
      if (!zero) {
#pragma unroll
        for (int i = 0; i < kBwdUnroll; ++i) {
          const int at = v + i * kBwdThreads + threadIdx.x;
          if (at < v1) u[i] = load_vec(from + static_cast<size_t>(at) * N);
        }
      }
#pragma unroll
      for (int i = 0; i < kBwdUnroll; ++i) {
        const int at = v + i * kBwdThreads + threadIdx.x;
        if (at >= v1) continue;
        float e[N];
        if (!zero) u[i].get(e);
#pragma unroll
        for (int k = 0; k < N; ++k) e[k] = zero ? 0.f : each(e[k]);
        u[i].set(e);
        *reinterpret_cast<uint4*>(to + static_cast<size_t>(at) * N) = u[i].u;
      }
    }
  } else {
#pragma unroll 4
    for (int j = v0 + threadIdx.x; j < v1; j += kBwdThreads) put(y + j, zero ? 0.f : each(to_f(x[j])));
  }
  if (zero) return;
  __syncthreads();
  for (int i = threadIdx.x; i <= a.top; i += kBwdThreads) {
    const int j = ids[i];
    if (j < 0 || !here(j)) continue;
    float sum = 0.f;
    bool again = false;  // the first of equal ids writes
    for (int k = 0; k <= a.top; ++k) {
      sum += ids[k] == j ? grads[k] : 0.f;
      again |= k < i && ids[k] == j;
    }
    if (!again) put(y + j, fmaf(a.scale, sum, each(values[i])));
  }
}

template <typename T>
int fwd(const LogprobArgs& a, float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, int num_sms, const DevCtl& ctl,
        cudaStream_t st) {
  // four blocks fit an SM; a share below 4,096 elements is not worth a block
  int blocks = 1;
  while (blocks < kMostBlocks && 2ll * a.N * blocks <= 4ll * num_sms && a.V / (2 * blocks) >= 4096) blocks *= 2;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(static_cast<unsigned>(a.N) * blocks), config.blockDim = dim3(kThreads), config.stream = st;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = blocks, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  config.attrs = &attr, config.numAttrs = 1;
  const cudaError_t rc = a.top ? cudaLaunchKernelEx(&config, logprob_fwd_kernel<T, true>, a, logp, entropy, lse, top_logp, top_ids, ctl)
                               : cudaLaunchKernelEx(&config, logprob_fwd_kernel<T, false>, a, logp, entropy, lse, top_logp, top_ids, ctl);
  return rc == cudaSuccess ? 1 : -1;
}

template <typename T>
int bwd(const LogprobArgs& a, const BwdArgs& b, T* out, cudaStream_t st) {
  const unsigned grid = static_cast<unsigned>(a.N) * b.pieces;
  if (b.dentropy)
    logprob_bwd_kernel<T, true><<<grid, kBwdThreads, 0, st>>>(a, b, out);
  else
    logprob_bwd_kernel<T, false><<<grid, kBwdThreads, 0, st>>>(a, b, out);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace

int logprob_fwd(const LogprobArgs& a, float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, bool bf16, int num_sms,
                const DevCtl& ctl, cudaStream_t st) {
  return bf16 ? fwd<__nv_bfloat16>(a, logp, entropy, lse, top_logp, top_ids, num_sms, ctl, st)
              : fwd<float>(a, logp, entropy, lse, top_logp, top_ids, num_sms, ctl, st);
}

int logprob_bwd(const LogprobArgs& a, const float* lse, const float* dlogp, const float* entropy, const float* dentropy, const int32_t* top_ids,
                const float* dtop, void* dlogits, long long out_stride, bool bf16, int num_sms, cudaStream_t st) {
  // eight blocks fit an SM: four waves of them, shares of at least two rounds of a block's loads
  const int elems = kBwdThreads * kBwdUnroll * (bf16 ? 8 : 4);
  int pieces = 1;
  while (static_cast<long long>(a.N) * pieces < 32ll * num_sms && a.V / (2 * pieces) >= elems) pieces *= 2;
  const BwdArgs b{lse, dlogp, entropy, dentropy, top_ids, dtop, out_stride, pieces};
  return bf16 ? bwd(a, b, static_cast<__nv_bfloat16*>(dlogits), st) : bwd(a, b, static_cast<float*>(dlogits), st);
}

}  // namespace topk
