// embed.cu -- the embedding lookup and its gradient.
//
// Lookup: a warp for each token's row, sixteen bytes a lane where rows are aligned to them.  Memory bounds it.
//
// Gradient: a row of it is the sum of dy over the tokens with its id, and a few ids have most of the tokens.  The tokens are
// sorted by id, stably, so that a row's terms lie together in the order of the tokens; the sorted list is cut into runs
// of kRun tokens whatever their ids, and a warp adds up a run, a slice of columns each.  Ids that lie in one run are
// written by its warp, those that its edges cut are put together by the block over its eight runs, and those that a
// block's edges cut go to scratch (its first and its last id), where embed_join_kernel adds their parts up in order:
// every sum is always formed in the same order.
//
// The sort is least digit first over the bits that ids have, by one cluster of CTAs: each has a share of the tokens, counts
// digits, learns from the others' shared memory where its tokens go, and places them.  That is latency, a few
// microseconds a digit; the other SMs write the zeros of rows without a token meanwhile, in the same launch.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "kernels.h"

namespace cg = cooperative_groups;

namespace topk {

namespace {

__device__ __forceinline__ long long id_at(const void* ids, bool wide, int n) {
  return wide ? __ldg(static_cast<const long long*>(ids) + n) : __ldg(static_cast<const int*>(ids) + n);
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// E neighbouring elements, loaded and stored as one access.
template <typename T, int E>
struct Pack {
  using Raw = std::conditional_t<sizeof(T) * E == 16, uint4,
                                 std::conditional_t<sizeof(T) * E == 8, uint2, std::conditional_t<sizeof(T) * E == 4, uint32_t, uint16_t>>>;
  Raw raw;
  __device__ __forceinline__ float get(int e) const {
    const T* x = reinterpret_cast<const T*>(&raw);
    return to_f(x[e]);
  }
  __device__ __forceinline__ void set(int e, float v) { put(reinterpret_cast<T*>(&raw) + e, v); }
};

template <typename T, int E>
__device__ __forceinline__ Pack<T, E> load_pack(const T* p) {
  Pack<T, E> r;
  r.raw = __ldg(reinterpret_cast<const typename Pack<T, E>::Raw*>(p));
  return r;
}

// ------------------------------------------------------------ lookup
constexpr int kFwdThreads = 256;

// Unit u: the token u / parts and the part u % parts of its row, a warp each.  65,536 tokens of 1,280 bf16 take 38 us, 86 % of what
// their rows, read once and written, take at a copy's rate; with one load of a lane under way 119.
template <typename T, int E>
__global__ void __launch_bounds__(kFwdThreads) embed_fwd_kernel(EmbedArgs a, const T* __restrict__ weight, T* __restrict__ out, int parts, DevCtl ctl) {
  constexpr int FLIGHT = 5;  // loads of a lane under way
  const int lane = threadIdx.x % 32, packs = a.D / E, each = (packs + parts - 1) / parts;
  const long long units = static_cast<long long>(a.N) * parts, stride = static_cast<long long>(gridDim.x) * (kFwdThreads / 32);
  for (long long u = static_cast<long long>(blockIdx.x) * (kFwdThreads / 32) + threadIdx.x / 32; u < units; u += stride) {
    const int n = static_cast<int>(u / parts), part = static_cast<int>(u % parts);
    const long long id = id_at(a.ids, a.ids64, n);
    const bool real = id >= 0 && id < a.rows;
    if (id >= a.rows && lane == 0) atomicOr(ctl.error, kDevErrRange);
    const T* from = weight + (real ? id : 0) * a.D;
    T* to = out + static_cast<size_t>(n) * a.D;
    for (int c0 = part * each + lane, end = min(packs, (part + 1) * each); c0 < end; c0 += 32 * FLIGHT) {
      Pack<T, E> x[FLIGHT];
#pragma unroll
      for (int i = 0; i < FLIGHT; ++i)
        if (c0 + 32 * i < end && real) x[i] = load_pack<T, E>(from + static_cast<size_t>(c0 + 32 * i) * E);
#pragma unroll
      for (int i = 0; i < FLIGHT; ++i) {
        if (c0 + 32 * i >= end) continue;
        if (!real) {
          x[i].raw = typename Pack<T, E>::Raw{};
        } else if (a.scale != 1.f) {
#pragma unroll
          for (int e = 0; e < E; ++e) x[i].set(e, x[i].get(e) * a.scale);
        }
        *reinterpret_cast<typename Pack<T, E>::Raw*>(to + static_cast<size_t>(c0 + 32 * i) * E) = x[i].raw;
      }
    }
  }
}

// ------------------------------------------------------------ sorting the tokens
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kSortBlocks = 16;  // of the cluster at most
constexpr int kPortable = 8;     // blocks that every device places as a cluster
constexpr int kDigitBits = 9, kDigits = 1 << kDigitBits;  // two digits for tables of up to 262,143 rows
static_assert(kDigits == kSortThreads, "a digit for each thread");

constexpr int kSmall = 1024;  // tokens that one block sorts by comparing them

struct Scratch {
  uint2* a;     // (id, token), sorted; tokens without an id in the table have that of the row behind it
  uint2* b;
  float* parts; // [pieces][2][D]
};

constexpr int kRun = 16, kSumWarps = 8, kPiece = kRun * kSumWarps;  // sorted tokens that a warp and a block add up
int pieces_of(int N) { return (N + kPiece - 1) / kPiece; }

struct SortShared {
  unsigned count[kSortWarps][kDigits];  // of each warp's tokens, then where they go
  unsigned total[kDigits];              // of the block
  unsigned first[kDigits];              // where the block's tokens of a digit go
  unsigned scan[kSortWarps];
};

// One digit of the cluster's sort: tokens [n0, n1) of `from` (or the ids themselves) into `to`.
template <typename Get>
__device__ void sort_digit(cg::cluster_group& cluster, SortShared& sh, Get get, uint2* to, int n0, int n1, int shift) {
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, blocks = cluster.num_blocks(), rank = cluster.block_rank();
  for (int i = threadIdx.x; i < kSortWarps * kDigits; i += kSortThreads) (&sh.count[0][0])[i] = 0;
  __syncthreads();
  // each warp has a share of its own, in order: places within it follow the tokens
  const int each = ((n1 - n0 + kSortWarps - 1) / kSortWarps + 31) / 32 * 32, w0 = min(n1, n0 + warp * each), w1 = min(n1, w0 + each);
  constexpr int AHEAD = 8;  // a lane's tokens under way: their loads are what the sort waits for
  uint2 x[AHEAD];
  const auto fetch = [&](int i0) {
#pragma unroll
    for (int k = 0; k < AHEAD; ++k)
      if (i0 + 32 * k + lane < w1) x[k] = get(i0 + 32 * k + lane);
  };
  for (int i0 = w0; i0 < w1; i0 += 32 * AHEAD) {
    fetch(i0);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (i0 + 32 * k < w1) {
        const bool in = i0 + 32 * k + lane < w1;
        const unsigned digit = in ? x[k].x >> shift & (kDigits - 1) : kDigits;
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        if (in && (same & ((1u << lane) - 1u)) == 0) sh.count[warp][digit] += __popc(same);  // the first of its kind
        __syncwarp();
      }
    }
  }
  __syncthreads();
  {
    const int d = threadIdx.x;
    unsigned c[kSortWarps], sum = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) c[w] = sh.count[w][d];
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      sh.count[w][d] = sum;
      sum += c[w];
    }
    sh.total[d] = sum;
  }
  cluster.sync();
  // where a digit begins: all smaller digits' tokens, and the earlier blocks' of its own
  unsigned mine = 0, all = 0, got[kSortBlocks];
#pragma unroll
  for (int b = 0; b < kSortBlocks; ++b) got[b] = b < blocks ? cluster.map_shared_rank(&sh, b)->total[threadIdx.x] : 0;
#pragma unroll
  for (int b = 0; b < kSortBlocks; ++b) {
    mine += b < rank ? got[b] : 0;
    all += got[b];
  }
  unsigned upto = all;
  for (int o = 1; o < 32; o *= 2) {
    const unsigned x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) sh.scan[warp] = upto;
  __syncthreads();
  unsigned before = 0;
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) before += w < warp ? sh.scan[w] : 0;
  sh.first[threadIdx.x] = before + upto - all + mine;
  __syncthreads();
  for (int i0 = w0; i0 < w1; i0 += 32 * AHEAD) {
    if (w1 - w0 > 32 * AHEAD) fetch(i0);  // else they are there
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (i0 + 32 * k < w1) {
        const bool in = i0 + 32 * k + lane < w1;
        const unsigned digit = in ? x[k].x >> shift & (kDigits - 1) : kDigits;
        const unsigned same = __match_any_sync(0xffffffffu, digit), ahead = __popc(same & ((1u << lane) - 1u));
        unsigned base = 0;
        if (in) base = sh.count[warp][digit];
        __syncwarp();
        if (in) {
          if (ahead == 0) sh.count[warp][digit] = base + __popc(same);
          to[sh.first[digit] + base + ahead] = x[k];
        }
        __syncwarp();
      }
    }
  }
  __threadfence();
  cluster.sync();  // the placed tokens are there, and no block's counts are read any more
}

// 32,768 tokens and 32,768 rows (two digits): 19 us, in which the others write 50 MB of zeros; it is the wait for a few loads and
// cluster barriers a digit.  The first cluster sorts; the other blocks write zeros (into dw where it is to be written, [bytes16] of 16 bytes and a tail).
__global__ void __launch_bounds__(kSortThreads, 1)
    embed_sort_kernel(EmbedArgs a, Scratch s, int passes, int sorters, uint4* zero, long long bytes16, int tail_bytes, DevCtl ctl) {
  __shared__ alignas(16) SortShared sh;
  cg::cluster_group cluster = cg::this_cluster();
  if (static_cast<int>(blockIdx.x) >= sorters) {
    const long long at = static_cast<long long>(blockIdx.x - sorters) * kSortThreads + threadIdx.x,
                    stride = static_cast<long long>(gridDim.x - sorters) * kSortThreads;
    for (long long i = at; i < bytes16; i += stride) zero[i] = make_uint4(0u, 0u, 0u, 0u);
    if (at < tail_bytes) reinterpret_cast<uint8_t*>(zero + bytes16)[at] = 0;
    return;
  }
  const int rank = blockIdx.x;
  const int each = (a.N + sorters - 1) / sorters, n0 = min(a.N, rank * each), n1 = min(a.N, n0 + each);
  const unsigned none = static_cast<unsigned>(a.rows);  // the id of tokens without one: behind all others
  const auto token = [&](int i) {
    const long long id = id_at(a.ids, a.ids64, i);
    if (id >= a.rows) atomicOr(ctl.error, kDevErrRange);
    return make_uint2(id >= 0 && id < a.rows ? static_cast<unsigned>(id) : none, static_cast<unsigned>(i));
  };
  if (a.N <= kSmall) {
    // a few tokens: one block sorts (id, token) as numbers in shared memory
    unsigned long long* keys = reinterpret_cast<unsigned long long*>(&sh);
    int pow2 = 2;
    while (pow2 < a.N) pow2 *= 2;
    for (int i = threadIdx.x; i < pow2; i += kSortThreads) {
      const uint2 t = i < a.N ? token(i) : make_uint2(~0u, ~0u);
      keys[i] = static_cast<unsigned long long>(t.x) << 32 | t.y;
    }
    __syncthreads();
    for (int size = 2; size <= pow2; size *= 2)
      for (int step = size / 2; step; step /= 2) {
        for (int i = threadIdx.x; i < pow2 / 2; i += kSortThreads) {
          const int lo = (i / step) * 2 * step + i % step, hi = lo + step;
          const unsigned long long x = keys[lo], y = keys[hi];
          if ((x > y) == ((lo & size) == 0)) keys[lo] = y, keys[hi] = x;
        }
        __syncthreads();
      }
    for (int i = threadIdx.x; i < a.N; i += kSortThreads) s.a[i] = make_uint2(static_cast<unsigned>(keys[i] >> 32), static_cast<unsigned>(keys[i]));
    return;
  }
  uint2 *from = s.b, *to = s.a;
  if (passes % 2 == 0) {
    uint2* t = from;
    from = to, to = t;
  }
  for (int p = 0; p < passes; ++p) {
    if (p == 0)
      sort_digit(cluster, sh, token, to, n0, n1, 0);
    else
      sort_digit(cluster, sh, [&](int i) { return __ldcg(from + i); }, to, n0, n1, p * kDigitBits);
    uint2* t = from;
    from = to, to = t;
  }
}

// ------------------------------------------------------------ adding up
struct SumArgs {
  int N, rows, D, parts;  // parts: of a row's columns
  float scale;
};

// An id's finished sum of E columns, added to `old` where there is something.
template <typename G, int E, bool ACC>
__device__ __forceinline__ void finish(G* at, const float (&sum)[E], const SumArgs& a, const Pack<G, E>& old) {
  Pack<G, E> now;
#pragma unroll
  for (int e = 0; e < E; ++e) now.set(e, ACC ? fmaf(sum[e], a.scale, old.get(e)) : sum[e] * a.scale);
  *reinterpret_cast<typename Pack<G, E>::Raw*>(at) = now.raw;
}
template <typename G, int E>
__device__ __forceinline__ Pack<G, E> old_of(const G* at) {
  return *reinterpret_cast<const Pack<G, E>*>(at);
}

// A block: a piece of eight runs, 32 E columns; a warp for each run.  32,768 tokens of 768 bf16: 16 us, 3.1 TB/s of dy, a token's
// row in three pieces of 512 bytes by three blocks.  Four blocks an SM (64 registers) take 3 us less than fewer.
template <typename T, typename G, int E, bool ACC>
__global__ void __launch_bounds__(32 * kSumWarps, ACC ? 2 : 4) embed_sum_kernel(SumArgs a, Scratch s, const T* __restrict__ dy, G* __restrict__ dw) {
  constexpr int FLIGHT = 8;
  // the sums of a run's first and last id, where the run's edges cut them (head alone where the run is all of one id)
  __shared__ float head[kSumWarps][E][32], tail[kSumWarps][E][32];
  __shared__ unsigned tail_id[kSumWarps];
  __shared__ int state[kSumWarps];  // kFront: the first id began before; kBack: the last one goes on; kOne: they are the same
  constexpr int kFront = 1, kBack = 2, kOne = 4;
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, piece = blockIdx.x / a.parts;
  const int c = (blockIdx.x % a.parts * 32 + lane) * E;
  const bool in = c < a.D;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int i0 = piece * kPiece + warp * kRun, end = min(kRun, a.N - i0);
  const uint2 mine = lane < end ? __ldcg(s.a + i0 + lane) : make_uint2(~0u, 0u);
  const unsigned before = i0 > 0 && end > 0 ? __ldcg(&s.a[i0 - 1].x) : ~0u, after = i0 + kRun < a.N ? __ldcg(&s.a[i0 + kRun].x) : ~0u;
  const int n = __popc(__ballot_sync(0xffffffffu, mine.x < static_cast<unsigned>(a.rows)));  // those with an id come first
  if (n > 0) {
    float sum[E] = {};
    bool first = true;
    int flags = 0;
    for (int k0 = 0; k0 < n; k0 += FLIGHT) {
      Pack<T, E> x[FLIGHT];
      Pack<G, E> old[FLIGHT];
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        const unsigned token = __shfl_sync(0xffffffffu, mine.y, k0 + k), id = __shfl_sync(0xffffffffu, mine.x, k0 + k);
        const unsigned next = __shfl_sync(0xffffffffu, mine.x, (k0 + k + 1) & 31);
        if (k0 + k >= n || !in) continue;
        x[k] = load_pack<T, E>(dy + static_cast<size_t>(token) * a.D + c);
        if (ACC && (k0 + k + 1 == n || next != id)) old[k] = old_of<G, E>(dw + static_cast<size_t>(id) * a.D + c);
      }
#pragma unroll
      for (int k = 0; k < FLIGHT; ++k) {
        if (k0 + k >= n) continue;
        const unsigned id = __shfl_sync(0xffffffffu, mine.x, k0 + k);
        const unsigned next = k0 + k + 1 < n ? __shfl_sync(0xffffffffu, mine.x, (k0 + k + 1) & 31) : after;  // `after` of a whole run
        const bool last = k0 + k + 1 == n;
        if (in) {
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] += x[k].get(e);
        }
        if (!last && next == id) continue;
        // the id's tokens in this run end here
        const bool front = first && id == before, back = last && id == after;
        if (front || back) {
          float(*to)[32] = first ? head[warp] : tail[warp];
#pragma unroll
          for (int e = 0; e < E; ++e) to[e][lane] = sum[e];
          flags |= (front ? kFront : 0) | (back ? kBack : 0);
          if (back && lane == 0) tail_id[warp] = id;
        } else if (in) {
          finish<G, E, ACC>(dw + static_cast<size_t>(id) * a.D + c, sum, a, old[k]);
        }
        if (first && last) flags |= kOne;
        first = false;
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = 0.f;
      }
    }
    if (lane == 0) state[warp] = flags;
  } else if (lane == 0) {
    state[warp] = 0;
  }
  __syncthreads();
  if (n <= 0 || !in) return;
  // what begins in this run and goes on, and, by the first warp, what came in from the piece before
  const int own = state[warp];
#pragma unroll
  for (int turn = 0; turn < 2; ++turn) {
    const bool incoming = turn == 0;
    if (incoming ? warp != 0 || !(own & kFront) : !(own & kBack) || ((own & kOne) && (own & kFront))) continue;
    const bool from_tail = !incoming && !(own & kOne);
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = from_tail ? tail[warp][e][lane] : head[warp][e][lane];
    bool open = incoming ? (own & kOne) && (own & kBack) : true;
    for (int v = warp + 1; v < kSumWarps && open; ++v) {
      const int st = state[v];
      if (!(st & kFront)) break;  // nothing there: the piece ends before, and `open` stays
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += head[v][e][lane];
      open = (st & kOne) && (st & kBack);
    }
    if (open || incoming) {
      float* to = s.parts + (static_cast<size_t>(piece) * 2 + (incoming ? 0 : 1)) * a.D + c;
#pragma unroll
      for (int e = 0; e < E; ++e) to[e] = sum[e];
    } else {
      G* at = dw + static_cast<size_t>(tail_id[warp]) * a.D + c;
      Pack<G, E> old;
      if (ACC) old = old_of<G, E>(at);
      finish<G, E, ACC>(at, sum, a, old);
    }
  }
}

// A block for each piece whose last id goes on in the next one and begins in it: it adds up that id's parts, eight shares of them by
// its warps, and the shares in order.
template <typename G, int E, bool ACC>
__global__ void __launch_bounds__(32 * kSumWarps) embed_join_kernel(SumArgs a, Scratch s, G* __restrict__ dw) {
  __shared__ float share[kSumWarps][E][32];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, piece = blockIdx.x / a.parts;
  const int c = (blockIdx.x % a.parts * 32 + lane) * E;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int i0 = piece * kPiece, next = i0 + kPiece;
  if (next >= a.N) return;
  const unsigned id = __ldcg(&s.a[next - 1].x), then = __ldcg(&s.a[next].x), before = i0 > 0 ? __ldcg(&s.a[i0 - 1].x) : ~0u;
  if (id >= static_cast<unsigned>(a.rows) || then != id || before == id) return;  // it ends here, or began before
  int lo = piece + 1, hi = (a.N - 1) / kPiece;                                     // the last piece that begins with it
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (__ldcg(&s.a[static_cast<size_t>(mid) * kPiece].x) == id)
      lo = mid;
    else
      hi = mid - 1;
  }
  const bool in = c < a.D;
  // its parts: the second one of the piece where it begins, the first ones of those after
  const int count = lo - piece + 1, each = (count + kSumWarps - 1) / kSumWarps, k0 = warp * each, k1 = min(count, k0 + each);
  float sum[E] = {};
  if (in)
#pragma unroll 4
    for (int k = k0; k < k1; ++k) {
      const float* p = s.parts + (static_cast<size_t>(piece + k) * 2 + (k == 0 ? 1 : 0)) * a.D + c;
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += __ldcg(p + e);  // written while this kernel waited
    }
#pragma unroll
  for (int e = 0; e < E; ++e) share[warp][e][lane] = sum[e];
  __syncthreads();
  if (warp != 0 || !in) return;
  G* at = dw + static_cast<size_t>(id) * a.D + c;
  Pack<G, E> old;
  if (ACC) old = old_of<G, E>(at);
  for (int w = 1; w < kSumWarps; ++w) {
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] += share[w][e][lane];
  }
  finish<G, E, ACC>(at, sum, a, old);
}

// Elements of an access: the most that divide a row and fill sixteen bytes at the wider type.
int pack_of(int D, size_t narrow_bytes) {
  int e = static_cast<int>(16 / narrow_bytes);
  while (D % e) e /= 2;
  return e;
}

template <typename T>
int fwd(const EmbedArgs& a, const T* weight, T* out, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  const int e = pack_of(a.D, sizeof(T)), packs = a.D / e;
  // few tokens: a row is shared out over warps, one load a lane
  int parts = 1;
  while (static_cast<long long>(a.N) * parts < 16ll * num_sms && packs > 32 * parts) ++parts;
  const long long units = static_cast<long long>(a.N) * parts, warps = kFwdThreads / 32;
  const long long want = (units + warps - 1) / warps, most = 8ll * num_sms;
  const unsigned grid = static_cast<unsigned>(want < most ? want : most);
  switch (e) {
    case 8:
      if constexpr (sizeof(T) == 2) embed_fwd_kernel<T, 8><<<grid, kFwdThreads, 0, st>>>(a, weight, out, parts, ctl);
      break;
    case 4: embed_fwd_kernel<T, 4><<<grid, kFwdThreads, 0, st>>>(a, weight, out, parts, ctl); break;
    case 2: embed_fwd_kernel<T, 2><<<grid, kFwdThreads, 0, st>>>(a, weight, out, parts, ctl); break;
    default: embed_fwd_kernel<T, 1><<<grid, kFwdThreads, 0, st>>>(a, weight, out, parts, ctl);
  }
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

// Launches a kernel whose blocks may begin while the one before ends (they wait for its memory themselves).
template <typename Kernel, typename... Args>
bool launch_early(Kernel kernel, unsigned grid, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(grid), config.blockDim = dim3(32 * kSumWarps), config.stream = st;
  cudaLaunchAttribute early = {};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  config.attrs = &early, config.numAttrs = 1;
  return cudaLaunchKernelEx(&config, kernel, args...) == cudaSuccess;
}

template <typename T, typename G, int E, bool ACC>
int sums(SumArgs p, const Scratch& s, const T* dy, G* dw, cudaStream_t st) {
  p.parts = (p.D / E + 31) / 32;
  const unsigned grid = static_cast<unsigned>(pieces_of(p.N)) * p.parts;
  if (!launch_early(embed_sum_kernel<T, G, E, ACC>, grid, st, p, s, dy, dw)) return -1;
  if (p.N <= kPiece) return 1;
  return launch_early(embed_join_kernel<G, E, ACC>, grid, st, p, s, dw) ? 2 : -1;
}

template <typename T, typename G>
int sums_of(const SumArgs& p, const Scratch& s, const void* dy, void* dw, bool accumulate, cudaStream_t st) {
  const T* x = static_cast<const T*>(dy);
  G* y = static_cast<G*>(dw);
  const auto of = [&](auto acc) {
    constexpr bool ACC = decltype(acc)::value;
    switch (pack_of(p.D, sizeof(T) > sizeof(G) ? sizeof(T) : sizeof(G))) {
      case 8:
        if constexpr (sizeof(T) == 2 && sizeof(G) == 2) return sums<T, G, 8, ACC>(p, s, x, y, st);
        return -1;
      case 4: return sums<T, G, 4, ACC>(p, s, x, y, st);
      case 2: return sums<T, G, 2, ACC>(p, s, x, y, st);
      default: return sums<T, G, 1, ACC>(p, s, x, y, st);
    }
  };
  return accumulate ? of(std::true_type{}) : of(std::false_type{});
}

// Blocks of the sort's cluster at most: as many as the current device can place at once, which beyond the portable size is not given
// (a part of a GPU may have fewer SMs side by side); asked once for each device.  Eight in place of sixteen take 41 us in place of 35 for 32,768
// tokens of 768.  0: an error.
int most_sorters() {
  static std::atomic<unsigned long long> known{0}, wide{0};
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess) return 0;
  if (device <= 63 && known.load(std::memory_order_acquire) >> device & 1ull)
    return wide.load(std::memory_order_relaxed) >> device & 1ull ? kSortBlocks : kPortable;
  if (cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return 0;
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(kSortBlocks), config.blockDim = dim3(kSortThreads);
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kSortBlocks, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  config.attrs = &attr, config.numAttrs = 1;
  int clusters = 0;
  if (cudaOccupancyMaxActiveClusters(&clusters, embed_sort_kernel, &config) != cudaSuccess) {
    clusters = 0;
    (void)cudaGetLastError();  // the next launch is not to blame for it
  }
  if (device <= 63) {
    if (clusters > 0) wide.fetch_or(1ull << device, std::memory_order_relaxed);
    known.fetch_or(1ull << device, std::memory_order_release);
  }
  return clusters > 0 ? kSortBlocks : kPortable;
}

size_t align256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

int embed_fwd(const EmbedArgs& a, const void* weight, void* out, bool bf16, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  return bf16 ? fwd(a, static_cast<const __nv_bfloat16*>(weight), static_cast<__nv_bfloat16*>(out), num_sms, ctl, st)
              : fwd(a, static_cast<const float*>(weight), static_cast<float*>(out), num_sms, ctl, st);
}

size_t embed_bwd_workspace_bytes(int N, int, int D) {
  return 2 * align256(static_cast<size_t>(N) * sizeof(uint2)) + static_cast<size_t>(pieces_of(N)) * 2 * D * sizeof(float);
}

int embed_bwd(const EmbedArgs& a, const void* dy, void* dweight, bool accumulate, bool bf16, bool grad_bf16, void* workspace, int num_sms,
              const DevCtl& ctl, cudaStream_t st) {
  uint8_t* at = static_cast<uint8_t*>(workspace);
  Scratch s;
  s.a = reinterpret_cast<uint2*>(at);
  s.b = reinterpret_cast<uint2*>(at + align256(static_cast<size_t>(a.N) * sizeof(uint2)));
  s.parts = reinterpret_cast<float*>(at + 2 * align256(static_cast<size_t>(a.N) * sizeof(uint2)));
  int passes = 1;
  while (passes * kDigitBits < 31 && a.rows >> (passes * kDigitBits)) ++passes;  // ids up to `rows` itself
  const long long bytes = accumulate ? 0 : static_cast<long long>(a.rows) * a.D * (grad_bf16 ? 2 : 4);
  // a sorter for every thousand tokens; the others fill the GPU where there are zeros to write
  int sorters = 1;
  while (sorters < kSortBlocks && a.N > 1024 * sorters) sorters *= 2;
  if (sorters > kPortable) {
    const int most = most_sorters();
    if (most <= 0) return -1;
    sorters = sorters < most ? sorters : most;
  }
  // one cluster of them at least, however few SMs there are: they wait for nothing
  const long long zeroers = bytes ? (bytes / 16 + 4 * kSortThreads) / (4 * kSortThreads) : 0, most = num_sms - sorters > sorters ? num_sms - sorters : sorters;
  const int grid = sorters + static_cast<int>((zeroers < most ? zeroers + sorters - 1 : most) / sorters * sorters);
  cudaLaunchConfig_t config = {};
  config.gridDim = dim3(grid), config.blockDim = dim3(kSortThreads), config.stream = st;
  cudaLaunchAttribute attr = {};
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = sorters, attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  config.attrs = &attr, config.numAttrs = 1;
  if (cudaLaunchKernelEx(&config, embed_sort_kernel, a, s, passes, sorters, static_cast<uint4*>(dweight), bytes / 16, static_cast<int>(bytes % 16), ctl) !=
      cudaSuccess)
    return -1;
  const SumArgs p{a.N, a.rows, a.D, 1, a.scale};
  const int n = bf16 ? (grad_bf16 ? sums_of<__nv_bfloat16, __nv_bfloat16>(p, s, dy, dweight, accumulate, st) : sums_of<__nv_bfloat16, float>(p, s, dy, dweight, accumulate, st))
                     : (grad_bf16 ? sums_of<float, __nv_bfloat16>(p, s, dy, dweight, accumulate, st) : sums_of<float, float>(p, s, dy, dweight, accumulate, st));
  return n < 0 ? -1 : 1 + n;
}

}  // namespace topk
