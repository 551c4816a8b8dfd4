// linear.cu -- the linear layer y = act(x W^T + b) + r and its backward pass, on
// the tensor cores.
//
// Three products of one form, D[m, n] = sum_k A(m, k) B(n, k), bf16 operands and fp32
// sums in TMEM:
//   forward  D = y  [M, N]: A = x (k contiguous),           B = W (k contiguous)
//   dx = dz W       [M, K]: A = dz (n, the sum, contiguous), B = W read across its rows
//   dW = dz^T x     [N, K]: A = dz and B = x read across their rows
// An operand whose sum index is contiguous is staged K-major, the other kind MN-major
// (64 x 64 boxes, 128-byte swizzle; the instruction transposes), so no transposed copy
// is ever made.  dz = dy act'(z) is formed once, as bf16 (its one rounding: the tensor
// cores take bf16), by a kernel that also adds up db.
//
// linear_mma_kernel is persistent, one CTA per SM: a TMA warp, an MMA warp that feeds
// 128 x BN tiles into one of two TMEM accumulators, and eight epilogue warps that read
// the other one: bias, activation and residual are applied to the fp32 sums, rounded
// once, staged in shared memory and stored by TMA, which clips ragged edges.  Few tiles
// and a long sum (dW, a few hundred tokens) are split along the sum: each part writes
// fp32 partial tiles, and linear_join_kernel adds them in a fixed order with the same
// epilogue.  A few tokens (decoding) go to linear_few_kernel, which is
// bound by reading W once.
#include <cuda_bf16.h>

#include <type_traits>

#include "kernels.h"

namespace topk {

namespace {

constexpr int BM = 128, BK = 64;
constexpr int kEpiWarps = 8;
constexpr int kThreads = 64 + 32 * kEpiWarps;

// CTAS = 2: two CTAs of a cluster (a pair of SMs) work on one 256 x BN tile.  Each stages its 128 rows of A and its
// half of B's rows, the pair's first CTA issues the products for both, and each ends up with its
// 128 x BN accumulator: B is read from shared memory once for two SMs.
template <int CTAS, int BN>
struct Layout {
  static constexpr uint32_t A_BYTES = BM * BK * 2, B_BYTES = BN / CTAS * BK * 2;
  static constexpr uint32_t STAGE = A_BYTES + B_BYTES;
  static constexpr uint32_t EPI = 2 * 4096;  // a warp's two buffers of 32 rows of 128 bytes
  static constexpr int FIT = (232448 - 2048 - kEpiWarps * EPI) / STAGE;
  static constexpr int S = FIT > 6 ? 6 : FIT;
  static constexpr size_t OFF_EPI = static_cast<size_t>(S) * STAGE;
  static constexpr size_t OFF_BAR = OFF_EPI + kEpiWarps * EPI;
  static constexpr int NBARS = 2 * S + 5 + 2 * kEpiWarps;  // full/empty per stage, accumulator full/empty x 2, drain, residual
  static constexpr size_t BYTES = 1024 + OFF_BAR + NBARS * 8 + 16;
  static constexpr uint32_t TMEM_COLS = 2 * BN <= 256 ? 256 : 512;
  static_assert(BYTES <= 232448 && S >= 3, "shared memory");
  static_assert(STAGE % 1024 == 0, "swizzle atoms");
};

// ------------------------------------------------------------ pairs of CTAs
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}

__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// The address of the first CTA's barrier.
__device__ __forceinline__ uint32_t leader_bar(const uint64_t* bar) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_u32(bar)));
  return r;
}

__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Bounded wait (as common.cuh's mbar_wait) that also acquires what the other CTA of the pair released.
__device__ __forceinline__ bool try_wait_cluster(uint64_t* bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_u32(bar)), "r"(parity)
      : "memory");
  return ok != 0;
}

static __device__ __noinline__ bool wait_cluster_slow(uint64_t* bar, uint32_t parity, const DevCtl& ctl, volatile int* abort_flag) {
  const unsigned long long t0 = global_ns();
  for (uint32_t spin = 1;; ++spin) {
    if (try_wait_cluster(bar, parity)) return true;
    if ((spin & 63u) == 0u) {
      if (*abort_flag) return false;
      if (global_ns() - t0 > ctl.wait_limit_ns) {
        atomicOr(ctl.error, kDevErrTimeout);
        *abort_flag = 1;
        return false;
      }
    }
  }
}

// For what the other CTA's threads arrive on; loads and products complete on a barrier by themselves.
template <int CTAS>
__device__ __forceinline__ bool wait_arrivals(uint64_t* bar, uint32_t parity, const DevCtl& ctl, volatile int* abort_flag) {
  if constexpr (CTAS == 1) return mbar_wait(bar, parity, ctl, abort_flag);
  return try_wait_cluster(bar, parity) || wait_cluster_slow(bar, parity, ctl, abort_flag);
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const DevCtl& ctl, volatile int* abort_flag) {
  int ok = 0;
  if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity, ctl, abort_flag) ? 1 : 0;
  return __shfl_sync(0xffffffffu, ok, 0) != 0;
}

__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity, const DevCtl& ctl) {
  if (mbar_try_wait(bar, parity)) return;
  const unsigned long long t0 = global_ns();
  while (!mbar_try_wait(bar, parity)) {
    if (global_ns() - t0 > ctl.wait_limit_ns) {
      atomicOr(ctl.error, kDevErrTimeout);
      return;
    }
  }
}

template <int CTAS>
__device__ __forceinline__ void tmem_take(uint32_t* dst, uint32_t cols) {
  if constexpr (CTAS == 1) {
    tmem_alloc(dst, cols);
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}

template <int CTAS>
__device__ __forceinline__ void tmem_give(uint32_t addr, uint32_t cols) {
  if constexpr (CTAS == 1)
    tmem_dealloc(addr, cols);
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}

// `bar`: an address in the cluster's shared memory (the first CTA's barrier for a pair).
template <int CTAS>
__device__ __forceinline__ void load_box(void* dst, const void* map, uint32_t bar, int c0, int c1) {
  if constexpr (CTAS == 1)
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(0)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(
            smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(0)
        : "memory");
}

template <int CTAS>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  if constexpr (CTAS == 1)
    mma_bf16_ss(d, a, b, idesc, accumulate);
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Arrives on the barrier (of both CTAs of a pair) when all products issued so far are done.
template <int CTAS>
__device__ __forceinline__ void commit(uint64_t* bar) {
  if constexpr (CTAS == 1)
    mma_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
                 "h"(static_cast<uint16_t>(3))
                 : "memory");
}

// Arrives on this CTA's barrier alone.
template <int CTAS>
__device__ __forceinline__ void commit_here(uint64_t* bar) {
  if constexpr (CTAS == 1)
    mma_commit(bar);
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// MN-major tile of 64 x 64 boxes (128-byte rows of 64 MN elements, one row per k): 64-element
// blocks of MN are 8192 bytes apart, groups of eight k 1024.
__device__ __forceinline__ uint64_t sdesc_mn128(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(8192 >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}

__device__ __forceinline__ void tma_store_3d(const void* map, const void* smem, int c0, int c1, int c2) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(map)),
               "r"(smem_u32(smem)), "r"(c0), "r"(c1), "r"(c2)
               : "memory");
}

__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// Waits until all but the last PENDING groups have read their shared memory.
template <int PENDING>
__device__ __forceinline__ void bulk_wait_read() {
  asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
}
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ void unpack8(uint4 u, float (&v)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) v[2 * e] = __uint_as_float(w[e] << 16), v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
}

// The hardware's 2^x and 1 / x, to 2^-22; results below 2^-126 are zero.
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float rcp_fast(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ float sigmoid(float z) { return rcp_fast(1.f + exp2_fast(z * -1.44269504f)); }

// The normal distribution's Phi(z), within 6e-7 (the fit's 7.5e-8, roundings, the two instructions): with
// x = |z| / sqrt(2) and t = 1 / (1 + 0.3275911 x), erfc(x) = t (a1 + t (a2 + ..)) e^(-x^2) (Abramowitz and Stegun,
// 7.1.26); half of it is Phi(-|z|).  e = e^(-z^2/2).  Towards minus infinity the relative error grows: 1e-3 at -4.5,
// 3.7e-3 (half a bf16 place) at -6, 3.2e-2 at -12, where z Phi(z) is below 1e-8, 1e-31.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float t = rcp_fast(fabsf(z) * 0.23164188f + 1.f);
  e = exp2_fast(z * z * -0.72134752f);
  float q = fmaf(t, 0.5307027145f, -0.7265760135f);
  q = fmaf(t, q, 0.7107068705f);
  q = fmaf(t, q, -0.142248368f);
  q = fmaf(t, q, 0.127414796f);
  q = q * t * e;
  return z > 0.f ? 1.f - q : q;
}

__device__ __forceinline__ float act_of(float z, int act) {
  if (act == kActRelu) return z < 0.f ? 0.f : z;  // a NaN stays
  if (act == kActGelu) {
    float e;
    return z * normal_cdf(z, e);
  }
  if (act == kActSilu) return z * sigmoid(z);
  return z;
}

__device__ __forceinline__ float act_slope(float z, int act) {
  if (act == kActRelu) return z > 0.f ? 1.f : 0.f;
  if (act == kActGelu) {
    float e;
    const float phi = normal_cdf(z, e);
    return phi + z * 0.39894228f * e;
  }
  if (act == kActSilu) {
    const float s = sigmoid(z);
    return s * (1.f + z * (1.f - s));
  }
  return 1.f;
}

struct Epi {
  const __nv_bfloat16* bias;      // [N] or null
  const __nv_bfloat16* residual;  // [M][N] or null
  int act, keep;                  // keep: also store the pre-activations
};

// Work units: output tiles in bands of eight row tiles (neighbouring CTAs share rows of A and
// columns of B in L2), for each part of the sum.
struct Grid {
  int m_tiles, n_tiles, parts, k_blocks;
};

__device__ __forceinline__ void unit_of(const Grid& g, int u, int& mt, int& nt, int& part) {
  constexpr int kBand = 8;
  const int tiles = g.m_tiles * g.n_tiles;
  part = u / tiles;
  int t = u - part * tiles;
  const int band = t / (kBand * g.n_tiles);
  t -= band * kBand * g.n_tiles;
  const int rows = min(kBand, g.m_tiles - band * kBand);
  nt = t / rows;
  mt = band * kBand + t - nt * rows;
}

// 16384 x 2048 x 8192: 312 us (1.76 PFLOP/s, 89 % of measured; the tensor pipe alone takes 279), 8192^3 611 us.  What
// bounds it: an SM takes in 62.5 bytes a clock for products at full rate, of 65 that it can; for short sums the
// fill of the first tile and the epilogue of the last.
// Out: __nv_bfloat16 or float (the result, or a part's partial sums).
template <int CTAS, int BN, bool A_MN, bool B_MN, typename Out>
__global__ void __launch_bounds__(kThreads, 1)
    linear_mma_kernel(const __grid_constant__ CUtensorMap tma, const __grid_constant__ CUtensorMap tmb,
                      const __grid_constant__ CUtensorMap tmo, const __grid_constant__ CUtensorMap tmz,
                      const __grid_constant__ CUtensorMap tmr, Epi epi, Grid grid, int M, int N, DevCtl ctl) {
  using L = Layout<CTAS, BN>;
  constexpr int S = L::S, NB = BN / CTAS;  // NB: rows of B that a CTA stages
  constexpr uint32_t IDESC = idesc_bf16_f32(BM * CTAS, BN) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u);
  static_assert(!B_MN || NB % 64 == 0, "whole boxes of B");

  extern __shared__ uint8_t smem_raw[];
  // the same offset in both CTAs of a pair: their windows start alike
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* full = bars;                   // the first CTA's are used, for the loads of both
  uint64_t* empty = bars + S;
  uint64_t* acc_full = bars + 2 * S;       // [2]
  uint64_t* acc_empty = bars + 2 * S + 2;  // [2], the first CTA's are used
  uint64_t* drain = bars + 2 * S + 4;
  uint64_t* res_full = bars + 2 * S + 5;   // [warp][2]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + L::NBARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CTAS == 2 ? static_cast<int>(cluster_rank()) : 0;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(&acc_full[b], 1);
      mbar_init(&acc_empty[b], kEpiWarps * CTAS);
    }
    mbar_init(drain, 1);
    for (int b = 0; b < 2 * kEpiWarps; ++b) mbar_init(&res_full[b], 1);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_take<CTAS>(tmem_slot, L::TMEM_COLS);
  tc_fence_before();
  __syncthreads();
  if constexpr (CTAS == 2) cluster_sync();  // the other CTA's barriers are there
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int units = grid.m_tiles * grid.n_tiles * grid.parts;
  const int unit0 = blockIdx.x / CTAS, stride = gridDim.x / CTAS;
  auto k_first = [&](int part) { return static_cast<int>(static_cast<long long>(grid.k_blocks) * part / grid.parts); };

  if (warp == 0) {
    // ------------------------------------------------------------ loads
    if (lane == 0) {
      tma_prefetch_desc(&tma);
      tma_prefetch_desc(&tmb);
      uint32_t it = 0;
      bool ok = true;
      for (int u = unit0; ok && u < units; u += stride) {
        int mt, nt, part;
        unit_of(grid, u, mt, nt, part);
        const int row = (mt * CTAS + rank) * BM, col = nt * BN + rank * NB;
        for (int kb = k_first(part), end = k_first(part + 1); kb < end; ++kb, ++it) {
          const int s = it % S;
          if (!mbar_wait(&empty[s], ((it / S) & 1u) ^ 1u, ctl, abort_flag)) {
            ok = false;
            break;
          }
          uint8_t* a = smem + static_cast<size_t>(s) * L::STAGE;
          uint8_t* b = a + L::A_BYTES;
          // the first CTA's barrier counts the bytes of both
          const uint32_t bar = CTAS == 2 ? leader_bar(&full[s]) : smem_u32(&full[s]);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], CTAS * L::STAGE);
          if constexpr (A_MN) {
            for (int r = 0; r < BM / 64; ++r) load_box<CTAS>(a + r * 8192, &tma, bar, row + r * 64, kb * BK);
          } else {
            load_box<CTAS>(a, &tma, bar, kb * BK, row);
          }
          if constexpr (B_MN) {
            for (int r = 0; r < NB / 64; ++r) load_box<CTAS>(b + r * 8192, &tmb, bar, col + r * 64, kb * BK);
          } else {
            load_box<CTAS>(b, &tmb, bar, kb * BK, col);
          }
        }
      }
      // every issued copy must land before the CTA exits: the first CTA waits for both's, the second for the
      // products' arrivals on its own barriers, which come after
      for (uint32_t back = 1; back <= static_cast<uint32_t>(S) && back <= it; ++back) {
        const uint32_t t = it - back;
        drain_wait(rank == 0 ? &full[t % S] : &empty[t % S], (t / S) & 1u, ctl);
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ products
    if (lane == 0 && rank == 0) {
      uint32_t it = 0, tile = 0;
      bool ok = true;
      for (int u = unit0; ok && u < units; u += stride, ++tile) {
        int mt, nt, part;
        unit_of(grid, u, mt, nt, part);
        const uint32_t buf = tile & 1u;
        if (!wait_arrivals<CTAS>(&acc_empty[buf], ((tile >> 1) & 1u) ^ 1u, ctl, abort_flag)) break;
        tc_fence_after();
        const uint32_t acc = tmem_base + buf * BN;
        const int first = k_first(part), end = k_first(part + 1);
        for (int kb = first; kb < end; ++kb, ++it) {
          const int s = it % S;
          if (!mbar_wait(&full[s], (it / S) & 1u, ctl, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t a = smem_u32(smem + static_cast<size_t>(s) * L::STAGE), b = a + L::A_BYTES;
#pragma unroll
          for (int k = 0; k < BK / 16; ++k)
            mma<CTAS>(acc, A_MN ? sdesc_mn128(a + k * 2048) : sdesc_k128(a + k * 32),
                      B_MN ? sdesc_mn128(b + k * 2048) : sdesc_k128(b + k * 32), IDESC, kb > first || k > 0 ? 1u : 0u);
          commit<CTAS>(&empty[s]);
        }
        if (ok) commit<CTAS>(&acc_full[buf]);
      }
      // all issued MMAs must complete before TMEM is freed
      commit_here<CTAS>(drain);
      drain_wait(drain, 0, ctl);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ epilogue
    // A warp has 32 rows (its quarter of TMEM's lanes) and every other chunk of columns, staged in two buffers in
    // turn: 128 bytes a row, sixteen-byte chunk c at c ^ (row & 7).  A residual is loaded into the
    // buffer its results will take, before the accumulator is there (TMA: a lane's own row would be 32 lines a load).
    const int quad = warp & 3, half = (warp - 2) >> 2;
    uint8_t* stage = smem + L::OFF_EPI + static_cast<size_t>(warp - 2) * L::EPI;
    uint64_t* res_bar = res_full + 2 * (warp - 2);
    constexpr int COLS = sizeof(Out) == 2 ? 64 : 32;  // columns of a staged 128-byte row
    constexpr int CHUNKS = BN / COLS / 2;             // of a warp
    uint32_t puts = 0;                                // buffers used so far
    auto row_of = [&](uint32_t b) { return stage + (b & 1u) * 4096u + lane * 128; };
    // Stores buffer `b`, which this warp has filled.
    auto store = [&](const CUtensorMap& map, uint32_t b, int col, int row0, int part) {
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        tma_store_3d(&map, stage + (b & 1u) * 4096u, col, row0, part);
        bulk_commit();
      }
    };
    auto put = [&](const CUtensorMap& map, const uint32_t (&w)[32], int col, int row0, int part) {
      const uint32_t b = puts++;
      if (lane == 0) bulk_wait_read<1>();  // the buffer's previous store has been read
      __syncwarp();
      uint8_t* row_s = row_of(b);
#pragma unroll
      for (int c = 0; c < 8; ++c)
        *reinterpret_cast<uint4*>(row_s + ((c ^ (lane & 7)) << 4)) = make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
      store(map, b, col, row0, part);
    };
    const bool has_residual = sizeof(Out) == 2 && epi.residual;
    const bool early = has_residual && !epi.keep;  // the kept pre-activations take the buffers first
    uint32_t loads = 0, waits = 0;                 // residual chunks asked for, and waited for
    auto load_residual = [&](int col, int row0) {
      if (lane == 0) {
        bulk_wait_read<0>();
        uint64_t* bar = &res_bar[loads & 1u];
        mbar_arrive_expect_tx(bar, 4096);
        tma_load_3d(stage + (loads & 1u) * 4096u, &tmr, bar, col, row0, 0);
      }
      ++loads;
    };
    uint32_t tile = 0;
    for (int u = unit0; u < units; u += stride, ++tile) {
      int mt, nt, part;
      unit_of(grid, u, mt, nt, part);
      const uint32_t buf = tile & 1u;
      const int row0 = (mt * CTAS + rank) * BM + quad * 32;
      if (early && row0 < M) {
        for (int i = 0; i < CHUNKS; ++i) {
          const int col = nt * BN + (2 * i + half) * COLS;
          if (col < N) load_residual(col, row0);
        }
      }
      if (!warp_wait(&acc_full[buf], (tile >> 1) & 1u, ctl, abort_flag)) break;
      tc_fence_after();
      const uint32_t taddr = tmem_base + buf * BN + (static_cast<uint32_t>(quad * 32) << 16);
      // the accumulator is free for the next tile but one when its last chunk is in registers
      auto release = [&]() {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if constexpr (CTAS == 2)
            arrive_cluster(leader_bar(&acc_empty[buf]));
          else
            mbar_arrive(&acc_empty[buf]);
        }
      };
#pragma unroll 1
      for (int i = 0; i < CHUNKS; ++i) {
        const int c = 2 * i + half, col = nt * BN + c * COLS;
        uint32_t w[32];
        if constexpr (sizeof(Out) == 4) {
          float v[32];
          tmem_ld32(taddr + c * COLS, v);
          tmem_wait_ld();
          if (i == CHUNKS - 1) release();
#pragma unroll
          for (int e = 0; e < 32; ++e) w[e] = __float_as_uint(v[e]);
          if (row0 < M && col < N) put(tmo, w, col, row0, part);
        } else {
          float v[64];
          // the bias is on its way while the sums are read
          uint4 bias[8];
          if (epi.bias) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              bias[e] = col + 8 * e < N ? __ldg(reinterpret_cast<const uint4*>(epi.bias + col) + e) : make_uint4(0u, 0u, 0u, 0u);
          }
          tmem_ld64(taddr + c * COLS, v);
          tmem_wait_ld();
          if (i == CHUNKS - 1) release();
          if (row0 >= M || col >= N) continue;
          if (epi.bias) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float b[8];
              unpack8(bias[e], b);
#pragma unroll
              for (int j = 0; j < 8; ++j) v[8 * e + j] += b[j];
            }
          }
          if (epi.keep) {
#pragma unroll
            for (int e = 0; e < 32; ++e) w[e] = pack2(v[2 * e], v[2 * e + 1]);
            put(tmz, w, col, row0, 0);
          }
          if (epi.act == kActRelu) {
#pragma unroll
            for (int e = 0; e < 64; ++e) v[e] = act_of(v[e], kActRelu);
          } else if (epi.act == kActGelu) {
#pragma unroll
            for (int e = 0; e < 64; ++e) v[e] = act_of(v[e], kActGelu);
          } else if (epi.act == kActSilu) {
#pragma unroll
            for (int e = 0; e < 64; ++e) v[e] = act_of(v[e], kActSilu);
          }
          if (has_residual) {
            if (!early) load_residual(col, row0);
            const uint32_t b = waits++;
            if (!warp_wait(&res_bar[b & 1u], (b >> 1) & 1u, ctl, abort_flag)) break;
            __syncwarp();
            uint8_t* row_s = row_of(b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              uint4* at = reinterpret_cast<uint4*>(row_s + ((e ^ (lane & 7)) << 4));
              float r[8];
              unpack8(*at, r);
              *at = make_uint4(pack2(v[8 * e] + r[0], v[8 * e + 1] + r[1]), pack2(v[8 * e + 2] + r[2], v[8 * e + 3] + r[3]),
                               pack2(v[8 * e + 4] + r[4], v[8 * e + 5] + r[5]), pack2(v[8 * e + 6] + r[6], v[8 * e + 7] + r[7]));
            }
            store(tmo, b, col, row0, 0);
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) w[e] = pack2(v[2 * e], v[2 * e + 1]);
            put(tmo, w, col, row0, 0);
          }
        }
      }
    }
    // residual loads that no chunk waited for (a wait ran out) must land before the CTA exits
    if (lane == 0)
      for (; waits < loads; ++waits) drain_wait(&res_bar[waits & 1u], (waits >> 1) & 1u, ctl);
    if (lane == 0) bulk_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  // a CTA of a pair may leave when the products that read its shared memory, and the loads into it, are done
  if constexpr (CTAS == 2) cluster_sync();
  if (warp == 1) {
    tc_fence_after();
    tmem_give<CTAS>(tmem_base, L::TMEM_COLS);
  }
}

// Eight neighbouring outputs from their fp32 sums.
template <typename Out>
__device__ __forceinline__ void finish8(float (&v)[8], const Epi& epi, Out* out, __nv_bfloat16* z, size_t at, int col) {
  if (epi.bias) {
    float b[8];
    unpack8(__ldg(reinterpret_cast<const uint4*>(epi.bias + col)), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
  }
  if (epi.keep)
    *reinterpret_cast<uint4*>(z + at) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = act_of(v[e], epi.act);
  if (epi.residual) {
    float b[8];
    unpack8(__ldg(reinterpret_cast<const uint4*>(epi.residual + at)), b);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += b[e];
  }
  if constexpr (sizeof(Out) == 2) {
    *reinterpret_cast<uint4*>(out + at) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
  } else {
    reinterpret_cast<float4*>(out + at)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(out + at)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// Adds the parts' partial sums [parts][M][N] in order and finishes the outputs.
template <typename Out>
__global__ void linear_join_kernel(const float* __restrict__ partial, int parts, long long MN, int N, Epi epi, Out* __restrict__ out,
                                   __nv_bfloat16* __restrict__ z) {
  const long long i = (static_cast<long long>(blockIdx.x) * blockDim.x + threadIdx.x) * 8;
  if (i >= MN) return;
  float v[8] = {};
  for (int p = 0; p < parts; ++p) {
    const float4* s = reinterpret_cast<const float4*>(partial + static_cast<size_t>(p) * MN + i);
    const float4 a = s[0], b = s[1];
    v[0] += a.x, v[1] += a.y, v[2] += a.z, v[3] += a.w, v[4] += b.x, v[5] += b.y, v[6] += b.z, v[7] += b.w;
  }
  finish8(v, epi, out, z, static_cast<size_t>(i), static_cast<int>(i % N));
}

// ------------------------------------------------------------ few rows
// y for at most 8 F tokens, where reading W once is the work: a block takes 16 rows of W, its eight warps 64 of the
// sum each in turn, straight from memory into the operand registers of mma.m16n8k16 (W's rows are M, the tokens
// N): a lane's 16 contiguous bytes of a row serve two steps, as the sum's order is free as long as W and x
// agree on it.  The warps' sums are added in shared memory, in order.  tcgen05's way through shared memory and TMEM
// costs 7 us for one tile of K = 768 (this kernel: 2 to 3).
constexpr int kFewWarps = 8;

// Up to 16 tokens always (8192 x 8192: 24 to 27 us, 5.5 TB/s; the tiles take 30).  Up to 64 where W is small: each
// block reads all of x, and 4096 x 1024 weights take 6 to 7 us against 8 to 9 in tiles, 8192 x 8192 75 against 32.
bool few_rows(int M, int N, int K) { return M <= 16 || (M <= 64 && K <= 1024 && static_cast<long long>(N) * K <= (4 << 20)); }

__device__ __forceinline__ uint4 load_once(const __nv_bfloat16* p) {
  uint4 u;
  asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
  return u;
}

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int F>
__global__ void __launch_bounds__(kFewWarps * 32) linear_few_kernel(const __nv_bfloat16* __restrict__ x, const __nv_bfloat16* __restrict__ w, int M,
                                                                   int N, int K, Epi epi, __nv_bfloat16* __restrict__ out,
                                                                   __nv_bfloat16* __restrict__ z) {
  __shared__ float sums[kFewWarps][16][8 * F + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int n0 = blockIdx.x * 16;
  const bool upper = n0 + 8 < N;  // N is a multiple of 8: rows 8 to 15 are all there or all not
  const __nv_bfloat16* w0 = w + static_cast<size_t>(n0 + g) * K + 8 * t;
  const __nv_bfloat16* w1 = upper ? w0 + static_cast<size_t>(8) * K : w0;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  float acc[F][4] = {};
#pragma unroll 2
  for (int k = warp * 64; k < K; k += kFewWarps * 64) {
    uint4 a[2][2], b[2][F];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kk = k + 32 * h;
      const bool in = kk + 8 * t < K;  // K is a multiple of 8
      a[h][0] = in ? load_once(w0 + kk) : zero;
      a[h][1] = in && upper ? load_once(w1 + kk) : zero;
#pragma unroll
      for (int f = 0; f < F; ++f)
        b[h][f] = in && 8 * f + g < M ? __ldg(reinterpret_cast<const uint4*>(x + static_cast<size_t>(8 * f + g) * K + 8 * t + kk)) : zero;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int f = 0; f < F; ++f) {
        mma_16x8x16(acc[f], a[h][0].x, a[h][1].x, a[h][0].y, a[h][1].y, b[h][f].x, b[h][f].y);
        mma_16x8x16(acc[f], a[h][0].z, a[h][1].z, a[h][0].w, a[h][1].w, b[h][f].z, b[h][f].w);
      }
  }
#pragma unroll
  for (int f = 0; f < F; ++f)
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[warp][g + (e & 2) * 4][8 * f + 2 * t + (e & 1)] = acc[f][e];
  __syncthreads();
  const int m = threadIdx.x >> 1, half = threadIdx.x & 1;  // eight outputs of a token
  if (m < M && (half == 0 || upper)) {
    float v[8] = {};
    for (int i = 0; i < kFewWarps; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += sums[i][8 * half + e][m];
    finish8(v, epi, out, z, static_cast<size_t>(m) * N + n0 + 8 * half, n0 + 8 * half);
  }
}

// ------------------------------------------------------------ dz and db
constexpr int kDzRows = 64;  // rows of a block

// dz = dy act'(z) as bf16 (nothing is written for act none: dz is dy), and the block's sums of its unrounded columns.
// Bound by HBM: a thread takes eight columns of every fourth row, two rows' loads in flight at once (8197 x 4096 with
// ReLU: 31 us, 6.5 TB/s; four or eight rows at once cost registers: 33 and 36).
template <int ACT>
__global__ void __launch_bounds__(256) linear_dz_kernel(const __nv_bfloat16* __restrict__ dy, const __nv_bfloat16* __restrict__ z, int M, int N,
                                                        __nv_bfloat16* __restrict__ dz, float* __restrict__ partial) {
  constexpr int U = 2;
  __shared__ float sums[4][64 * 8];
  const int cx = threadIdx.x & 63, ry = threadIdx.x >> 6;
  const int col = (blockIdx.y * 64 + cx) * 8;
  const long long m0 = static_cast<long long>(blockIdx.x) * kDzRows;
  float a[8] = {};
  if (col < N) {
#pragma unroll 1
    for (int r = ry; r < kDzRows; r += 4 * U) {
      uint4 gr[U], zr[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const long long m = m0 + r + 4 * u;
        if (m < M) {
          gr[u] = __ldg(reinterpret_cast<const uint4*>(dy + m * N + col));
          if (ACT != kActNone) zr[u] = __ldg(reinterpret_cast<const uint4*>(z + m * N + col));
        } else {
          gr[u] = zr[u] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float g[8];
        unpack8(gr[u], g);
        if (ACT != kActNone) {
          float zv[8];
          unpack8(zr[u], zv);
#pragma unroll
          for (int e = 0; e < 8; ++e) g[e] *= act_slope(zv[e], ACT);
          const long long m = m0 + r + 4 * u;
          if (m < M)
            *reinterpret_cast<uint4*>(dz + m * N + col) = make_uint4(pack2(g[0], g[1]), pack2(g[2], g[3]), pack2(g[4], g[5]), pack2(g[6], g[7]));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) a[e] += g[e];
      }
    }
  }
  if (!partial) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) sums[ry][cx * 8 + e] = a[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += 256)
    if (blockIdx.y * 512 + i < N)
      partial[static_cast<size_t>(blockIdx.x) * N + blockIdx.y * 512 + i] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
}

// db[n] = the row blocks' partial sums, in order: 32 columns a block, 32 threads each.
template <typename Out>
__global__ void __launch_bounds__(1024) linear_db_kernel(const float* __restrict__ partial, int rows, int N, Out* __restrict__ db) {
  __shared__ float sums[32][33];
  const int n = blockIdx.x * 32 + threadIdx.x;
  float a = 0.f;
  if (n < N) {
#pragma unroll 4
    for (int r = threadIdx.y; r < rows; r += 32) a += partial[static_cast<size_t>(r) * N + n];
  }
  sums[threadIdx.y][threadIdx.x] = a;
  __syncthreads();
  if (threadIdx.y == 0 && n < N) {
    for (int y = 1; y < 32; ++y) a += sums[y][threadIdx.x];
    if constexpr (sizeof(Out) == 2)
      db[n] = __float2bfloat16_rn(a);
    else
      db[n] = a;
  }
}

// ------------------------------------------------------------ host
bool make_out_map(CUtensorMap* map, const void* base, bool f32, uint64_t cols, uint64_t rows, uint64_t parts) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return false;
  const uint64_t e = f32 ? 4 : 2;
  cuuint64_t dims[3] = {cols, rows, parts};
  cuuint64_t strides[2] = {cols * e, cols * rows * e};
  cuuint32_t box[3] = {f32 ? 32u : 64u, 32, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(map, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box,
             estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product is cut: CTAs and width of a tile, parts of the sum.
struct Cut {
  int ctas, bn, parts;
};

// `out_rows` x `out_cols`, summed over `sum`.  The cut with the least estimated time, in microseconds as measured: a
// block of 64 of the sum takes 0.36 on a 256 x 256 tile of a pair, 0.40 on 128 x 256, and 0.33 on 128 x 128 (the
// tensor pipe runs at half rate for 128 columns); a split sum writes and reads its partial tiles (about 5 TB/s) and
// takes another launch (3).
Cut cut_of(int out_rows, int out_cols, int sum, int num_sms) {
  constexpr Cut kCuts[3] = {{2, 256, 1}, {1, 256, 1}, {1, 128, 1}};
  constexpr double kBlock[3] = {0.36, 0.40, 0.33};
  const int kb = (sum + BK - 1) / BK;
  Cut best = kCuts[0];
  double least = 1e30;
  for (int i = 0; i < 3; ++i) {
    const int rows = BM * kCuts[i].ctas;
    const long long tiles = static_cast<long long>((out_rows + rows - 1) / rows) * ((out_cols + kCuts[i].bn - 1) / kCuts[i].bn);
    const long long places = num_sms / kCuts[i].ctas;
    // more parts than fill the places once do not pay; a part has at least four blocks
    for (int p = 1; p == 1 || (p <= kb / 4 && tiles * (p - 1) < places); ++p) {
      const double waves = static_cast<double>((tiles * p + places - 1) / places);
      double us = waves * ((kb + p - 1) / p) * kBlock[i];
      if (p > 1) us += 3.0 + static_cast<double>(p) * out_rows * out_cols * 8.0 / 5e6;
      if (us < least) least = us, best = kCuts[i], best.parts = p;
    }
  }
  return best;
}

template <int CTAS, int BN, bool A_MN, bool B_MN, typename Out>
int launch_mma(const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& to, const CUtensorMap& tz, const CUtensorMap& tr, const Epi& epi, const Grid& g, int rows,
               int cols, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  auto kern = linear_mma_kernel<CTAS, BN, A_MN, B_MN, Out>;
  constexpr int bytes = static_cast<int>(Layout<CTAS, BN>::BYTES);
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return -1;
  const long long units = static_cast<long long>(g.m_tiles) * g.n_tiles * g.parts, most = num_sms / CTAS;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(units < most ? units : most) * CTAS);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = CTAS;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = CTAS > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kern, ta, tb, to, tz, tr, epi, g, rows, cols, ctl) == cudaSuccess ? 1 : -1;
}

// D [rows][cols] = sum over `sum`; a is [rows][sum] or, A_MN, [sum][rows]; b likewise.
template <bool A_MN, bool B_MN>
int product(const void* a, const void* b, int rows, int cols, int sum, const Epi& epi, void* out, bool out_f32, void* z, float* partial,
            int num_sms, const DevCtl& ctl, cudaStream_t st) {
  const Cut cut = cut_of(rows, cols, sum, num_sms);
  CUtensorMap ta, tb, to, tz, tr;
  if (!(A_MN ? make_tmap_bf16_3d(&ta, a, rows, sum, 1, 64) : make_tmap_bf16_3d(&ta, a, sum, rows, 1, BM))) return -1;
  if (!(B_MN ? make_tmap_bf16_3d(&tb, b, cols, sum, 1, 64) : make_tmap_bf16_3d(&tb, b, sum, cols, 1, cut.bn / cut.ctas))) return -1;
  const bool f32 = out_f32 || cut.parts > 1;
  if (!make_out_map(&to, cut.parts > 1 ? partial : out, f32, cols, rows, cut.parts)) return -1;
  tz = tr = to;
  if (epi.keep && cut.parts == 1 && !make_out_map(&tz, z, false, cols, rows, 1)) return -1;
  if (epi.residual && cut.parts == 1 && !make_out_map(&tr, epi.residual, false, cols, rows, 1)) return -1;
  const int tile = BM * cut.ctas;
  const Grid g{(rows + tile - 1) / tile, (cols + cut.bn - 1) / cut.bn, cut.parts, (sum + BK - 1) / BK};
  auto go = [&](auto ctas, auto bn) {
    constexpr int C = decltype(ctas)::value, W = decltype(bn)::value;
    return f32 ? launch_mma<C, W, A_MN, B_MN, float>(ta, tb, to, tz, tr, epi, g, rows, cols, num_sms, ctl, st)
               : launch_mma<C, W, A_MN, B_MN, __nv_bfloat16>(ta, tb, to, tz, tr, epi, g, rows, cols, num_sms, ctl, st);
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  const int n = cut.ctas == 2   ? go(Two(), std::integral_constant<int, 256>())
                : cut.bn == 256 ? go(One(), std::integral_constant<int, 256>())
                                : go(One(), std::integral_constant<int, 128>());
  if (n < 0 || cut.parts == 1) return n;
  const long long MN = static_cast<long long>(rows) * cols;
  const int blocks = static_cast<int>((MN / 8 + 255) / 256);
  if (out_f32)
    linear_join_kernel<float><<<blocks, 256, 0, st>>>(partial, cut.parts, MN, cols, epi, static_cast<float*>(out), static_cast<__nv_bfloat16*>(z));
  else
    linear_join_kernel<__nv_bfloat16><<<blocks, 256, 0, st>>>(partial, cut.parts, MN, cols, epi, static_cast<__nv_bfloat16*>(out),
                                                              static_cast<__nv_bfloat16*>(z));
  return cudaGetLastError() == cudaSuccess ? n + 1 : -1;
}

size_t partial_bytes(int rows, int cols, int sum, int num_sms) {
  const Cut c = cut_of(rows, cols, sum, num_sms);
  return c.parts > 1 ? static_cast<size_t>(c.parts) * rows * cols * sizeof(float) : 0;
}

size_t round256(size_t b) { return (b + 255) / 256 * 256; }

template <int F>
int launch_few(const LinearArgs& a, const Epi& epi, cudaStream_t st) {
  linear_few_kernel<F><<<(a.N + 15) / 16, kFewWarps * 32, 0, st>>>(static_cast<const __nv_bfloat16*>(a.x), static_cast<const __nv_bfloat16*>(a.w), a.M, a.N,
                                                                  a.K, epi, static_cast<__nv_bfloat16*>(a.y), static_cast<__nv_bfloat16*>(a.z));
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace

size_t linear_fwd_workspace_bytes(int M, int N, int K, int num_sms) { return few_rows(M, N, K) ? 0 : partial_bytes(M, N, K, num_sms); }

int linear_fwd(const LinearArgs& a, void* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  const Epi epi{static_cast<const __nv_bfloat16*>(a.bias), static_cast<const __nv_bfloat16*>(a.residual), a.act, a.z != nullptr};
  if (few_rows(a.M, a.N, a.K)) {
    if (a.M <= 8) return launch_few<1>(a, epi, st);
    if (a.M <= 16) return launch_few<2>(a, epi, st);
    if (a.M <= 32) return launch_few<4>(a, epi, st);
    return launch_few<8>(a, epi, st);
  }
  return product<false, false>(a.x, a.w, a.M, a.N, a.K, epi, a.y, false, a.z, static_cast<float*>(workspace), num_sms, ctl, st);
}

// dz (unless act is none), the row blocks' sums for db, and the larger of the two products' partial sums.
size_t linear_bwd_workspace_bytes(int M, int N, int K, int act, int num_sms) {
  const size_t dz = act == kActNone ? 0 : round256(static_cast<size_t>(M) * N * 2);
  const size_t db = round256(static_cast<size_t>((M + kDzRows - 1) / kDzRows) * N * sizeof(float));
  const size_t p1 = partial_bytes(M, K, N, num_sms), p2 = partial_bytes(N, K, M, num_sms);
  return dz + db + (p1 > p2 ? p1 : p2);
}

int linear_bwd(const LinearBwdArgs& a, void* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  const size_t dz_bytes = a.act == kActNone ? 0 : round256(static_cast<size_t>(a.M) * a.N * 2);
  const int row_blocks = (a.M + kDzRows - 1) / kDzRows;
  float* sums = reinterpret_cast<float*>(ws + dz_bytes);
  float* partial = reinterpret_cast<float*>(ws + dz_bytes + round256(static_cast<size_t>(row_blocks) * a.N * sizeof(float)));
  const void* dz = a.act == kActNone ? a.dy : ws;
  const Epi none{nullptr, nullptr, kActNone, 0};
  int launches = 0;
  if (a.act != kActNone || a.db) {
    const dim3 grid(row_blocks, (a.N + 511) / 512);
    const __nv_bfloat16 *dy = static_cast<const __nv_bfloat16*>(a.dy), *z = static_cast<const __nv_bfloat16*>(a.z);
    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(ws);
    float* to = a.db ? sums : nullptr;
    if (a.act == kActNone)
      linear_dz_kernel<kActNone><<<grid, 256, 0, st>>>(dy, z, a.M, a.N, out, to);
    else if (a.act == kActRelu)
      linear_dz_kernel<kActRelu><<<grid, 256, 0, st>>>(dy, z, a.M, a.N, out, to);
    else if (a.act == kActGelu)
      linear_dz_kernel<kActGelu><<<grid, 256, 0, st>>>(dy, z, a.M, a.N, out, to);
    else
      linear_dz_kernel<kActSilu><<<grid, 256, 0, st>>>(dy, z, a.M, a.N, out, to);
    if (cudaGetLastError() != cudaSuccess) return -1;
    ++launches;
  }
  if (a.db) {
    if (a.grad_f32)
      linear_db_kernel<float><<<(a.N + 31) / 32, dim3(32, 32), 0, st>>>(sums, row_blocks, a.N, static_cast<float*>(a.db));
    else
      linear_db_kernel<__nv_bfloat16><<<(a.N + 31) / 32, dim3(32, 32), 0, st>>>(sums, row_blocks, a.N, static_cast<__nv_bfloat16*>(a.db));
    if (cudaGetLastError() != cudaSuccess) return -1;
    ++launches;
  }
  if (a.dx) {
    const int n = product<false, true>(dz, a.w, a.M, a.K, a.N, none, a.dx, false, nullptr, partial, num_sms, ctl, st);
    if (n < 0) return -1;
    launches += n;
  }
  if (a.dw) {
    const int n = product<true, true>(dz, a.x, a.N, a.K, a.M, none, a.dw, a.grad_f32, nullptr, partial, num_sms, ctl, st);
    if (n < 0) return -1;
    launches += n;
  }
  return launches;
}

}  // namespace topk
