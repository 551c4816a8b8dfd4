// grouped.cu -- plain attention (Eq. 1) of grouped heads on the tensor cores: over packed prompts of different
// lengths, and of drafted tokens over key/value caches.  One kernel serves both.
//
// A unit of work is a key head of a sequence with the rows of two 128-row tiles: a row is one query head of one
// token, and a tile takes as many tokens as its 128 rows hold of the group's heads, so that a group's heads share
// every key tile that is staged.  Per 64 keys and tile
//   S = Q K^T      tcgen05.mma, fp32 in TMEM;
//   P = 2^(S - m)  four warps, a row each thread, written over S as the bf16 operand that the next product
//                  reads from TMEM;
//   O += P V       tcgen05.mma, V as it lies in memory (its keys are the sum: the instruction transposes).
// P is two bf16, the rounded weight and the rest, with a product each: the result is then rounded once, where a single bf16 is a
// second rounding of the same size (error against 64 bits 1.6e-3 in place of 2.1e-3).  It is so for every call, so that a sequence's
// precision does not depend on what it is packed with.  Where the products bound a call that costs a quarter: 12 prompts of up to 4,093
// tokens 477 -> 586 us, 16,384 tokens 758 -> 949, 64 drafted tokens of 16 caches of 16,384 rows 146 -> 177; caches of fewer rows a key head are
// bound by memory (16 drafted tokens 204 either way).
// While the warps of one tile are at its exponentials, the tensor pipe works for the other.  A row's running maximum
// m is raised only when a tile's exceeds it by more than kRaise; O and the sum are scaled then.
//
// Sequences differ in length by orders of magnitude, and only the device knows the lengths.  So the key tiles of all
// units are numbered in one row, with a few more behind each unit for what it costs by itself, and every CTA takes an equal run of them: it
// computes from the lengths where its run begins.  A run that begins or ends inside a unit leaves that unit's (m, sum, O) in scratch, at most two
// such parts for each CTA, and grouped_join_kernel joins the parts of a unit in order.
#include <cuda_bf16.h>

#include <atomic>

#include "kernels.h"
#include "pairs.cuh"

namespace topk {

namespace {

constexpr int BM = 128, BN = 64;  // rows of a tile, keys of a step
constexpr int kThreads = 384;     // loads, scores, products of each tile with the values; two groups of four softmax warps
constexpr float kRaise = 8.0f;    // natural-log units
constexpr float kLog2e = 1.4426950408889634f;

// Where a CTA's run of steps begins, of how many steps and CTAs with work.
struct Place {
  int b, h, block, kt;
  long long total;
  int ctas, skip;     // skip: steps of the run that are none, at its beginning
  int q0, Lq, tiles;  // of the sequence, and of the unit: for the join
};

template <int D, bool TREE>
struct Layout {
  static constexpr int R = D / 64;                 // blocks of 128 bytes of a row
  static constexpr uint32_t Q_TILE = BM * D * 2, Q_BLOCK = BM * 128;
  static constexpr uint32_t TILE = BN * D * 2, BLOCK = BN * 128;  // keys or values of a step
  static constexpr int STAGE = TREE ? 0 : 32 * 128;  // a softmax warp's outputs on their way out (prompts, whose units are short)
  static constexpr int FIT = (232448 - 3072 - 8 * STAGE - 2 * static_cast<int>(Q_TILE)) / static_cast<int>(TILE);
  static constexpr int S = FIT > 16 ? 16 : FIT;      // keys and values of a step in turn: 8 or 10 for D = 128, 16 for 64
  static constexpr size_t OFF_RING = 2 * static_cast<size_t>(Q_TILE);
  static constexpr size_t OFF_STAGE = OFF_RING + static_cast<size_t>(S) * TILE;
  static constexpr size_t OFF_BAR = OFF_STAGE + 8 * STAGE;
  static constexpr int NBARS = 2 * S + 22;
  static constexpr size_t OFF_EXCH = OFF_BAR + NBARS * 8 + 64;  // flags and the place between them
  static constexpr size_t BYTES = 1024 + OFF_EXCH + BM * 8;
  static_assert(BYTES <= 232448, "shared memory");
  static_assert(2 * sizeof(int) + sizeof(Place) + sizeof(long long) <= 64, "between the barriers and the exchange");
  static_assert(S >= 8 && S % 2 == 0, "scores run at most three steps ahead of the products with the values; keys lie in the even slots");
  // TMEM columns: two score buffers of each tile, two outputs
  static constexpr uint32_t O_COL = 4 * BN;
  static constexpr uint32_t COLS = 512;
};

// A part of a unit in scratch: O as float4 [D / 4][256 rows], then m and the sum of each row.
template <int D>
constexpr size_t kPartFloats = 256 * (D + 2);

// What a unit costs beside its steps (first and last steps that wait, the output), in steps: they count in the runs, so that CTAs with
// many short units have as much to do as those with a few long ones.  12 prompts of up to 4,093 tokens take 697 us with 0, 592 with 2, 583 with
// 3, 586 with 4, 614 with 6 (heads of 64: 509, 427, 428, 432, 450); a prompt of 16,384 tokens 1040, 974, 949, 949, 958; single tokens of 4 sequences
// 25.1, 24.6, 24.5, 24.1, 23.8.
constexpr int kUnit = 4;

constexpr int kMostParts = 160;  // of a unit: one from each CTA, of which there are no more than SMs (152)

struct Work {
  const int32_t* q_starts;   // prompts
  const int32_t* k_starts;
  const int32_t* kv_len;     // caches
  const int64_t* words;
  long long word_stride;
  __nv_bfloat16* out;
  float* parts;
  Place* places;  // of every CTA, for the join
  int B, Hq, Hkv, group, Tq, Tk, T, cap, causal, clear_rest;
  int tokens;  // of a tile
};

// One sequence: its rows in q and k, and how many; with a cache, how many keys precede the drafted ones.
struct Seq {
  int q0, Lq, k0, Lk, prefix;
  int blocks;  // pairs of tiles
};

template <bool TREE>
__device__ __forceinline__ Seq seq_of(const Work& w, int b, bool* bad = nullptr) {
  Seq s;
  if constexpr (TREE) {
    const int n = __ldg(w.kv_len + b);
    s.q0 = s.k0 = 0;
    s.Lq = w.T;
    s.prefix = min(max(n, 0), w.cap);
    s.Lk = n < 0 ? 0 : min(s.prefix + w.T, w.cap);
    if (bad) *bad = static_cast<long long>(n) + w.T > w.cap;
  } else {
    const int q0 = __ldg(w.q_starts + b), q1 = __ldg(w.q_starts + b + 1);
    s.q0 = min(max(q0, 0), w.Tq);
    const int qe = max(s.q0, min(max(q1, 0), w.Tq));
    const int k0 = __ldg(w.k_starts + b), k1 = __ldg(w.k_starts + b + 1);
    s.k0 = min(max(k0, 0), w.Tk);
    const int ke = max(s.k0, min(max(k1, 0), w.Tk));
    s.Lq = qe - s.q0, s.Lk = ke - s.k0;
    s.prefix = 0;
    if (bad) *bad = q0 != s.q0 || q1 != qe || k0 != s.k0 || k1 != ke;
  }
  s.blocks = (s.Lq + 2 * w.tokens - 1) / (2 * w.tokens);
  return s;
}

// Key tiles that the tokens up to `last` read: one at least, which is masked where they read nothing.
template <bool TREE>
__device__ __forceinline__ int key_tiles(const Work& w, const Seq& s, int last) {
  const int lim = !TREE && w.causal ? last + 1 + s.Lk - s.Lq : s.Lk;
  return max(1, (lim + BN - 1) / BN);
}

template <bool TREE>
__device__ __forceinline__ int block_tiles(const Work& w, const Seq& s, int block) {
  return key_tiles<TREE>(w, s, min((block + 1) * 2 * w.tokens, s.Lq) - 1);
}

// sum over i < n of floor((a i + b) / BN), by the steps of Euclid's algorithm for (a, BN)
__device__ __forceinline__ long long floor_sum(unsigned n, unsigned a, unsigned b) {
  // the first step, whose divisor is known
  long long sum = static_cast<long long>(a / BN) * (static_cast<long long>(n) * (n - 1) / 2) + static_cast<long long>(b / BN) * n;
  a %= BN, b %= BN;
  const unsigned y = a * n + b;
  if (y < BN) return sum;
  n = y / BN, b = y % BN;
  unsigned m = a;
  a = BN;
  while (n) {
    sum += static_cast<long long>(a / m) * (static_cast<long long>(n) * (n - 1) / 2) + static_cast<long long>(b / m) * n;
    a %= m, b %= m;
    const unsigned y = a * n + b;
    if (y < m) break;
    n = y / m, b = y % m;
    const unsigned t = a;
    a = m, m = t;
  }
  return sum;
}

// Key tiles of a head's blocks before `block`.
template <bool TREE>
__device__ __forceinline__ long long tiles_before(const Work& w, const Seq& s, int block) {
  if (block == 0) return 0;
  if (TREE || !w.causal) return static_cast<long long>(block) * max(1, (s.Lk + BN - 1) / BN);
  if (block == s.blocks) return tiles_before<TREE>(w, s, block - 1) + block_tiles<TREE>(w, s, block - 1);
  // block i < blocks - 1 reads (i + 1) step + Lk - Lq keys
  const int step = 2 * w.tokens, more = s.Lk - s.Lq;
  const int none = more < 0 ? min(block, -more / step) : 0;  // blocks that read nothing
  if (block == none) return none;
  return none + floor_sum(block - none, step, (none + 1) * step + more + BN - 1);
}

// x / y; most are small, and a division of 64 bits takes hundreds of cycles
__device__ __forceinline__ long long quotient(long long x, long long y) {
  if (x >> 32 == 0 && y >> 32 == 0) return static_cast<unsigned>(x) / static_cast<unsigned>(y);
  return x / y;
}

// Steps of a head's blocks before `block`, kUnit behind each one's own among them.
template <bool TREE>
__device__ __forceinline__ long long steps_before(const Work& w, const Seq& s, int block) {
  return tiles_before<TREE>(w, s, block) + static_cast<long long>(kUnit) * block;
}

// The step that the run of CTA i of `ctas` begins with.  What memory holds makes fewer than 2^52 steps.
__device__ __forceinline__ long long run_start(long long total, int ctas, int i) { return quotient(total * i, ctas); }

// Where the step number run_start(total, .., i) is; computed by a whole warp.
template <bool TREE>
__device__ Place locate(const Work& w, int i, int grid, unsigned* error) {
  const int lane = threadIdx.x & 31;
  Place p{};
  bool wrong = false;
  Seq s{};
  long long mine = 0;  // of the last sequence looked at: with up to 32 of them the lane's own
  for (int b = lane; b < w.B; b += 32) {
    bool bad;
    s = seq_of<TREE>(w, b, &bad);
    wrong |= bad;
    mine = steps_before<TREE>(w, s, s.blocks) * w.Hkv;
    p.total += mine;
  }
  if (error && wrong) atomicOr(error, kDevErrRange);
  for (int o = 16; o; o >>= 1) p.total += __shfl_xor_sync(0xffffffffu, p.total, o);
  p.ctas = static_cast<int>(min(static_cast<long long>(grid), p.total));
  if (i >= p.ctas) return p;
  long long left = run_start(p.total, p.ctas, i);
  for (int b0 = 0; b0 < w.B; b0 += 32) {
    if (w.B > 32) {
      mine = 0;
      if (b0 + lane < w.B) {
        s = seq_of<TREE>(w, b0 + lane);
        mine = steps_before<TREE>(w, s, s.blocks) * w.Hkv;
      }
    }
    long long upto = mine;
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    const unsigned at = __ballot_sync(0xffffffffu, upto > left);
    if (at) {
      const int k = __ffs(at) - 1;
      int h = 0, block = 0, kt = 0, tiles = 0, skip = 0;
      if (lane == k) {
        left -= upto - mine;
        const long long head = quotient(mine, w.Hkv);
        h = static_cast<int>(quotient(left, head));
        left -= h * head;
        int lo = 0, hi = s.blocks - 1;  // the last block with steps_before <= left
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (steps_before<TREE>(w, s, mid) <= left)
            lo = mid;
          else
            hi = mid - 1;
        }
        block = lo;
        kt = static_cast<int>(left - steps_before<TREE>(w, s, lo));
        tiles = block_tiles<TREE>(w, s, lo);
        if (kt >= tiles) skip = tiles + kUnit - kt, kt = 0, ++block;  // behind the unit's steps: the next one (or the next head's first)
      }
      p.b = b0 + k;
      p.h = __shfl_sync(0xffffffffu, h, k);
      p.block = __shfl_sync(0xffffffffu, block, k);
      p.kt = __shfl_sync(0xffffffffu, kt, k);
      p.skip = __shfl_sync(0xffffffffu, skip, k);
      p.q0 = __shfl_sync(0xffffffffu, s.q0, k);
      p.Lq = __shfl_sync(0xffffffffu, s.Lq, k);
      p.tiles = __shfl_sync(0xffffffffu, tiles, k);
      return p;
    }
    left -= __shfl_sync(0xffffffffu, upto, 31);
  }
  return p;
}

// A run's part of one unit: steps [kt0, kt1) of its n; tile x of the two takes those below n_tile[x].  Of a unit of one
// tile the two groups of warps take every other step, each with an output of its own.
struct Segment {
  int b, h, block, kt0, kt1, n;
  int n_tile[2];
  Seq seq;
  __device__ __forceinline__ bool split() const { return n_tile[1] == 0; }
  __device__ __forceinline__ bool active(int x) const { return split() ? kt1 - kt0 > x : kt0 < min(kt1, n_tile[x]); }
  __device__ __forceinline__ bool whole() const { return kt0 == 0 && kt1 == n; }
};

template <bool TREE>
struct Run {
  const Work& w;
  Seq seq;
  int b, h, block, kt;
  long long left;

  __device__ __forceinline__ Run(const Work& work, const Place& p, long long tiles) : w(work), b(p.b), h(p.h), block(p.block), kt(p.kt), left(tiles) {
    if (left > 0) seq = seq_of<TREE>(w, b);
  }
  __device__ __forceinline__ bool next(Segment& s) {
    if (left <= 0) return false;
    if (block >= seq.blocks) {
      block = 0;
      if (++h == w.Hkv) {
        h = 0;
        do {
          if (++b >= w.B) return false;
          seq = seq_of<TREE>(w, b);
        } while (seq.blocks == 0);
      }
    }
    s.b = b, s.h = h, s.block = block, s.kt0 = kt;
    s.seq = seq;
    s.n = 0;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int t0 = (2 * block + x) * w.tokens;
      s.n_tile[x] = t0 < seq.Lq ? key_tiles<TREE>(w, seq, min(t0 + w.tokens, seq.Lq) - 1) : 0;
      s.n = max(s.n, s.n_tile[x]);
    }
    s.kt1 = static_cast<int>(min(static_cast<long long>(s.n), kt + left));
    left -= (s.kt1 == s.n ? s.n + kUnit : s.kt1) - kt;
    kt = 0;
    ++block;
    return true;
  }
};

// A place in the ring of keys and values, which alternate, and the parity of its phase.
struct Slot {
  uint32_t slot, parity;
  __device__ __forceinline__ void advance(uint32_t slots) {
    slot += 2;
    if (slot >= slots) slot -= slots, parity ^= 1u;
  }
};

// ------------------------------------------------------------ instructions
__device__ __forceinline__ void load_4d(void* dst, const void* map, uint64_t* bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// D[tmem] (+)= A[tmem] B[smem]: A's rows are lanes, two bf16 of a row in each column.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}

// V's tile, keys x d, as an operand whose sum runs over the rows: 64-column blocks a whole tile of rows apart, groups of eight
// keys 1024 bytes.
__device__ __forceinline__ uint64_t sdesc_values(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>((BN * 128) >> 4) << 16;
  d |= static_cast<uint64_t>(1024 >> 4) << 32;
  d |= static_cast<uint64_t>(1) << 46;
  d |= static_cast<uint64_t>(2) << 61;
  return d;
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
      "r"(r[14]), "r"(r[15])
      : "memory");
}

__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ F2 add2(F2 a, F2 b) {
  F2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
  return r;
}

// 2^x (ex2.approx, 2^-22); 2^-inf = 0
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const DevCtl& ctl, volatile int* abort_flag) {
  const bool ok = mbar_wait(bar, parity, ctl, abort_flag);
  return __all_sync(0xffffffffu, ok);
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

// Which of the keys j0 .. j0 + 63 a row reads, a bit each: those below `lim`, and drafted key i, at prefix + i, where bit
// i of `word` is set.
template <bool TREE>
__device__ __forceinline__ void key_bits(uint32_t (&bits)[BN / 32], int j0, int lim, int prefix, unsigned long long word) {
  const auto below = [](int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; };
#pragma unroll
  for (int i = 0; i < BN / 32; ++i) {
    const int j = j0 + 32 * i;
    if constexpr (TREE) {
      const int first = prefix - j;  // of the drafted keys
      uint32_t drafted = 0;
      if (first <= 0 && first > -64) drafted = static_cast<uint32_t>(word >> -first);
      if (first > 0 && first < 32) drafted = static_cast<uint32_t>(word << first);
      bits[i] = below(first) | (drafted & below(lim - j));
    } else {
      bits[i] = below(lim - j);
    }
  }
}

// ------------------------------------------------------------ the kernel
template <int D, bool TREE>
__global__ void __launch_bounds__(kThreads, 1)
    grouped_kernel(const __grid_constant__ CUtensorMap tmq, const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv,
                   const __grid_constant__ Work w, DevCtl ctl) {
  using L = Layout<D, TREE>;
  constexpr int S = L::S, R = L::R;
  constexpr uint32_t IDESC_S = idesc_bf16_f32(BM, BN), IDESC_O = idesc_bf16_f32(BM, D) | (1u << 16);

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* ring = smem + L::OFF_RING;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + L::OFF_BAR);
  uint64_t* empty = full + S;
  uint64_t* q_full = full + 2 * S;
  uint64_t* q_empty = q_full + 1;
  uint64_t* s_full = q_full + 2;    // [tile][buffer]
  uint64_t* p_full = q_full + 6;    // [tile][buffer]
  uint64_t* pv_done = q_full + 10;  // [tile][buffer]
  uint64_t* o_full = q_full + 14;   // [tile]
  uint64_t* o_free = q_full + 16;   // [tile]
  uint64_t* v_tail = q_full + 18;   // [tile]
  uint64_t* exch_full = q_full + 20;
  uint64_t* drain = q_full + 21;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(full + L::NBARS);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  Place* place_s = reinterpret_cast<Place*>(tmem_slot + 2);  // 8-byte aligned
  long long* steps_s = reinterpret_cast<long long*>(place_s + 1);
  float2* exch = reinterpret_cast<float2*>(smem + L::OFF_EXCH);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], s % 2 == 0 ? 1 : 2);  // values: the products of both tiles
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int x = 0; x < 4; ++x) {
      mbar_init(&s_full[x], 1);
      mbar_init(&p_full[x], 4);
      mbar_init(&pv_done[x], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&o_full[x], 1);
      mbar_init(&o_free[x], 4);
      mbar_init(&v_tail[x], 1);
    }
    mbar_init(exch_full, 4);
    mbar_init(drain, 3);
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, L::COLS);
  if (warp == 3 && lane < 3) tma_prefetch_desc(lane == 0 ? &tmq : lane == 1 ? &tmk : &tmv);
  if (warp == 2) {
    const Place p = locate<TREE>(w, blockIdx.x, gridDim.x, blockIdx.x == 0 ? ctl.error : nullptr);
    if (lane == 0) {
      const int i = blockIdx.x, ctas = p.ctas;
      *place_s = p;
      w.places[i] = p;
      *steps_s = i < ctas ? run_start(p.total, ctas, i + 1) - run_start(p.total, ctas, i) - p.skip : 0;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the join's blocks may wait from now on
  const uint32_t tmem = *tmem_slot;
  const long long steps = *steps_s;
  const Place place = *place_s;

  if (warp == 0) {
    // ------------------------------------------------------------ loads
    if (elect_one()) {
      Run<TREE> run(w, place, steps);
      Segment seg;
      uint32_t it = 0, segs = 0;  // ring tiles and units' queries loaded
      bool ok = true;
      auto load = [&](const CUtensorMap& map, int row, int h, int b) {
        const uint32_t s = it % S;
        if (!mbar_wait(&empty[s], ((it / S) & 1u) ^ 1u, ctl, abort_flag)) return false;
        mbar_arrive_expect_tx(&full[s], L::TILE);
#pragma unroll
        for (int r = 0; r < R; ++r) load_4d(ring + s * L::TILE + r * L::BLOCK, &map, &full[s], r * 64, row, h, b);
        ++it;
        return true;
      };
      while (ok && run.next(seg)) {
        const int b = TREE ? seg.b : 0;
        for (int kt = seg.kt0; ok && kt < seg.kt1; ++kt) {
          const int row = seg.seq.k0 + kt * BN;
          ok = load(tmk, row, seg.h, b);
          if (ok && kt == seg.kt0) {
            ok = mbar_wait(q_empty, (segs & 1u) ^ 1u, ctl, abort_flag);
            if (ok) {
              const int n = seg.split() ? 1 : 2;
              mbar_arrive_expect_tx(q_full, static_cast<uint32_t>(n * R * 128 * w.tokens * w.group));
              for (int x = 0; x < n; ++x)
#pragma unroll
                for (int r = 0; r < R; ++r)
                  load_4d(smem + x * L::Q_TILE + r * L::Q_BLOCK, &tmq, q_full, r * 64, seg.h * w.group, seg.seq.q0 + (2 * seg.block + x) * w.tokens, b);
              ++segs;
            }
          }
          ok = ok && load(tmv, row, seg.h, b);
        }
      }
      // every issued copy must land before the CTA exits
      for (uint32_t back = 1; back <= static_cast<uint32_t>(S) && back <= it; ++back) drain_wait(&full[(it - back) % S], ((it - back) / S) & 1u, ctl);
      if (segs) drain_wait(q_full, (segs - 1) & 1u, ctl);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ------------------------------------------------------------ scores
    // A tile has two score buffers (P takes its scores' place), so that the scores of its next step are there when its warps
    // are done with this one.  A barrier's phase is known by its parity alone, so whoever waits on one waits for its every phase: both
    // tiles take note of values that only one of them reads.  Every warp that issues products does so under elect: under a test
    // of the lane the compiler does not know that one thread is left, and each product costs 110 cycles in place of 40.
    if (elect_one()) {
      Run<TREE> run(w, place, steps);
      Segment seg;
      uint32_t used0 = 0, used1 = 0, segs = 0;
      Slot at{0, 0};
      const uint64_t ring_k = sdesc_k128(smem_u32(ring)), q0 = sdesc_k128(smem_u32(smem)), q1 = sdesc_k128(smem_u32(smem + L::Q_TILE));
      bool ok = true;
      while (ok && run.next(seg)) {
        ok = mbar_wait(q_full, segs++ & 1u, ctl, abort_flag);
        const bool split = seg.split();
        const int end0 = min(seg.kt1, seg.n_tile[0]), end1 = min(seg.kt1, seg.n_tile[1]);
        for (int kt = seg.kt0; ok && kt < seg.kt1; ++kt, at.advance(S)) {
          ok = mbar_wait(&full[at.slot], at.parity, ctl, abort_flag);
          const uint64_t kd = ring_k + at.slot * (L::TILE >> 4);
          auto scores = [&](int x, uint32_t& used) {
            if (!ok || (split ? ((kt - seg.kt0) & 1) != x : kt >= (x ? end1 : end0))) return;
            const uint32_t buf = 2 * x + (used & 1u);
            // the product with the P that lies there is done
            if (used >= 2) ok = mbar_wait(&pv_done[buf], ((used >> 1) - 1) & 1u, ctl, abort_flag);
            if (!ok) return;
            tc_fence_after();
            const uint64_t qd = split || x == 0 ? q0 : q1;
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              mma_bf16_ss(tmem + buf * BN, qd + (((k / 4) * L::Q_BLOCK + (k % 4) * 32) >> 4), kd + (((k / 4) * L::BLOCK + (k % 4) * 32) >> 4), IDESC_S,
                          k > 0 ? 1u : 0u);
            mma_commit(&s_full[buf]);
            ++used;
          };
          scores(0, used0);
          scores(1, used1);
          if (ok) mma_commit(&empty[at.slot]);
        }
        if (ok) mma_commit(q_empty);
      }
      // all products must be done before TMEM is freed
      mma_commit(drain);
      drain_wait(drain, 0, ctl);
    }
    __syncwarp();
  } else if (warp < 4) {
    // ------------------------------------------------------------ products of tile x with the values
    const int x = warp - 2;
    if (elect_one()) {
      Run<TREE> run(w, place, steps);
      Segment seg;
      uint32_t used = 0, units = 0;
      Slot at{1, 0};
      const uint64_t ring_v = sdesc_values(smem_u32(ring));
      bool ok = true;
      while (ok && run.next(seg)) {
        bool first = true;
        const bool split = seg.split();
        const int end = min(seg.kt1, seg.n_tile[x]);
        for (int kt = seg.kt0; ok && kt < seg.kt1; ++kt, at.advance(S)) {
          ok = mbar_wait(&full[at.slot], at.parity, ctl, abort_flag);
          if (!ok) break;
          if (split ? ((kt - seg.kt0) & 1) != x : kt >= end) {
            mbar_arrive(&empty[at.slot]);
            continue;
          }
          if ((kt + 1) * BN > seg.seq.Lk) mbar_arrive(&v_tail[x]);
          if (first) ok = mbar_wait(&o_free[x], (units++ & 1u) ^ 1u, ctl, abort_flag);  // O of the unit before has been read
          const uint32_t buf = 2 * x + (used & 1u);
          ok = ok && mbar_wait(&p_full[buf], (used >> 1) & 1u, ctl, abort_flag);
          if (!ok) break;
          tc_fence_after();
          const uint64_t vd = ring_v + at.slot * (L::TILE >> 4);
#pragma unroll
          for (int k = 0; k < 2 * (BN / 16); ++k)  // the weights, and their rests
            mma_bf16_ts(tmem + L::O_COL + x * D, tmem + buf * BN + k * 8, vd + ((k % (BN / 16) * 2048) >> 4), IDESC_O, first && k == 0 ? 0u : 1u);
          mma_commit(&pv_done[buf]);
          mma_commit(&empty[at.slot]);
          if (split ? kt + 2 >= seg.kt1 : kt + 1 == end) mma_commit(&o_full[x]);
          first = false;
          ++used;
        }
      }
      mma_commit(drain);
      drain_wait(drain, 0, ctl);
    }
    __syncwarp();
  } else {
    // ------------------------------------------------------------ softmax
    const int x = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;  // TMEM lane
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t s_addr = tmem + lanes + 2 * x * BN, o_addr = tmem + lanes + L::O_COL + x * D;
    const int token_in = row / w.group, head_in = row % w.group;
    uint32_t step = 0, used = 0;      // steps of the run, and of this tile
    uint32_t outs = 0, exchanges = 0, tails = 0;
    bool ok = true;
    Run<TREE> run(w, place, steps);
    Segment seg;
    while (ok && run.next(seg)) {
      const bool split = seg.split(), mine = seg.active(x);
      const int token = (2 * seg.block + (split ? 0 : x)) * w.tokens + token_in;
      const bool real = row < w.tokens * w.group && token < seg.seq.Lq;
      float m = -INFINITY, z = 0.f;
      if (mine) {
        const int Lk = seg.seq.Lk, prefix = seg.seq.prefix;
        const int lim = !TREE && w.causal ? min(token + 1 + Lk - seg.seq.Lq, Lk) : Lk;
        unsigned long long word = 0;
        if (TREE && real) word = w.words ? static_cast<unsigned long long>(__ldg(w.words + seg.b * w.word_stride + token)) : ~0ull >> (63 - token);
        const int clear = TREE ? min(prefix, Lk) : lim;  // keys below it are read without a look at the mask
        const int kt_first = seg.kt0 + (split ? x : 0), kt_step = split ? 2 : 1, kt_end = split ? seg.kt1 : min(seg.kt1, seg.n_tile[x]);
        for (int kt = kt_first; kt < kt_end; kt += kt_step, ++used) {
          const uint32_t buf = used & 1u;
          if (!warp_wait(&s_full[2 * x + buf], (used >> 1) & 1u, ctl, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          float s[BN];
          tmem_ld32(s_addr + buf * BN, *reinterpret_cast<float(*)[32]>(s));
          tmem_ld32(s_addr + buf * BN + 32, *reinterpret_cast<float(*)[32]>(s + 32));
          tmem_wait_ld();
          const int j0 = kt * BN;
          if (__any_sync(0xffffffffu, j0 + BN > clear)) {
            uint32_t bits[BN / 32];
            key_bits<TREE>(bits, j0, lim, prefix, word);
#pragma unroll
            for (int e = 0; e < BN; ++e)
              if (!(bits[e / 32] >> (e % 32) & 1u)) s[e] = -INFINITY;
            // a product takes 0 x value for a key that no row reads: values behind the sequence must be finite.  v_tail says
            // which phase of the slot is the one to look at
            if (j0 + BN > Lk) {
              const uint32_t at = 2 * (step + kt - seg.kt0) + 1;
              ok = warp_wait(&v_tail[x], tails++ & 1u, ctl, abort_flag) && warp_wait(&full[at % S], (at / S) & 1u, ctl, abort_flag);
              if (!ok) break;
              if (row < BN && j0 + row >= Lk) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                  uint4* p = reinterpret_cast<uint4*>(ring + (at % S) * L::TILE + r * L::BLOCK + row * 128);
#pragma unroll
                  for (int c = 0; c < 8; ++c) p[c] = make_uint4(0u, 0u, 0u, 0u);
                }
              }
              fence_proxy_async_smem();
            }
          }
          float tops[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            tops[i] = s[16 * i];
#pragma unroll
            for (int e = 1; e + 1 < 16; e += 2) tops[i] = max3f(tops[i], s[16 * i + e], s[16 * i + e + 1]);
            tops[i] = fmaxf(tops[i], s[16 * i + 15]);
          }
          const float top = fmaxf(max3f(tops[0], tops[1], tops[2]), tops[3]);
          const bool raise = top > m + kRaise || (m == -INFINITY && top > -INFINITY);
          float alpha = 1.f;
          if (__any_sync(0xffffffffu, raise)) {
            if (raise) {
              if (m > -INFINITY) alpha = exp2_fast((m - top) * kLog2e);
              m = top;
              z *= alpha;
            }
            if (kt > kt_first && __any_sync(0xffffffffu, alpha != 1.f)) {
              // O is between two products: the one before this step's is done
              if (!warp_wait(&pv_done[2 * x + (buf ^ 1u)], ((used - 1) >> 1) & 1u, ctl, abort_flag)) {
                ok = false;
                break;
              }
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                uint32_t o[16];
                asm volatile(
                    "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                    : "=r"(o[0]), "=r"(o[1]), "=r"(o[2]), "=r"(o[3]), "=r"(o[4]), "=r"(o[5]), "=r"(o[6]), "=r"(o[7]), "=r"(o[8]), "=r"(o[9]), "=r"(o[10]),
                      "=r"(o[11]), "=r"(o[12]), "=r"(o[13]), "=r"(o[14]), "=r"(o[15])
                    : "r"(o_addr + c));
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                tmem_st16(o_addr + c, o);
              }
            }
          }
          const float ml = m == -INFINITY ? 0.f : m * kLog2e;
          const F2 scale = f2(kLog2e, kLog2e), minus = f2(-ml, -ml);
          F2 sum[2] = {f2(0.f, 0.f), f2(0.f, 0.f)};
#pragma unroll
          for (int c = 0; c < BN / 32; ++c) {
            uint32_t p[16], rest[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const F2 d = fma2(f2(s[32 * c + 2 * e], s[32 * c + 2 * e + 1]), scale, minus);
              const float a = exp2_fast(lo(d)), b = exp2_fast(hi(d));
              p[e] = pack2(a, b);
              rest[e] = pack2(a - __uint_as_float(p[e] << 16), b - __uint_as_float(p[e] & 0xffff0000u));
              sum[e & 1] = add2(sum[e & 1], f2(a, b));
            }
            tmem_st16(s_addr + buf * BN + 16 * c, p);
            tmem_st16(s_addr + buf * BN + BN / 2 + 16 * c, rest);
          }
          const F2 both = add2(sum[0], sum[1]);
          z += lo(both) + hi(both);
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (elect_one()) mbar_arrive(&p_full[2 * x + buf]);
        }
        if (!ok) break;
      }
      if (mine && !warp_wait(&o_full[x], outs++ & 1u, ctl, abort_flag)) {  // the last product is done
        ok = false;
        break;
      }
      tc_fence_after();
      step += seg.kt1 - seg.kt0;
      float f0 = 1.f, f1 = 0.f;  // of the two outputs of a split unit
      if (split && seg.active(1)) {
        // the second group hands its rows' maxima and sums over, and the first one adds up
        if (x == 1) {
          exch[row] = make_float2(m, z);
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(exch_full);
        } else {
          if (!warp_wait(exch_full, exchanges & 1u, ctl, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const float2 e = exch[row];
          const float both = fmaxf(m, e.x), base = both == -INFINITY ? 0.f : both;
          f0 = z == 0.f ? 0.f : exp2_fast((m - base) * kLog2e);
          f1 = e.y == 0.f ? 0.f : exp2_fast((e.x - base) * kLog2e);
          z = (z == 0.f ? 0.f : z * f0) + (e.y == 0.f ? 0.f : e.y * f1);
          m = both;
        }
        ++exchanges;
      }
      if (split && x == 1) continue;
      const bool two = split && seg.active(1);
      auto sums = [&](int c, float (&o)[32]) {  // 32 columns of the row's weighted values
        tmem_ld32(o_addr + c, o);
        if (two) {
          float p[32];
          tmem_ld32(o_addr + D + c, p);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = o[e] * f0 + p[e] * f1;
        } else {
          tmem_wait_ld();
        }
      };
      if (seg.whole()) {
        const float f = z == 0.f ? 0.f : 1.f / z;
        const int head = seg.h * w.group + head_in;
        __nv_bfloat16* out = w.out + (TREE ? (static_cast<size_t>(seg.b) * w.Hq + head) * w.T + token : static_cast<size_t>(seg.seq.q0 + token) * w.Hq + head) * D;
        // Rows lie apart: a lane that stored its own row would make a warp's store touch 32 lines, which the load/store unit
        // takes one a cycle (4,700 cycles a unit of 128 columns, 3,600 this way).  Prompts' rows go through shared memory, eight lanes to a row.
        if (mine) {
#pragma unroll 1
          for (int c = 0; c < D; c += TREE ? 32 : 64) {
            uint32_t u[32];
#pragma unroll
            for (int h = 0; h < (TREE ? 1 : 2); ++h) {
              float o[32];
              sums(c + 32 * h, o);
#pragma unroll
              for (int e = 0; e < 16; ++e) u[16 * h + e] = z == 0.f ? 0u : pack2(o[2 * e] * f, o[2 * e + 1] * f);
            }
            if constexpr (TREE) {
              if (real) {
#pragma unroll
                for (int e = 0; e < 4; ++e) reinterpret_cast<uint4*>(out + c)[e] = make_uint4(u[4 * e], u[4 * e + 1], u[4 * e + 2], u[4 * e + 3]);
              }
            } else {
              uint8_t* stage = smem + L::OFF_STAGE + (warp - 4) * L::STAGE;
              __syncwarp();  // what was there has been read
#pragma unroll
              for (int e = 0; e < 8; ++e)
                *reinterpret_cast<uint4*>(stage + lane * 128 + ((e ^ (lane & 7)) << 4)) = make_uint4(u[4 * e], u[4 * e + 1], u[4 * e + 2], u[4 * e + 3]);
              __syncwarp();
              const unsigned long long mine_at = real ? reinterpret_cast<unsigned long long>(out + c) : 0ull;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int r = 4 * e + lane / 8, chunk = lane % 8;
                const unsigned long long at = __shfl_sync(0xffffffffu, mine_at, r);
                const uint4 v = *reinterpret_cast<const uint4*>(stage + r * 128 + ((chunk ^ (r & 7)) << 4));
                if (at) reinterpret_cast<uint4*>(at)[chunk] = v;
              }
            }
          }
        }
      } else {
        // the run's first unit goes to its first part, unless it begins with it
        float* part = w.parts + (2 * static_cast<size_t>(blockIdx.x) + (seg.kt0 > 0 ? 0 : 1)) * kPartFloats<D>;
        const int at = x * BM + row;
        if (mine) {
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            sums(c, o);
            if (real) {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                reinterpret_cast<float4*>(part)[(c / 4 + e) * 256 + at] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
            }
          }
        }
        part[256 * D + at] = m;
        part[256 * D + 256 + at] = z;
      }
      if (mine) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&o_free[x]);
          if (two) mbar_arrive(&o_free[1]);
        }
      }
    }
    if (!TREE && w.clear_rest) {
      // rows of no sequence
      const int first = min(max(__ldg(w.q_starts), 0), w.Tq), last = max(first, min(max(__ldg(w.q_starts + w.B), 0), w.Tq));
      const long long row_words = static_cast<long long>(w.Hq) * D / 8, n = row_words * (first + w.Tq - last);
      for (long long i = blockIdx.x * 256 + (threadIdx.x - 128); i < n; i += gridDim.x * 256)
        reinterpret_cast<uint4*>(w.out)[i < first * row_words ? i : i + (last - first) * row_words] = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, L::COLS);
  }
}

// Joins a unit's parts.  Block (i, y) looks at the place where CTA i + 1's run begins: where that is the first such place
// inside its unit, it adds up the unit's parts, for 4 2^fours of the columns and 32 of the rows.  Few rows of many parts (one token over
// a long cache) are shared out over the parts, and the shares added in order.  The time is that of a few loads behind one
// another: 18 us for 151 units of 256 rows and 2 or 3 parts, 6 for single tokens of 4 sequences.
template <int D, bool TREE>
__global__ void __launch_bounds__(256) grouped_join_kernel(const __grid_constant__ Work w, int fours) {
  __shared__ float weight[kMostParts][32];  // a part's maximum, -inf where it has no key; then what its O counts for
  __shared__ long long to[32];              // where the rows go in out
  __shared__ float4 share[256];
  __shared__ float2 shared[8][32];  // the maximum and the sum over every eighth part
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int i = blockIdx.x + 1;
  const Place p = w.places[i];
  if (i >= p.ctas || p.kt == 0) return;
  const long long first = run_start(p.total, p.ctas, i) - p.kt, last = first + p.tiles;
  if (run_start(p.total, p.ctas, i - 1) > first) return;
  // rows of this block: at most 32 of tile x
  const int slices = D / 4 >> fours, c0 = blockIdx.y % slices << (fours + 2), at0 = blockIdx.y / slices * 32, x = at0 / BM, row0 = at0 % BM;
  const int t0 = (2 * p.block + x) * w.tokens;
  const int rows = min(32, min(w.tokens, p.Lq - t0) * w.group - row0);
  if (rows <= 0) return;
  // CTAs i - 1 .. end - 1 have parts: run_start(end) is the first that is not below `last`
  const int end = min(p.ctas, static_cast<int>(quotient(last * p.ctas + p.total - 1, p.total)));
  const int parts = end - i + 1;
  const auto part = [&](int k) { return w.parts + (2 * static_cast<size_t>(i - 1 + k) + (k == 0 ? 1 : 0)) * kPartFloats<D>; };

  // a row's maxima and sums, every eighth part's by a thread, four on their way at once
  const int row = threadIdx.x % 32, group = threadIdx.x / 32;
  float2 mine = make_float2(-INFINITY, 0.f);
  for (int k0 = group; k0 < parts; k0 += 32) {
    float mk[4], zk[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const bool in = k0 + 8 * t < parts && row < rows;
      const float* p = part(k0 + 8 * t) + 256 * D + at0 + row;
      mk[t] = in ? __ldcg(p) : -INFINITY, zk[t] = in ? __ldcg(p + 256) : 0.f;
    }
    float m = mine.x;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (k0 + 8 * t < parts) weight[k0 + 8 * t][row] = zk[t] == 0.f ? -INFINITY : mk[t];
      m = fmaxf(m, mk[t]);
    }
    const float base = m == -INFINITY ? 0.f : m;
    float z = mine.y == 0.f ? 0.f : mine.y * exp2_fast((mine.x - base) * kLog2e);
#pragma unroll
    for (int t = 0; t < 4; ++t) z += zk[t] == 0.f ? 0.f : zk[t] * exp2_fast((mk[t] - base) * kLog2e);
    mine = make_float2(m, z);
  }
  shared[group][row] = mine;
  __syncthreads();
  {
    const int lists = min(8, parts);
    float m = -INFINITY, z = 0.f;
    for (int g = 0; g < lists; ++g) m = fmaxf(m, shared[g][row].x);
    const float base = m == -INFINITY ? 0.f : m;
    for (int g = 0; g < lists; ++g) z += shared[g][row].y == 0.f ? 0.f : shared[g][row].y * exp2_fast((shared[g][row].x - base) * kLog2e);
    const float f = z == 0.f ? 0.f : 1.f / z;
    for (int k = group; k < parts; k += 8) {
      const float top = weight[k][row];
      weight[k][row] = top == -INFINITY && z == z ? 0.f : exp2_fast((top - base) * kLog2e) * f;
    }
    if (group == 0) {
      const int token = t0 + (row0 + row) / w.group, head = p.h * w.group + (row0 + row) % w.group;
      to[row] = (TREE ? (static_cast<long long>(p.b) * w.Hq + head) * w.T + token : static_cast<long long>(p.q0 + token) * w.Hq + head) * D + c0;
    }
  }
  __syncthreads();

  // 2^fours columns of four for each row; the rest of the block's threads take other parts
  const int bits = 32 - __clz(rows - 1), wide = 1 << bits;  // rows <= wide <= 32
  const int items = wide << fours, lanes = max(1, 256 / items);  // lanes: over the parts
  for (int j = threadIdx.x; j < items * lanes; j += 256) {
    const int r = j & (wide - 1), c = j >> bits & ((1 << fours) - 1), lane = j >> (bits + fours);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows)
      for (int k0 = lane; k0 < parts; k0 += 4 * lanes) {
        float4 v[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int k = k0 + t * lanes;
          if (k < parts && weight[k][r] != 0.f) v[t] = __ldcg(reinterpret_cast<const float4*>(part(k)) + (c0 / 4 + c) * 256 + at0 + r);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const int k = k0 + t * lanes;
          const float f = k < parts ? weight[k][r] : 0.f;
          if (f != 0.f) o.x += v[t].x * f, o.y += v[t].y * f, o.z += v[t].z * f, o.w += v[t].w * f;
        }
      }
    if (lanes > 1) {
      share[threadIdx.x] = o;
      __syncthreads();
      for (int l = 1; l < lanes && lane == 0; ++l) {
        const float4 v = share[threadIdx.x + l * items];
        o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w;
      }
    }
    if (lane == 0 && r < rows) *reinterpret_cast<uint2*>(w.out + to[r] + 4 * c) = make_uint2(pack2(o.x, o.y), pack2(o.z, o.w));
  }
}

// bf16 [n3][n2][n1][n0], strides in elements, boxes of 64 x b1 x b2 elements.
bool make_map(CUtensorMap* map, const void* base, uint64_t n0, uint64_t n1, long long s1, uint64_t n2, long long s2, uint64_t n3, long long s3, uint32_t b1,
              uint32_t b2) {
  const cuuint64_t dims[4] = {n0, n1, n2, n3};
  // the stride of an axis of one is never used
  const cuuint64_t strides[3] = {(n1 > 1 ? static_cast<cuuint64_t>(s1) : n0) * 2, (n2 > 1 ? static_cast<cuuint64_t>(s2) : n0) * 2,
                                 (n3 > 1 ? static_cast<cuuint64_t>(s3) : n0) * 2};
  const cuuint32_t box[4] = {64, b1, b2, 1}, one[4] = {1, 1, 1, 1};
  return encode_tiled_fn()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool TREE>
int launch(const CUtensorMap& tmq, const CUtensorMap& tmk, const CUtensorMap& tmv, const Work& w, int grid, int fours, const DevCtl& ctl, cudaStream_t st) {
  using L = Layout<D, TREE>;
  const auto kernel = grouped_kernel<D, TREE>;
  int device = 0;
  static std::atomic<unsigned long long> ready{0};  // a bit for each device whose kernel may take the shared memory
  if (cudaGetDevice(&device) != cudaSuccess) return -1;
  if (device > 63 || !(ready.load(std::memory_order_acquire) >> device & 1ull)) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(L::BYTES)) != cudaSuccess) return -1;
    if (device <= 63) ready.fetch_or(1ull << device, std::memory_order_release);
  }
  kernel<<<grid, kThreads, L::BYTES, st>>>(tmq, tmk, tmv, w, ctl);
  if (cudaGetLastError() != cudaSuccess) return -1;
  if (grid == 1) return 1;
  cudaLaunchConfig_t config = {};
  // rows that a unit can have: the second tile's begin at 128
  const int rows = TREE && w.T <= w.tokens ? w.T * w.group : 2 * BM;
  config.gridDim = dim3(grid - 1, (D / 4 >> fours) * ((rows + 31) / 32)), config.blockDim = dim3(256), config.stream = st;
  cudaLaunchAttribute early = {};
  early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  early.val.programmaticStreamSerializationAllowed = 1;
  config.attrs = &early, config.numAttrs = 1;
  return cudaLaunchKernelEx(&config, grouped_join_kernel<D, TREE>, w, fours) == cudaSuccess ? 2 : -1;
}

}  // namespace

size_t grouped_workspace_bytes(int d, int num_sms) {
  return num_sms * (2 * (d == 64 ? kPartFloats<64> : kPartFloats<128>) * sizeof(float) + sizeof(Place));
}

int prompt_attn(const topk_prompt_args& a, void* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  if (!encode_tiled_fn() || num_sms > kMostParts) return -1;
  Work w = {};
  w.q_starts = a.q_starts, w.k_starts = a.k_starts ? a.k_starts : a.q_starts;
  w.out = static_cast<__nv_bfloat16*>(a.out), w.parts = static_cast<float*>(workspace);
  w.places = reinterpret_cast<Place*>(w.parts + num_sms * 2 * (a.d == 64 ? kPartFloats<64> : kPartFloats<128>));
  w.B = a.B, w.Hq = a.Hq, w.Hkv = a.Hkv, w.group = a.Hq / a.Hkv, w.Tq = a.Tq, w.Tk = a.Tk, w.causal = a.causal, w.clear_rest = a.clear_rest;
  w.tokens = BM / w.group;
  CUtensorMap q, k, v;
  if (!make_map(&q, a.q, a.d, a.Hq, a.q_stride[1], a.Tq, a.q_stride[0], 1, 0, w.group, w.tokens) ||
      !make_map(&k, a.k, a.d, a.Tk, a.k_stride[0], a.Hkv, a.k_stride[1], 1, 0, BN, 1) ||
      !make_map(&v, a.v, a.d, a.Tk, a.v_stride[0], a.Hkv, a.v_stride[1], 1, 0, BN, 1))
    return -1;
  return a.d == 64 ? launch<64, false>(q, k, v, w, num_sms, 4, ctl, st) : launch<128, false>(q, k, v, w, num_sms, 4, ctl, st);
}

int tree_attn(const topk_tree_args& a, void* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  if (!encode_tiled_fn() || num_sms > kMostParts) return -1;
  Work w = {};
  w.kv_len = a.kv_len, w.words = a.tree, w.word_stride = a.tree_stride;
  w.out = static_cast<__nv_bfloat16*>(a.out), w.parts = static_cast<float*>(workspace);
  w.places = reinterpret_cast<Place*>(w.parts + num_sms * 2 * (a.d == 64 ? kPartFloats<64> : kPartFloats<128>));
  w.B = a.B, w.Hq = a.Hq, w.Hkv = a.Hkv, w.group = a.Hq / a.Hkv, w.T = a.T, w.cap = a.cap;
  w.tokens = BM / w.group;
  CUtensorMap q, k, v;
  if (!make_map(&q, a.q, a.d, a.Hq, a.q_stride[1], a.T, a.q_stride[2], a.B, a.q_stride[0], w.group, w.tokens) ||
      !make_map(&k, a.keys, a.d, a.cap, a.key_stride[2], a.Hkv, a.key_stride[1], a.B, a.key_stride[0], BN, 1) ||
      !make_map(&v, a.values, a.d, a.cap, a.value_stride[2], a.Hkv, a.value_stride[1], a.B, a.value_stride[0], BN, 1))
    return -1;
  const long long units = static_cast<long long>(a.B) * a.Hkv * ((a.T + 2 * w.tokens - 1) / (2 * w.tokens)), most = units * ((a.cap + BN - 1) / BN);  // key tiles
  const int grid = static_cast<int>(most < num_sms ? most : num_sms);
  // units of 16 parts and more are joined by blocks of 16 columns: 2 units of six rows over up to 55,568 keys
  // take 22 us in place of 28; 48 units (single tokens of 4 sequences), of four parts, would take 27 in place of 25
  const int fours = units * 16 <= grid ? 2 : 4;
  return a.d == 64 ? launch<64, true>(q, k, v, w, grid, fours, ctl, st) : launch<128, true>(q, k, v, w, grid, fours, ctl, st);
}

}  // namespace topk
