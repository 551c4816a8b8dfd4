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
//   g = R^T dout,  dw += g x r,  u = g w,  dx = r (u - x r^2 mean(u x)).
//
// Every element is read once and written once: the floor is HBM's.  G = d / 8 lanes
// (rounded up to a power of two) own a row, eight elements each, chosen so that both
// members of a pair sit in one lane: the rotation needs no exchange, and the norm one
// butterfly over the G lanes.  A warp takes some heads of one kind (q, k or v) of one
// token, with all their loads in flight at once, and the token's angles serve them all;
// the warps of a block take neighbouring tokens, whose rows of a head are neighbours in the
// output.  What is left beside HBM is the chain position -> table row -> product and the
// issue of some hundred instructions a row: positions go out before anything else and are
// checked when they are used, and products run in pairs (f32x2).
#include <cuda_bf16.h>

#include "kernels.h"
#include "pairs.cuh"

namespace topk {

namespace {

constexpr int kWarps = 8;  // tokens of a block at a time
constexpr unsigned kFull = 0xffffffffu;
// Measured on 65,536 tokens x 36 heads of 64 (bf16) forward, and 32,768 x 48 heads of 128 (fp32 gradients)
// backward: 106 and 234 us with these (5.9 and 6.3 TB/s, 86 and 93 % of a copy's rate).  More forward blocks per SM
// spill registers (151 us); blocks of a single token (no walk) wait for position and table in turn (135 us).  Backward,
// rows held in registers take 262 us (fp32 rows 285 against 173 for 16,384 x 48 heads of 128), three blocks per
// SM of fewer rows 322.
constexpr int kFwdBlocksPerSm = 4, kBwdBlocksPerSm = 2;
constexpr int kRowsPerLane = 4;  // at most, held at once (fp32: two)
constexpr int kWaves = 4;        // blocks for each place on the GPU: values cost less than queries, and are not waited for

__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
  const float4 f = *reinterpret_cast<const float4*>(p);
  v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
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
  int axis, split;  // the axis of its first pair, and how many of its four pairs (or more) are on it
  bool on, rotated;
};

__device__ __forceinline__ int axis_of(const QkArgs& p, int pair) {
  int axis = 0;
  for (int x = 0; x + 1 < p.axes; ++x) axis += pair >= p.bound[x];
  return axis;
}

__device__ __forceinline__ Lane lane_of(const QkArgs& p, int j) {
  Lane l;
  l.on = 8 * j < p.d;
  l.rotated = 8 * j < p.rot;
  const bool half = l.rotated && !p.interleaved;
  l.a = half ? 4 * j : 8 * j;
  l.b = half ? p.rot / 2 + 4 * j : 8 * j + 4;
  l.axis = axis_of(p, 4 * j);
  l.split = p.positions && p.axes > 1 ? p.bound[l.axis] - 4 * j : 4;
  return l;
}

// A lane's eight values of a row: [a, a + 4) in x[0], x[1] and [b, b + 4) in x[2], x[3].
struct Eight {
  F2 x[4];
};

// The same as they lie in memory: a bf16 row takes half the registers while it is in flight.
template <typename T>
struct Raw;
template <>
struct Raw<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p, const Lane& l) {
    a = *reinterpret_cast<const float4*>(p + l.a);
    b = *reinterpret_cast<const float4*>(p + l.b);
  }
  __device__ __forceinline__ void from(const uint8_t* pa, const uint8_t* pb) {
    a = *reinterpret_cast<const float4*>(pa);
    b = *reinterpret_cast<const float4*>(pb);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ Eight get() const { return {f2(a.x, a.y), f2(a.z, a.w), f2(b.x, b.y), f2(b.z, b.w)}; }
  __device__ __forceinline__ void set(const Eight& v) {
    a = make_float4(lo(v.x[0]), hi(v.x[0]), lo(v.x[1]), hi(v.x[1]));
    b = make_float4(lo(v.x[2]), hi(v.x[2]), lo(v.x[3]), hi(v.x[3]));
  }
  __device__ __forceinline__ void store(float* p, const Lane& l) const {
    *reinterpret_cast<float4*>(p + l.a) = a;
    *reinterpret_cast<float4*>(p + l.b) = b;
  }
};
template <>
struct Raw<__nv_bfloat16> {
  uint2 a, b;
  __device__ __forceinline__ void load(const __nv_bfloat16* p, const Lane& l) {
    a = *reinterpret_cast<const uint2*>(p + l.a);
    b = *reinterpret_cast<const uint2*>(p + l.b);
  }
  __device__ __forceinline__ void from(const uint8_t* pa, const uint8_t* pb) {
    a = *reinterpret_cast<const uint2*>(pa);
    b = *reinterpret_cast<const uint2*>(pb);
  }
  __device__ __forceinline__ void zero() { a = b = make_uint2(0u, 0u); }
  static __device__ __forceinline__ F2 wide(uint32_t u) { return f2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u)); }
  // the one rounding of a result, to nearest
  static __device__ __forceinline__ uint32_t narrow(F2 v) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo(v), hi(v));
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  __device__ __forceinline__ Eight get() const { return {wide(a.x), wide(a.y), wide(b.x), wide(b.y)}; }
  __device__ __forceinline__ void set(const Eight& v) {
    a = make_uint2(narrow(v.x[0]), narrow(v.x[1]));
    b = make_uint2(narrow(v.x[2]), narrow(v.x[3]));
  }
  __device__ __forceinline__ void store(__nv_bfloat16* p, const Lane& l) const {
    *reinterpret_cast<uint2*>(p + l.a) = a;
    *reinterpret_cast<uint2*>(p + l.b) = b;
  }
};

// A lane's pieces of the next token, copied into shared memory while it works on one: they take no registers, and only
// the lane that asked for a piece reads it, so that its own wait is enough.  Nothing is read for a piece that is not
// `on`; it is zero.
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool on) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(on ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until all but the newest group have landed.
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group 1;" ::: "memory"); }

// The positions of the lane's four pairs 4j .. 4j + 3 for token (b, t), as they are given.  The four lie on one axis, or,
// where an axis ends among them, on two; NARROW: on up to four.  Nothing here may wait for the loads, not even a
// copy: they go out a token ahead.
template <bool NARROW>
struct Positions {
  int row[NARROW ? 4 : 2];
  __device__ __forceinline__ void load(const QkArgs& p, const Lane& l, int j, int b, int t) {
    if (!l.rotated) return;
    if (!p.positions) {
#pragma unroll
      for (int& r : row) r = t;
      return;
    }
    const int32_t* at = p.positions + static_cast<size_t>(b) * p.L + t;
    const size_t axis = static_cast<size_t>(p.B) * p.L;
    if constexpr (NARROW) {
#pragma unroll
      for (int e = 0; e < 4; ++e) row[e] = __ldg(at + axis_of(p, 4 * j + e) * axis);
    } else {
      row[0] = __ldg(at + l.axis * axis);
      if (l.split < 4) row[1] = __ldg(at + axis_of(p, 4 * j + 3) * axis);
    }
  }
};

// The angles of a lane's four pairs; minus the sines too, which a paired product cannot negate.
struct Angles {
  F2 c[2], s[2], m[2];
  __device__ __forceinline__ void set(const float (&cs)[4], const float (&sn)[4]) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      c[e] = f2(cs[2 * e], cs[2 * e + 1]);
      s[e] = f2(sn[2 * e], sn[2 * e + 1]);
      m[e] = f2(-sn[2 * e], -sn[2 * e + 1]);
    }
  }
};

// cos and sin of the four pairs; identity where the lane does not rotate.  A position outside the tables is reported and clamped.
template <bool NARROW>
__device__ __forceinline__ void load_angles(const QkArgs& p, const Lane& l, int j, const Positions<NARROW>& at, const DevCtl& ctl,
                                            Angles& t) {
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
  if (l.rotated) {
    const int half = p.rot / 2, last = p.table_rows - 1;
    bool out = false;
    auto inside = [&](int row) {
      const int r = min(max(row, 0), last);
      out |= r != row;
      return static_cast<size_t>(r) * half + 4 * j;
    };
    if constexpr (NARROW) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const size_t r = inside(at.row[e]) + e;
        c[e] = __ldg(p.cos + r);
        s[e] = __ldg(p.sin + r);
      }
    } else {
      const size_t r = inside(at.row[0]);
      load4(p.cos + r, c);
      load4(p.sin + r, s);
      if (l.split < 4) {
        const size_t r1 = inside(at.row[1]);
        float c1[4], s1[4];
        load4(p.cos + r1, c1);
        load4(p.sin + r1, s1);
#pragma unroll
        for (int e = 1; e < 4; ++e)
          if (e >= l.split) c[e] = c1[e], s[e] = s1[e];
      }
    }
    if (out) atomicOr(ctl.error, kDevErrRange);
  }
  t.set(c, s);
}

// The same in two steps: the copies into shared memory, and the reading of them.
template <bool NARROW>
__device__ __forceinline__ void fetch_angles(const QkArgs& p, const Lane& l, int j, const Positions<NARROW>& at, const DevCtl& ctl,
                                             float* cos_s, float* sin_s) {
  if (!l.rotated) return;
  const int half = p.rot / 2, last = p.table_rows - 1;
  bool out = false;
  auto inside = [&](int row) {
    const int r = min(max(row, 0), last);
    out |= r != row;
    return static_cast<size_t>(r) * half + 4 * j;
  };
  const uint32_t c = smem_u32(cos_s), s = smem_u32(sin_s);
  if (!NARROW && l.split >= 4) {
    const size_t r = inside(at.row[0]);
    copy_async<16>(c, p.cos + r, true);
    copy_async<16>(s, p.sin + r, true);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const size_t r = inside(NARROW ? at.row[NARROW ? e : 0] : (e < l.split ? at.row[0] : at.row[1])) + e;
      copy_async<4>(c + 4 * e, p.cos + r, true);
      copy_async<4>(s + 4 * e, p.sin + r, true);
    }
  }
  if (out) atomicOr(ctl.error, kDevErrRange);
}

__device__ __forceinline__ void read_angles(const Lane& l, const float* cos_s, const float* sin_s, Angles& t) {
  float c[4] = {1.f, 1.f, 1.f, 1.f}, s[4] = {0.f, 0.f, 0.f, 0.f};
  if (l.rotated) {
    load4(cos_s, c);
    load4(sin_s, s);
  }
  t.set(c, s);
}

// Turns the pairs by their angles, or back by the transpose (the other sign of the sines).
template <bool BACK>
__device__ __forceinline__ void rotate(Eight& v, const Angles& t, bool interleaved) {
  if (!interleaved) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const F2 a = v.x[e], b = v.x[e + 2];
      v.x[e] = fma2(b, BACK ? t.s[e] : t.m[e], mul2(a, t.c[e]));
      v.x[e + 2] = fma2(a, BACK ? t.m[e] : t.s[e], mul2(b, t.c[e]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = lo(v.x[e]), y = hi(v.x[e]);
      const float c = e & 1 ? hi(t.c[e / 2]) : lo(t.c[e / 2]), s = e & 1 ? hi(t.s[e / 2]) : lo(t.s[e / 2]);
      v.x[e] = BACK ? f2(x * c + y * s, y * c - x * s) : f2(x * c - y * s, y * c + x * s);
    }
  }
}

template <typename T>
__device__ __forceinline__ Eight load_weight(const void* w, const Lane& l) {
  if (!w || !l.on) return {f2(1.f, 1.f), f2(1.f, 1.f), f2(1.f, 1.f), f2(1.f, 1.f)};
  Raw<T> r;
  r.load(static_cast<const T*>(w), l);
  return r.get();
}

__device__ __forceinline__ float dot8(const Eight& a, const Eight& b) {
  const F2 s = fma2(a.x[0], b.x[0], mul2(a.x[1], b.x[1])), t = fma2(a.x[2], b.x[2], mul2(a.x[3], b.x[3]));
  return (lo(s) + hi(s)) + (lo(t) + hi(t));
}

// A warp's place in the batch, moved along by the grid's stride of tokens without a division a step.
struct Place {
  int b, t;
};

struct Walk {
  int L, db, dt;
  __device__ __forceinline__ Walk(int L_, unsigned stride) : L(L_), db(stride / L_), dt(stride % L_) {}
  __device__ __forceinline__ Place at(unsigned token) const { return {static_cast<int>(token / L), static_cast<int>(token % L)}; }
  __device__ __forceinline__ Place next(Place p) const {
    p.b += db, p.t += dt;
    if (p.t >= L) p.t -= L, ++p.b;
    return p;
  }
};

// A warp's share of a token: `rows` heads of one kind from h0 on, U x R at most.  The groups of a
// token are q's, then k's, then v's.
enum Kind { kQ, kK, kV };

struct Group {
  int kind, h0, rows;
};

__device__ __forceinline__ Group group_of(const QkArgs& p, int g, int size) {
  const int nq = (p.Hq + size - 1) / size, nk = (p.Hkv + size - 1) / size;
  Group o;
  o.kind = g < nq ? kQ : (g < nq + nk ? kK : kV);
  const int i = g - (o.kind == kQ ? 0 : (o.kind == kK ? nq : nq + nk));
  o.h0 = i * size;
  o.rows = min(size, (o.kind == kQ ? p.Hq : p.Hkv) - o.h0);
  return o;
}

template <typename T, int G, int U, bool NARROW>
__global__ void __launch_bounds__(kWarps * 32, kFwdBlocksPerSm)
    qk_fwd_kernel(const __grid_constant__ QkArgs p, T* __restrict__ qo, T* __restrict__ ko, T* __restrict__ vo, int cap,
                  const int32_t* __restrict__ start, DevCtl ctl) {
  constexpr int R = 32 / G;  // rows (heads) of a warp at a time
  const int lane = threadIdx.x & 31, j = lane % G, sub = lane / G;
  const unsigned tokens = static_cast<unsigned>(p.B) * p.L, stride = gridDim.x * kWarps;
  unsigned token = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (token >= tokens) return;
  const Group g = group_of(p, blockIdx.y, R * U);
  const Lane l = lane_of(p, j);
  const bool turns = g.kind != kV;
  Positions<NARROW> at;
  const Walk walk(p.L, stride);
  Place here = walk.at(token);
  if (turns) at.load(p, l, j, here.b, here.t);
  const long long* step = g.kind == kQ ? p.q_stride : (g.kind == kK ? p.k_stride : p.v_stride);
  const T* in = static_cast<const T*>(g.kind == kQ ? p.q : (g.kind == kK ? p.k : p.v)) + (g.h0 + sub) * step[2];
  const int heads = g.kind == kQ ? p.Hq : p.Hkv, rows = g.kind == kQ ? p.L : cap;
  T* const out = (g.kind == kQ ? qo : (g.kind == kK ? ko : vo)) + static_cast<long long>(g.h0 + sub) * rows * p.d;
  const long long out_step = static_cast<long long>(R) * rows * p.d;
  const float scale = g.kind == kQ ? p.q_scale : 1.f, inv_d = 1.f / p.d;
  for (; token < tokens; token += stride) {
    const int b = here.b, t = here.t;
    here = walk.next(here);
    const T* src = in + b * step[0] + t * step[1];
    Raw<T> x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u * R + sub < g.rows && l.on)
        x[u].load(src + u * R * step[2], l);
      else
        x[u].zero();
    }
    // the output row of the group's first head
    long long to = t;
    if (start && g.kind != kQ) {
      to += __ldg(start + b);
      if (to < 0 || to >= cap) {
        if (lane == 0) atomicOr(ctl.error, kDevErrRange);
        to = -1;
      }
    }
    if (turns) {
      Angles turn;
      load_angles(p, l, j, at, ctl, turn);
      if (token + stride < tokens) at.load(p, l, j, here.b, here.t);
      const Eight w = load_weight<T>(g.kind == kQ ? p.q_weight : p.k_weight, l);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        Eight v = x[u].get();
        // one factor a row: the norm's and the scale's (weights are ones without the norm)
        const float r = p.normalize ? rsqrtf(group_sum<G>(dot8(v, v)) * inv_d + p.eps) * scale : scale;
        const F2 rr = f2(r, r);
#pragma unroll
        for (int e = 0; e < 4; ++e) v.x[e] = mul2(mul2(v.x[e], rr), w.x[e]);
        rotate<false>(v, turn, p.interleaved);
        x[u].set(v);
      }
    }
    T* dst = out + (static_cast<long long>(b) * heads * rows + to) * p.d;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (u * R + sub < g.rows && l.on && to >= 0) x[u].store(dst + u * out_step, l);
  }
}

template <typename T, typename GT, int U>
struct BwdStage {
  float4 cos[kWarps * 32], sin[kWarps * 32];
  uint8_t ya[U][kWarps * 32][4 * sizeof(GT)], yb[U][kWarps * 32][4 * sizeof(GT)];
  uint8_t xa[U][kWarps * 32][4 * sizeof(T)], xb[U][kWarps * 32][4 * sizeof(T)];
};

// Backward.  A block keeps one group of heads and walks over tokens in strides of the grid, the next
// token's rows and angles being copied into shared memory meanwhile, so that its lanes sum their eight elements' weight gradient in registers; at the end the
// block adds its lanes up in a fixed order and writes one partial row.
// qk_bwd_weights_kernel adds the partial rows: the result does not depend on the order in
// which blocks run.
template <typename T, typename GT, int G, int U, bool NARROW>
__global__ void __launch_bounds__(kWarps * 32, kBwdBlocksPerSm)
    qk_bwd_kernel(const __grid_constant__ QkArgs p, const GT* __restrict__ dq, const GT* __restrict__ dk, const GT* __restrict__ dv,
                  T* __restrict__ dqkv, float* __restrict__ partial, DevCtl ctl) {
  constexpr int R = 32 / G;
  extern __shared__ __align__(16) uint8_t smem[];
  BwdStage<T, GT, U>* stages = reinterpret_cast<BwdStage<T, GT, U>*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, j = lane % G, sub = lane / G;
  const int all = p.Hq + (dv ? 2 : 1) * p.Hkv;
  const unsigned tokens = static_cast<unsigned>(p.B) * p.L, stride = gridDim.x * kWarps;
  const Lane l = lane_of(p, j);
  const Group g = group_of(p, blockIdx.y, R * U);
  const int heads = g.kind == kQ ? p.Hq : p.Hkv;
  const GT* grad = (g.kind == kQ ? dq : (g.kind == kK ? dk : dv)) + static_cast<long long>(g.h0 + sub) * p.L * p.d;
  const long long* step = g.kind == kQ ? p.q_stride : p.k_stride;
  const T* in = static_cast<const T*>(g.kind == kQ ? p.q : p.k) + (g.h0 + sub) * step[2];
  T* const out = dqkv + static_cast<long long>((g.kind == kQ ? 0 : (g.kind == kK ? p.Hq : p.Hq + p.Hkv)) + g.h0 + sub) * p.d;
  const bool turns = g.kind != kV, norm = p.normalize && turns;
  const Eight w = load_weight<T>(g.kind == kQ ? p.q_weight : p.k_weight, l);
  const float scale = g.kind == kQ ? p.q_scale : 1.f, inv_d = 1.f / p.d;
  Eight dw = {f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f), f2(0.f, 0.f)};
  Positions<NARROW> at;
  unsigned token = blockIdx.x * kWarps + warp;
  const Walk walk(p.L, stride);
  auto fetch = [&](Place o, int s) {
    const GT* gs = grad + (static_cast<long long>(o.b) * heads * p.L + o.t) * p.d;
    const T* xs = in + o.b * step[0] + o.t * step[1];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool on = u * R + sub < g.rows && l.on;
      const GT* yr = on ? gs + static_cast<long long>(u * R) * p.L * p.d : dq;
      copy_async<4 * sizeof(GT)>(smem_u32(stages[s].ya[u][tid]), yr + (on ? l.a : 0), on);
      copy_async<4 * sizeof(GT)>(smem_u32(stages[s].yb[u][tid]), yr + (on ? l.b : 0), on);
      if (norm) {
        const T* xr = on ? xs + u * R * step[2] : in;
        copy_async<4 * sizeof(T)>(smem_u32(stages[s].xa[u][tid]), xr + (on ? l.a : 0), on);
        copy_async<4 * sizeof(T)>(smem_u32(stages[s].xb[u][tid]), xr + (on ? l.b : 0), on);
      }
    }
    if (turns) fetch_angles(p, l, j, at, ctl, &stages[s].cos[tid].x, &stages[s].sin[tid].x);
  };
  Place next_at = {0, 0};  // of the token after the one worked on
  if (token < tokens) {
    const Place first = walk.at(token);
    if (turns) at.load(p, l, j, first.b, first.t);
    fetch(first, 0);
    next_at = walk.next(first);
    if (turns && token + stride < tokens) at.load(p, l, j, next_at.b, next_at.t);
  }
  copies_commit();
  for (int s = 0; token < tokens; token += stride, s ^= 1) {
    const unsigned next = token + stride;
    if (next < tokens) {
      fetch(next_at, s ^ 1);
      next_at = walk.next(next_at);
      if (turns && next + stride < tokens) at.load(p, l, j, next_at.b, next_at.t);
    }
    copies_commit();
    copies_wait();
    Angles turn;
    if (turns) read_angles(l, &stages[s].cos[tid].x, &stages[s].sin[tid].x, turn);
    T* dst = out + static_cast<long long>(token) * all * p.d;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      Raw<GT> y;
      y.from(stages[s].ya[u][tid], stages[s].yb[u][tid]);
      Eight v = y.get();
      if (turns) rotate<true>(v, turn, p.interleaved);
      if (norm) {
        Raw<T> x;
        x.from(stages[s].xa[u][tid], stages[s].xb[u][tid]);
        Eight z = x.get(), vz;
#pragma unroll
        for (int e = 0; e < 4; ++e) vz.x[e] = mul2(v.x[e], z.x[e]);
        const float ss = group_sum<G>(dot8(z, z)), ux = group_sum<G>(dot8(vz, w));
        // rows that are not there are zeros, whose root has no reciprocal without eps
        const float r = u * R + sub < g.rows ? rsqrtf(ss * inv_d + p.eps) : 0.f, k = -r * r * ux * inv_d;
        const F2 rr = f2(r * scale, r * scale), kk = f2(k, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          dw.x[e] = fma2(vz.x[e], rr, dw.x[e]);
          v.x[e] = mul2(rr, fma2(z.x[e], kk, mul2(v.x[e], w.x[e])));
        }
      } else if (turns) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v.x[e] = mul2(v.x[e], f2(scale, scale));
      }
      if (u * R + sub >= g.rows || !l.on) continue;
      Raw<T> o;
      o.set(v);
      o.store(dst + static_cast<long long>(u * R) * p.d, l);
    }
  }
  if (!partial || !turns) return;
  // lanes of one j, then warps, in a fixed order
  __shared__ float sums[kWarps][G][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float a = e & 1 ? hi(dw.x[e / 2]) : lo(dw.x[e / 2]);
#pragma unroll
    for (int o = G; o < 32; o <<= 1) a += __shfl_xor_sync(kFull, a, o);
    if (sub == 0) sums[warp][j][e] = a;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < G * 8; i += kWarps * 32) {
    const int jj = i / 8, e = i % 8;
    const Lane o = lane_of(p, jj);
    if (!o.on) continue;
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) a += sums[k][jj][e];
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

// Groups are a grid's y: 65,535 at most.  Heads that make more, one row a lane, take more rows a lane.
constexpr int kMostGroups = 65535;

int rows_that_fit(const QkArgs& p, int R, int u, int most) {
  while (u < most && groups_of(p.Hq, R * u) + 2 * groups_of(p.Hkv, R * u) > kMostGroups) ++u;
  return u;
}

// Rows a lane holds at once, u: a token's groups cost their rows, present or padded, and `group` rows' worth of angles,
// weights and addresses each.  Forward a group costs 2.5 rows (16 query and 2 key heads of 64: two rows a lane take
// 59 us where one, without padding, takes 80); backward, where the next token's copies hide it, next to nothing (16 and
// 16 heads of 128: two rows 243 us, three 255).
int rows_per_lane(const QkArgs& p, int R, int most, double group) {
  int best = 1;
  double least = 1e30;
  for (int u = 1; u <= most; ++u) {
    const double cost = (groups_of(p.Hq, R * u) + 2 * groups_of(p.Hkv, R * u)) * (u + group);
    if (cost < least) least = cost, best = u;
  }
  return best;
}

// Whether a lane's four pairs can lie on more than two axes.
bool narrow_axes(const QkArgs& p) {
  if (!p.positions) return false;
  for (int x = 1; x + 1 < p.axes; ++x)
    if (p.bound[x] - p.bound[x - 1] < 3) return true;
  return false;
}

// f(rows a lane holds, NARROW).  Narrow axes cost four positions and eight table loads a lane: one row at a time.
template <int MOST, typename F>
int by_rows(const QkArgs& p, int u, F f) {
  if (narrow_axes(p)) return f(std::integral_constant<int, 1>(), std::true_type());
  if constexpr (MOST >= 4) {
    if (u == 4) return f(std::integral_constant<int, 4>(), std::false_type());
  }
  if constexpr (MOST >= 3) {
    if (u == 3) return f(std::integral_constant<int, 3>(), std::false_type());
  }
  if constexpr (MOST >= 2) {
    if (u == 2) return f(std::integral_constant<int, 2>(), std::false_type());
  }
  return f(std::integral_constant<int, 1>(), std::false_type());
}

// Blocks that walk over the tokens, for each group.
int walkers(int B, int L, int groups, int places) {
  const long long want = (static_cast<long long>(B) * L + kWarps - 1) / kWarps, most = places / groups;
  return static_cast<int>(want < most ? want : (most > 1 ? most : 1));
}

template <typename T, int G>
int launch_fwd(const QkArgs& p, void* qo, void* ko, void* vo, int cap, const int32_t* start, int num_sms, const DevCtl& ctl,
               cudaStream_t st) {
  constexpr int R = 32 / G;
  // few tokens: one row a lane, for more warps
  const bool few = static_cast<long long>(p.B) * p.L <= static_cast<long long>(num_sms) * kWarps;
  constexpr int kRows = sizeof(T) == 2 ? kRowsPerLane : 2;
  return by_rows<kRows>(p, rows_that_fit(p, R, few ? 1 : rows_per_lane(p, R, kRows, 2.5), kRows), [&](auto n, auto narrow) {
    constexpr int U = decltype(n)::value;
    const int groups = groups_of(p.Hq, R * U) + (p.v ? 2 : 1) * groups_of(p.Hkv, R * U);
    if (groups > kMostGroups) return 0;
    const dim3 grid(walkers(p.B, p.L, groups, num_sms * kFwdBlocksPerSm * kWaves), groups);
    qk_fwd_kernel<T, G, U, decltype(narrow)::value><<<grid, kWarps * 32, 0, st>>>(p, static_cast<T*>(qo), static_cast<T*>(ko), static_cast<T*>(vo),
                                                                                 cap, start, ctl);
    return cudaGetLastError() == cudaSuccess ? 1 : -1;
  });
}

template <typename T, typename GT, int G>
int launch_bwd(const QkArgs& p, const void* dq, const void* dk, const void* dv, void* dqkv, float* dqw, float* dkw,
               float* workspace, int num_sms, const DevCtl& ctl, cudaStream_t st) {
  constexpr int R = 32 / G;
  const bool weights = p.normalize && (dqw || dkw);
  // what two blocks' shared memory holds of two tokens' rows and gradients (88 KB a block at most)
  constexpr int kRows = sizeof(T) + sizeof(GT) == 4 ? 4 : (sizeof(T) + sizeof(GT) == 6 ? 3 : 2);
  return by_rows<kRows>(p, rows_that_fit(p, R, rows_per_lane(p, R, kRows, 0.01), kRows), [&](auto n, auto narrow) {
    constexpr int U = decltype(n)::value;
    const int nq = groups_of(p.Hq, R * U), nk = groups_of(p.Hkv, R * U), groups = nq + (dv ? 2 : 1) * nk;
    if (groups > kMostGroups) return 0;
    const int blocks = walkers(p.B, p.L, groups, num_sms * kBwdBlocksPerSm * kWaves);
    auto kern = qk_bwd_kernel<T, GT, G, U, decltype(narrow)::value>;
    constexpr int bytes = 2 * sizeof(BwdStage<T, GT, U>);
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return -1;
    kern<<<dim3(blocks, groups), kWarps * 32, bytes, st>>>(p, static_cast<const GT*>(dq), static_cast<const GT*>(dk), static_cast<const GT*>(dv),
                                                           static_cast<T*>(dqkv), weights ? workspace : nullptr, ctl);
    if (cudaGetLastError() != cudaSuccess) return -1;
    if (!weights) return 1;
    qk_bwd_weights_kernel<<<dim3((p.d + 31) / 32, 2), dim3(32, 32), 0, st>>>(workspace, nq * blocks, nk * blocks, p.d, dqw, dkw);
    return cudaGetLastError() == cudaSuccess ? 2 : -1;
  });
}

template <typename F>
int by_lanes(int d, F f) {
  const int lanes = (d + 7) / 8;
  if (lanes <= 4) return f(std::integral_constant<int, 4>());
  if (lanes <= 8) return f(std::integral_constant<int, 8>());
  if (lanes <= 16) return f(std::integral_constant<int, 16>());
  return f(std::integral_constant<int, 32>());
}

}  // namespace

// Partial rows of weight gradients: at most one for each block of a full grid and one more for each
// group, or one for each eight tokens and head.
int qk_bwd_partial_rows(int B, int L, int Hq, int Hkv, int num_sms) {
  const long long heads = static_cast<long long>(Hq) + Hkv, full = static_cast<long long>(num_sms) * kBwdBlocksPerSm * kWaves + heads;
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
