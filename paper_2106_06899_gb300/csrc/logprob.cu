// logprob.cu -- log probabilities of tokens from their logits: the target's, the entropy, the largest
// alternatives, and the gradient.
#include <cuda_bf16.h>

#include "kernels.h"

namespace topk {

namespace {

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

__device__ __forceinline__ long long target_at(const LogprobArgs& a, int n) {
  if (!a.targets) return -1;
  return a.targets64 ? __ldg(static_cast<const long long*>(a.targets) + n) : __ldg(static_cast<const int*>(a.targets) + n);
}

constexpr int kThreads = 256;

template <typename Op>
__device__ float block_reduce(float v, Op op, float* shared) {
  for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  v = shared[0];
  for (int w = 1; w < kThreads / 32; ++w) v = op(v, shared[w]);
  return v;
}

// A block for each row: its maximum, its sums, then its alternatives one after the other.
template <typename T>
__global__ void __launch_bounds__(kThreads)
    logprob_fwd_kernel(LogprobArgs a, float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, DevCtl ctl) {
  __shared__ float shared[kThreads / 32];
  __shared__ unsigned long long best[kThreads / 32];
  const int n = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(n) * a.stride;
  float m = -INFINITY;
  bool bad = false;
  for (int j = threadIdx.x; j < a.V; j += kThreads) {
    const float v = to_f(x[j]);
    bad |= !(v < INFINITY);
    m = fmaxf(m, v);
  }
  bad = __syncthreads_or(bad);
  m = block_reduce(m, [](float p, float q) { return fmaxf(p, q); }, shared);
  const bool none = m == -INFINITY;
  float s = 0.f, t = 0.f;
  if (!bad && !none)
    for (int j = threadIdx.x; j < a.V; j += kThreads) {
      const float d = (to_f(x[j]) - m) * a.scale, e = expf(d);
      s += e;
      t += e == 0.f ? 0.f : e * d;
    }
  const auto add = [](float p, float q) { return p + q; };
  s = block_reduce(s, add, shared), t = block_reduce(t, add, shared);
  const float ln = logf(s);
  if (threadIdx.x == 0) {
    if (lse) lse[n] = bad ? NAN : none ? -INFINITY : m * a.scale + ln;
    if (entropy) entropy[n] = bad ? NAN : none ? 0.f : ln - t / s;
    const long long target = target_at(a, n);
    if (target >= a.V) atomicOr(ctl.error, kDevErrRange);
    if (logp) {
      const bool real = target >= 0 && target < a.V;
      logp[n] = !real ? 0.f : bad ? NAN : none ? -INFINITY : (to_f(x[target]) - m) * a.scale - ln;
    }
  }
  // the largest (value, lowest index) below the last one taken
  unsigned long long last = ~0ull;
  for (int i = 0; i < a.top; ++i) {
    unsigned long long mine = 0;
    if (!bad)
      for (int j = threadIdx.x; j < a.V; j += kThreads) {
        const float v = to_f(x[j]) + 0.f;  // -0 as 0
        if (v == -INFINITY) continue;
        const unsigned b = __float_as_uint(v), o = b & 0x80000000u ? ~b : b | 0x80000000u;
        const unsigned long long key = static_cast<unsigned long long>(o) << 32 | ~static_cast<unsigned>(j);
        if (key < last && key > mine) mine = key;
      }
    for (int o = 16; o; o >>= 1) mine = max(mine, __shfl_xor_sync(0xffffffffu, mine, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) best[threadIdx.x >> 5] = mine;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) mine = max(mine, best[w]);
    if (threadIdx.x == 0) {
      const int at = mine ? static_cast<int>(~static_cast<unsigned>(mine)) : -1;
      top_ids[static_cast<size_t>(n) * a.top + i] = at;
      top_logp[static_cast<size_t>(n) * a.top + i] = bad ? NAN : at < 0 ? -INFINITY : (to_f(x[at]) - m) * a.scale - ln;
    }
    last = mine;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
    logprob_bwd_kernel(LogprobArgs a, const float* lse, const float* dlogp, const float* entropy, const float* dentropy, const int32_t* top_ids,
                       const float* dtop, T* out, long long out_stride) {
  const int n = blockIdx.x;
  const T* x = static_cast<const T*>(a.logits) + static_cast<size_t>(n) * a.stride;
  T* y = out + static_cast<size_t>(n) * out_stride;
  const long long target = target_at(a, n);
  const float g = dlogp && target >= 0 && target < a.V ? dlogp[n] : 0.f;
  float total = g;
  bool any = g != 0.f;
  for (int m = 0; m < a.top; ++m) {
    const int at = top_ids[static_cast<size_t>(n) * a.top + m];
    if (at < 0 || at >= a.V) continue;
    total += dtop[static_cast<size_t>(n) * a.top + m];
    any |= dtop[static_cast<size_t>(n) * a.top + m] != 0.f;
  }
  const float h = dentropy ? dentropy[n] : 0.f, H = dentropy ? entropy[n] : 0.f, l = lse[n];
  any |= h != 0.f;
  for (int j = threadIdx.x; j < a.V; j += kThreads) {
    float d = 0.f;
    if (any && l != -INFINITY) {
      const float lp = to_f(x[j]) * a.scale - l, p = expf(lp);
      d = -p * total;
      if (h != 0.f && p != 0.f) d -= h * p * (lp + H);
      if (j == target) d += g;
      for (int m = 0; m < a.top; ++m)
        if (top_ids[static_cast<size_t>(n) * a.top + m] == j) d += dtop[static_cast<size_t>(n) * a.top + m];
    }
    put(y + j, d * a.scale);
  }
}

}  // namespace

int logprob_fwd(const LogprobArgs& a, float* logp, float* entropy, float* lse, float* top_logp, int32_t* top_ids, bool bf16, int,
                const DevCtl& ctl, cudaStream_t st) {
  if (bf16)
    logprob_fwd_kernel<__nv_bfloat16><<<a.N, kThreads, 0, st>>>(a, logp, entropy, lse, top_logp, top_ids, ctl);
  else
    logprob_fwd_kernel<float><<<a.N, kThreads, 0, st>>>(a, logp, entropy, lse, top_logp, top_ids, ctl);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int logprob_bwd(const LogprobArgs& a, const float* lse, const float* dlogp, const float* entropy, const float* dentropy, const int32_t* top_ids,
                const float* dtop, void* dlogits, long long out_stride, bool bf16, int, cudaStream_t st) {
  if (bf16)
    logprob_bwd_kernel<<<a.N, kThreads, 0, st>>>(a, lse, dlogp, entropy, dentropy, top_ids, dtop, static_cast<__nv_bfloat16*>(dlogits), out_stride);
  else
    logprob_bwd_kernel<<<a.N, kThreads, 0, st>>>(a, lse, dlogp, entropy, dentropy, top_ids, dtop, static_cast<float*>(dlogits), out_stride);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace topk
