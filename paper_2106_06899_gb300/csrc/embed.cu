// embed.cu -- the embedding lookup and its gradient.
#include <cuda_bf16.h>

#include "kernels.h"

namespace topk {

namespace {

__device__ __forceinline__ long long id_at(const void* ids, bool wide, int n) {
  return wide ? __ldg(static_cast<const long long*>(ids) + n) : __ldg(static_cast<const int*>(ids) + n);
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// A block for each token.
template <typename T>
__global__ void embed_fwd_kernel(EmbedArgs a, const T* __restrict__ weight, T* __restrict__ out, DevCtl ctl) {
  const long long id = id_at(a.ids, a.ids64, blockIdx.x);
  if (id >= a.rows && threadIdx.x == 0) atomicOr(ctl.error, kDevErrRange);
  const bool real = id >= 0 && id < a.rows;
  const T* w = weight + (real ? static_cast<size_t>(id) * a.D : 0);
  for (int c = threadIdx.x; c < a.D; c += blockDim.x)
    put(out + static_cast<size_t>(blockIdx.x) * a.D + c, real ? to_f(w[c]) * a.scale : 0.f);
}

// A block for each row of the gradient: it reads all ids and adds up its tokens in order.
template <typename T, typename G>
__global__ void __launch_bounds__(256) embed_bwd_kernel(EmbedArgs a, const T* __restrict__ dy, G* __restrict__ dw, bool accumulate, DevCtl ctl) {
  __shared__ int found[256];
  __shared__ int count[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int c0 = 0; c0 < a.D; c0 += 256) {
    const int c = c0 + threadIdx.x;
    float sum = 0.f;
    bool any = false;
    for (int n0 = 0; n0 < a.N; n0 += 256) {
      const int n = n0 + threadIdx.x;
      const long long id = n < a.N ? id_at(a.ids, a.ids64, n) : -1;
      if (id >= a.rows && blockIdx.x == 0) atomicOr(ctl.error, kDevErrRange);
      const bool mine = id == static_cast<long long>(blockIdx.x);
      const unsigned votes = __ballot_sync(0xffffffffu, mine);
      if (lane == 0) count[warp] = __popc(votes);
      __syncthreads();
      int at = __popc(votes & ((1u << lane) - 1u)), total = 0;
      for (int w = 0; w < 8; ++w) {
        if (w < warp) at += count[w];
        total += count[w];
      }
      if (mine) found[at] = n;
      __syncthreads();
      any |= total > 0;
      if (c < a.D)
        for (int i = 0; i < total; ++i) sum += to_f(dy[static_cast<size_t>(found[i]) * a.D + c]);
      __syncthreads();
    }
    if (c < a.D) {
      G* p = dw + static_cast<size_t>(blockIdx.x) * a.D + c;
      if (!accumulate)
        put(p, sum * a.scale);
      else if (any)
        put(p, to_f(*p) + sum * a.scale);
    }
  }
}

}  // namespace

int embed_fwd(const EmbedArgs& a, const void* weight, void* out, bool bf16, int, const DevCtl& ctl, cudaStream_t st) {
  if (bf16)
    embed_fwd_kernel<<<a.N, 256, 0, st>>>(a, static_cast<const __nv_bfloat16*>(weight), static_cast<__nv_bfloat16*>(out), ctl);
  else
    embed_fwd_kernel<<<a.N, 256, 0, st>>>(a, static_cast<const float*>(weight), static_cast<float*>(out), ctl);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

size_t embed_bwd_workspace_bytes(int, int, int) { return 16; }

template <typename T>
static void bwd_of(const EmbedArgs& a, const void* dy, void* dw, bool accumulate, bool grad_bf16, const DevCtl& ctl, cudaStream_t st) {
  if (grad_bf16)
    embed_bwd_kernel<<<a.rows, 256, 0, st>>>(a, static_cast<const T*>(dy), static_cast<__nv_bfloat16*>(dw), accumulate, ctl);
  else
    embed_bwd_kernel<<<a.rows, 256, 0, st>>>(a, static_cast<const T*>(dy), static_cast<float*>(dw), accumulate, ctl);
}

int embed_bwd(const EmbedArgs& a, const void* dy, void* dweight, bool accumulate, bool bf16, bool grad_bf16, void*, int, const DevCtl& ctl,
              cudaStream_t st) {
  if (bf16)
    bwd_of<__nv_bfloat16>(a, dy, dweight, accumulate, grad_bf16, ctl, st);
  else
    bwd_of<float>(a, dy, dweight, accumulate, grad_bf16, ctl, st);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace topk
