// grouped.cu -- plain attention (Eq. 1) of grouped heads: over packed prompts, and of drafted tokens over caches.
#include <cuda_bf16.h>

#include "kernels.h"

namespace topk {

namespace {

// A warp for each query row: the softmax's running maximum and sum over its keys.
template <typename Valid>
__device__ void attend(const __nv_bfloat16* q, const __nv_bfloat16* k, long long k_stride, const __nv_bfloat16* v, long long v_stride, int keys, int d,
                       __nv_bfloat16* out, Valid valid) {
  const int lane = threadIdx.x & 31, each = d / 32;
  float x[4], acc[4] = {}, m = -INFINITY, z = 0.f;
  for (int e = 0; e < each; ++e) x[e] = __bfloat162float(q[lane * each + e]);
  for (int j = 0; j < keys; ++j) {
    if (!valid(j)) continue;
    float s = 0.f;
    for (int e = 0; e < each; ++e) s += x[e] * __bfloat162float(k[j * k_stride + lane * each + e]);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const float to = fmaxf(m, s), f = m == -INFINITY ? 0.f : expf(m - to), p = s == -INFINITY ? 0.f : expf(s - to);
    m = to;
    z = z * f + p;
    for (int e = 0; e < each; ++e) acc[e] = acc[e] * f + p * __bfloat162float(v[j * v_stride + lane * each + e]);
  }
  for (int e = 0; e < each; ++e) out[lane * each + e] = __float2bfloat16_rn(z > 0.f ? acc[e] / z : z == 0.f ? 0.f : NAN);
}

// Sequence b's rows [first, end), cut to the tensor.
__device__ bool bounds_of(const int32_t* starts, int b, int T, int& first, int& end) {
  const int s = __ldg(starts + b), e = __ldg(starts + b + 1);
  first = min(max(s, 0), T), end = max(first, min(max(e, 0), T));
  return s == first && e == end;
}

__global__ void prompt_kernel(topk_prompt_args a, DevCtl ctl) {
  const int row = blockIdx.x, head = blockIdx.y * blockDim.y + threadIdx.y;
  if (head >= a.Hq) return;
  __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (static_cast<size_t>(row) * a.Hq + head) * a.d;
  for (int b = 0; b < a.B; ++b) {
    int q0, q1, k0, k1;
    bool ok = bounds_of(a.q_starts, b, a.Tq, q0, q1);
    ok &= bounds_of(a.k_starts ? a.k_starts : a.q_starts, b, a.Tk, k0, k1);
    if (!ok) atomicOr(ctl.error, kDevErrRange);
    if (row < q0 || row >= q1) continue;
    const int g = head / (a.Hq / a.Hkv), keys = k1 - k0, lim = a.causal ? row - q0 + keys - (q1 - q0) + 1 : keys;
    attend(static_cast<const __nv_bfloat16*>(a.q) + row * a.q_stride[0] + head * a.q_stride[1],
           static_cast<const __nv_bfloat16*>(a.k) + k0 * a.k_stride[0] + g * a.k_stride[1], a.k_stride[0],
           static_cast<const __nv_bfloat16*>(a.v) + k0 * a.v_stride[0] + g * a.v_stride[1], a.v_stride[0], min(lim, keys), a.d, out,
           [](int) { return true; });
    return;
  }
  if (a.clear_rest)
    for (int e = threadIdx.x; e < a.d; e += 32) out[e] = __float2bfloat16_rn(0.f);
}

__global__ void tree_kernel(topk_tree_args a, DevCtl ctl) {
  const int i = blockIdx.x % a.T, b = blockIdx.x / a.T, head = blockIdx.y * blockDim.y + threadIdx.y;
  if (head >= a.Hq) return;
  const int n = __ldg(a.kv_len + b), g = head / (a.Hq / a.Hkv);
  if (static_cast<long long>(n) + a.T > a.cap) atomicOr(ctl.error, kDevErrRange);
  const int prefix = min(max(n, 0), a.cap), keys = n < 0 ? 0 : min(prefix + a.T, a.cap);
  const unsigned long long word = a.tree ? static_cast<unsigned long long>(a.tree[b * a.tree_stride + i]) : ~0ull >> (63 - i);
  attend(static_cast<const __nv_bfloat16*>(a.q) + b * a.q_stride[0] + head * a.q_stride[1] + i * a.q_stride[2],
         static_cast<const __nv_bfloat16*>(a.keys) + b * a.key_stride[0] + g * a.key_stride[1], a.key_stride[2],
         static_cast<const __nv_bfloat16*>(a.values) + b * a.value_stride[0] + g * a.value_stride[1], a.value_stride[2], keys, a.d,
         static_cast<__nv_bfloat16*>(a.out) + ((static_cast<size_t>(b) * a.Hq + head) * a.T + i) * a.d,
         [=](int j) { return j < prefix || (word >> (j - prefix) & 1ull); });
}

}  // namespace

size_t grouped_workspace_bytes(int, int) { return 0; }

int prompt_attn(const topk_prompt_args& a, void*, int, const DevCtl& ctl, cudaStream_t st) {
  prompt_kernel<<<dim3(a.Tq, (a.Hq + 7) / 8), dim3(32, 8), 0, st>>>(a, ctl);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

int tree_attn(const topk_tree_args& a, void*, int, const DevCtl& ctl, cudaStream_t st) {
  tree_kernel<<<dim3(a.B * a.T, (a.Hq + 7) / 8), dim3(32, 8), 0, st>>>(a, ctl);
  return cudaGetLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace topk
