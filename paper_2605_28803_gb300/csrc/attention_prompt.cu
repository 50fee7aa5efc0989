// Softmax attention over packed prompts: o_i = sum_j p_ij v_j, p_ij = exp(scale q_i.k_j) / sum exp, in one pass over the keys
// with a running maximum and sum.  A block takes one query head of one token; its warps take every kWarps-th key and
// are joined at the end.
#include <cuda_runtime.h>

#include "kv4.cuh"

namespace qvla {
namespace {

constexpr int kWarps = 4;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T, int kDim>
__global__ void __launch_bounds__(32 * kWarps) attention_prompt_kernel(const PromptArgs a) {
  constexpr int kPer = kDim / 32;
  __shared__ float s_acc[kWarps][kDim], s_m[kWarps], s_l[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int t = blockIdx.x, h = blockIdx.y, kvh = h / (a.heads / a.kv_heads);
  int b, q0;
  if (!find_sequence(a.cu_q, a.batch, t, b, q0)) return;
  const int n = min(a.cu_q[b + 1], a.total_q) - q0;
  const int k0 = min(max(a.cu_k[b], 0), a.total_k), k1 = min(max(a.cu_k[b + 1], k0), a.total_k);
  const int keys = k1 - k0, seen = a.causal ? min(keys, keys - n + (t - q0) + 1) : keys;
  float q[kPer], acc[kPer];
  const T* qp = static_cast<const T*>(a.q) + t * a.q_stride + h * kDim + lane * kPer;
#pragma unroll
  for (int c = 0; c < kPer; ++c) {
    q[c] = static_cast<float>(qp[c]) * (a.scale * kLog2e);
    acc[c] = 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  for (int j = warp; j < seen; j += kWarps) {
    const T* kp = static_cast<const T*>(a.k) + (k0 + j) * a.k_stride + kvh * kDim + lane * kPer;
    const T* vp = static_cast<const T*>(a.v) + (k0 + j) * a.v_stride + kvh * kDim + lane * kPer;
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < kPer; ++c) s = fmaf(q[c], static_cast<float>(kp[c]), s);
#pragma unroll
    for (int x = 16; x > 0; x /= 2) s += __shfl_xor_sync(0xffffffffu, s, x);
    const float top = fmaxf(m, s), keep = m == top ? 1.0f : exp2f(m - top), p = exp2f(s - top);
    m = top;
    l = l * keep + p;
#pragma unroll
    for (int c = 0; c < kPer; ++c) acc[c] = fmaf(p, static_cast<float>(vp[c]), acc[c] * keep);
  }
  if (lane == 0) {
    s_m[warp] = m;
    s_l[warp] = l;
  }
#pragma unroll
  for (int c = 0; c < kPer; ++c) s_acc[warp][lane * kPer + c] = acc[c];
  __syncthreads();
  float top = -INFINITY, sum = 0.0f;
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, s_m[w]);
  for (int w = 0; w < kWarps; ++w) sum += s_l[w] == 0.0f ? 0.0f : s_l[w] * exp2f(s_m[w] - top);
  for (int c = threadIdx.x; c < kDim; c += 32 * kWarps) {
    float o = 0.0f;
    for (int w = 0; w < kWarps; ++w) o += s_l[w] == 0.0f ? 0.0f : s_acc[w][c] * exp2f(s_m[w] - top);
    static_cast<T*>(a.o)[(static_cast<size_t>(t) * a.heads + h) * kDim + c] = static_cast<T>(sum == 0.0f ? 0.0f : o / sum);
  }
}

template <typename T>
void launch(const PromptArgs& a) {
  const dim3 grid(a.total_q, a.heads);
  if (a.head_dim == 64) attention_prompt_kernel<T, 64><<<grid, 32 * kWarps, 0, a.stream>>>(a);
  if (a.head_dim == 128) attention_prompt_kernel<T, 128><<<grid, 32 * kWarps, 0, a.stream>>>(a);
  if (a.head_dim == 256) attention_prompt_kernel<T, 256><<<grid, 32 * kWarps, 0, a.stream>>>(a);
}

}  // namespace

cudaError_t launch_attention_prompt(const PromptArgs& a) {
  if (a.dt == 0) launch<__half>(a);
  else launch<__nv_bfloat16>(a);
  return cudaGetLastError();
}

cudaError_t read_and_clear_error_word_prompt(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

}  // namespace qvla
