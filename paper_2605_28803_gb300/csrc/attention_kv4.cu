// Attention of a few query tokens over the 4-bit key/value cache.  A block takes one query head of one token; its warps take
// every kWarps-th cached token and are joined at the end.
#include <cuda_runtime.h>

#include "kv4.cuh"

namespace qvla {
namespace {

constexpr int kWarps = 4;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T, int kDim>
__global__ void __launch_bounds__(32 * kWarps) attention_kv4_kernel(const Kv4AttentionArgs a) {
  constexpr int kTeam = kDim / 8, kTeams = 32 / kTeam;
  __shared__ float s_acc[kWarps * kTeams][kDim], s_m[kWarps * kTeams], s_l[kWarps * kTeams];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, team = lane / kTeam, tl = lane % kTeam;
  const int t = blockIdx.x, h = blockIdx.y, kvh = h / (a.heads / a.pool.kv_heads);
  int b, q0;
  if (!find_sequence(a.cu_q, a.batch, t, b, q0)) return;
  const int n = min(a.cu_q[b + 1], a.total_q) - q0, keys = a.kv_len[b];
  if (n > a.max_q || keys < 0 || keys > a.max_len) {
    report_index();
    return;
  }
  const int seen = a.causal ? min(keys, keys - n + (t - q0) + 1) : keys;
  float q[8], acc[8] = {};
  unpack8<T>(*reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + t * a.q_stride + h * kDim + tl * 8), q);
  if (a.pool.rotate) rotate_head<kTeam>(q);
  const int plane = (kDim / 2) << a.pool.log_page;
  const int part = warp * kTeams + team;
  float m = -INFINITY, l = 0.0f;
  for (int j0 = 0; j0 < seen; j0 += kWarps * kTeams) {
    const int j = j0 + part;
    uint8_t* page = j < seen ? kv4_block(a.pool, a.table, a.max_pages, b, j, kvh) : nullptr;
    const int slot = j & ((1 << a.pool.log_page) - 1);
    uint32_t kc = 0, vc = 0;
    float ks = 0.0f, vs = 0.0f;
    if (page) {
      kc = *reinterpret_cast<const uint32_t*>(page + slot * (kDim / 2) + tl * 4);
      vc = *reinterpret_cast<const uint32_t*>(page + plane + slot * (kDim / 2) + tl * 4);
      ks = reinterpret_cast<const float*>(page + 2 * plane)[slot];
      vs = reinterpret_cast<const float*>(page + 2 * plane)[(1 << a.pool.log_page) + slot];
    }
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c) s = fmaf(q[c], static_cast<float>(static_cast<int>(kc << (28 - 4 * c)) >> 28), s);
#pragma unroll
    for (int x = 1; x < kTeam; x *= 2) s += __shfl_xor_sync(0xffffffffu, s, x);
    if (!page) continue;
    s *= ks * a.scale * kLog2e;
    const float top = fmaxf(m, s), keep = m == top ? 1.0f : exp2f(m - top), p = exp2f(s - top);
    m = top;
    l = l * keep + p;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      acc[c] = fmaf(p * vs, static_cast<float>(static_cast<int>(vc << (28 - 4 * c)) >> 28), acc[c] * keep);
  }
  if (tl == 0) {
    s_m[part] = m;
    s_l[part] = l;
  }
#pragma unroll
  for (int c = 0; c < 8; ++c) s_acc[part][tl * 8 + c] = acc[c];
  __syncthreads();
  if (warp > 0) return;
  float top = -INFINITY, sum = 0.0f, o[8] = {};
  for (int w = 0; w < kWarps * kTeams; ++w) top = fmaxf(top, s_m[w]);
  for (int w = 0; w < kWarps * kTeams; ++w) {
    if (s_l[w] == 0.0f) continue;
    const float f = exp2f(s_m[w] - top);
    sum += s_l[w] * f;
    for (int c = 0; c < 8; ++c) o[c] += s_acc[w][tl * 8 + c] * f;
  }
  for (int c = 0; c < 8; ++c) o[c] = sum == 0.0f ? 0.0f : o[c] / sum;
  if (a.pool.rotate) rotate_head<kTeam>(o);
  if (team == 0)
    *reinterpret_cast<uint4*>(static_cast<T*>(a.o) + (static_cast<size_t>(t) * a.heads + h) * kDim + tl * 8) = pack8<T>(o);
}

template <typename T>
void launch(const Kv4AttentionArgs& a) {
  const dim3 grid(a.total_q, a.heads);
  if (a.pool.head_dim == 64) attention_kv4_kernel<T, 64><<<grid, 32 * kWarps, 0, a.stream>>>(a);
  if (a.pool.head_dim == 128) attention_kv4_kernel<T, 128><<<grid, 32 * kWarps, 0, a.stream>>>(a);
  if (a.pool.head_dim == 256) attention_kv4_kernel<T, 256><<<grid, 32 * kWarps, 0, a.stream>>>(a);
}

}  // namespace

size_t attention_kv4_workspace(const Kv4AttentionArgs&) { return 0; }

cudaError_t launch_attention_kv4(const Kv4AttentionArgs& a) {
  if (a.dt == 0) launch<__half>(a);
  else launch<__nv_bfloat16>(a);
  return cudaGetLastError();
}

cudaError_t read_and_clear_error_word_attention_kv4(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

}  // namespace qvla
