// The 4-bit key/value cache: tokens in (rotate, quantise, store to their pages) and tokens out.
//
// Per token and key/value head: y = x . H / sqrt(D) (or x), Delta = max |y| / 7, codes clamp(round(y / Delta), -7, 7), round half
// to even on the exact quotient; out again, x^ = (Delta q) . H / sqrt(D), rounded to the output's type.
//
// Both are bound by HBM (read 2 D bytes, write D / 2 + 4, and the other way round); the rest hides behind it.  A head is
// a team of D / 8 lanes with 8 channels (16 bytes in, 4 bytes of codes) each, so that loads and stores of a team are contiguous
// and the rotation stays in registers and shuffles.  A warp takes kRows heads of one token per team, all loaded before
// the first is used: the sequence search and the page lookup are made once for them.
#include <cuda_runtime.h>

#include "kv4.cuh"

namespace qvla {
namespace {

constexpr int kThreads = 128;
constexpr int kRows = 4;  // heads a team holds at once

// The code of y at scale d, r = 1 / d: round half to even on the exact quotient y / d.  y r is within 2 ulp of it, so away
// from a half-integer both round alike; near one the rounded quotient t and the sign of the remainder y - t d decide.
__device__ __forceinline__ int code_of(float y, float d, float r) {
  const float t = y * r;
  float n = rintf(t);
  if (fabsf(fabsf(t - n) - 0.5f) < 1e-5f) {
    const float t2 = __fdiv_rn(y, d);
    n = rintf(t2);
    if (fabsf(t2 - n) == 0.5f) {  // the quotient rounds to a half-integer: is it one?
      const float rest = fmaf(-t2, d, y);
      if (rest > 0.0f) n = ceilf(t2);
      if (rest < 0.0f) n = floorf(t2);
    }
  }
  return static_cast<int>(fminf(fmaxf(n, -7.0f), 7.0f));
}

template <typename T, int kTeam, bool kAppend>
__global__ void __launch_bounds__(kThreads) kv4_rows_kernel(const Kv4RowsArgs a) {
  constexpr int kDim = 8 * kTeam, kTeams = 32 / kTeam;
  const int lane = threadIdx.x & 31, team = lane / kTeam, tl = lane % kTeam;
  const int rows = 2 * a.pool.kv_heads;  // a token's heads: keys, then values
  const int chunks = (rows + kTeams * kRows - 1) / (kTeams * kRows);
  const int64_t item = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;  // the same in a whole warp
  if (item >= static_cast<int64_t>(a.total) * chunks) return;
  const int t = static_cast<int>(item / chunks), row0 = static_cast<int>(item % chunks) * kTeams * kRows;
  int b, first;
  if (!find_sequence(a.cu, a.batch, t, b, first)) return;
  const int64_t pos = static_cast<int64_t>(a.start ? __ldg(a.start + b) : 0) + (t - first);
  uint8_t* const page = kv4_block(a.pool, a.table, a.max_pages, b, pos, 0);
  const int slot = static_cast<int>(pos) & ((1 << a.pool.log_page) - 1);
  if (kAppend && page == nullptr) return;
  const size_t block = kv4_block_bytes(a.pool);
  const int plane = (kDim / 2) << a.pool.log_page;  // bytes of a block's key codes

  uint4 x[kRows];
  float scale[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int row = row0 + i * kTeams + team;
    x[i] = make_uint4(0, 0, 0, 0);
    scale[i] = 0.0f;
    if (row >= rows) continue;
    const int value = row >= a.pool.kv_heads, head = row - value * a.pool.kv_heads;
    if constexpr (kAppend) {
      const T* src = static_cast<const T*>(value ? a.v : a.k) + t * (value ? a.v_stride : a.k_stride) + head * kDim + tl * 8;
      x[i] = __ldg(reinterpret_cast<const uint4*>(src));
    } else if (page != nullptr) {
      const uint8_t* src = page + head * block;
      x[i].x = __ldg(reinterpret_cast<const unsigned int*>(src + value * plane + slot * (kDim / 2) + tl * 4));
      scale[i] = __ldg(reinterpret_cast<const float*>(src + 2 * plane) + (value << a.pool.log_page) + slot);
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (row0 + i * kTeams >= rows) break;
    const int row = row0 + i * kTeams + team;
    const bool live = row < rows;  // (every lane takes the shuffles)
    const int value = row >= a.pool.kv_heads, head = row - value * a.pool.kv_heads;
    float y[8];
    if constexpr (kAppend) {
      unpack8<T>(x[i], y);
      if (a.pool.rotate) rotate_head<kTeam>(y);
      float m = 0.0f;
      bool nan = false;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        m = fmaxf(m, fabsf(y[c]));
        nan |= y[c] != y[c];
      }
      if (nan) m = __int_as_float(0x7fffffff);
#pragma unroll
      for (int h = 1; h < kTeam; h *= 2) {  // the maximum of the bits: a NaN stands above every number
        m = __uint_as_float(max(__float_as_uint(m), __shfl_xor_sync(0xffffffffu, __float_as_uint(m), h)));
      }
      const float d = __fdiv_rn(m, 7.0f);
      uint32_t w = 0;
      if (d > 0.0f && d < __int_as_float(0x7f800000)) {  // not zero, infinite or NaN
        const bool tiny = d < 1e-28f;  // the remainder of a quotient could leave the numbers: decide on scaled values
        const float ds = tiny ? d * 0x1p64f : d, r = __frcp_rn(ds);
#pragma unroll
        for (int c = 0; c < 8; ++c)
          w |= (static_cast<uint32_t>(code_of(tiny ? y[c] * 0x1p64f : y[c], ds, r)) & 15u) << (4 * c);
      }
      if (live) {
        uint8_t* dst = page + head * block;
        *reinterpret_cast<uint32_t*>(dst + value * plane + slot * (kDim / 2) + tl * 4) = w;
        // an infinity reads back as NaN, like a NaN
        if (tl == 0)
          reinterpret_cast<float*>(dst + 2 * plane)[(value << a.pool.log_page) + slot] =
              d < __int_as_float(0x7f800000) ? d : __int_as_float(0x7fffffff);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c)  // (a product of its own: fused into the rotation's first sums it would not be rounded)
        y[c] = __fmul_rn(static_cast<float>(static_cast<int>(x[i].x << (28 - 4 * c)) >> 28), scale[i]);
      if (a.pool.rotate) rotate_head<kTeam>(y);
      if (live) {
        T* dst = static_cast<T*>(value ? a.v : a.k) + t * (value ? a.v_stride : a.k_stride) + head * kDim + tl * 8;
        *reinterpret_cast<uint4*>(dst) = pack8<T>(y);
      }
    }
  }
}

template <typename T, int kTeam, bool kAppend>
cudaError_t launch_rows(const Kv4RowsArgs& a) {
  const int rows = 2 * a.pool.kv_heads, per = 32 / kTeam * kRows;
  const int64_t items = static_cast<int64_t>(a.total) * ((rows + per - 1) / per);
  const int64_t blocks = (items * 32 + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
  kv4_rows_kernel<T, kTeam, kAppend><<<static_cast<unsigned int>(blocks), kThreads, 0, a.stream>>>(a);
  return cudaGetLastError();
}

template <bool kAppend>
cudaError_t launch_rows(const Kv4RowsArgs& a) {
  const int d = a.pool.head_dim;
  if (a.dt == 0) {
    return d == 64 ? launch_rows<__half, 8, kAppend>(a) : d == 128 ? launch_rows<__half, 16, kAppend>(a) : launch_rows<__half, 32, kAppend>(a);
  }
  return d == 64 ? launch_rows<__nv_bfloat16, 8, kAppend>(a)
                 : d == 128 ? launch_rows<__nv_bfloat16, 16, kAppend>(a) : launch_rows<__nv_bfloat16, 32, kAppend>(a);
}

}  // namespace

cudaError_t launch_kv4_append(const Kv4RowsArgs& a) { return launch_rows<true>(a); }
cudaError_t launch_kv4_gather(const Kv4RowsArgs& a) { return launch_rows<false>(a); }

cudaError_t read_and_clear_error_word_kv4(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess) return e;
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

}  // namespace qvla
