// What runs between two quantised products, a row at a time: the residual's update and the norms around a block, the Hadamard
// rotation and the quantiser to 4-bit floating point, in one pass over memory.
//
//   branch   u = y, or norm(y) (post_w + offset);  r' = R(a r + g u), R the residual's type
//   norm     h = T(norm(r') (pre_w + offset) + pre_b), with conditioning T((...)(1 + scale) + shift)
//   rotation z = h BlockDiag(H_b / sqrt b): float32 butterflies, the longest distance first, one product with 1/sqrt(b)
//   codes    MX and NV as in fp4.cuh
//
// A row takes whole warps, 32 channels a thread, in registers from the loads to the stores.  The norm and the rotation's first
// stages do not care which channels a thread holds, so the loads already bring them as those stages want them:
//   kPieces   norm only: pieces of 8 channels, neighbouring threads neighbouring pieces
//   kPlain    b <= 32: 32 consecutive channels
//   kFour     b = 64, 128: of the 4 lines (32 channels each) of 128 channels, thread p of 4 holds quads 2p, 2p + 1 of each
//   kEight    b = 256 .. 2048: thread q of 8 holds quad q of 8 lines, which differ in the high bits of the block's index
//   kSixteen  b = 4096: half a quad of 16 lines
// and one or two exchanges through shared memory (128 bytes a thread) end with 32 consecutive channels a thread, which is what
// the quantiser wants: one MX block or two NV blocks, 16 bytes of codes.  Running the stages from the longest distance
// down is what makes that the end and not the beginning.
#pragma once

#include "fp4.cuh"
#include "griddep.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rotate_quant.cuh"

namespace qvla {
namespace fp4 {

enum Layout { kPieces, kPlain, kFour, kEight, kSixteen };

constexpr int kRowThreads = 512;  // most threads of a CTA (K = 16384: one row)
constexpr int kMaxWarps = kRowThreads / 32;
constexpr int kSlots = 5;  // reductions over a row: two norms of two sums each, and the maximum

// N consecutive channels as float2 pairs.
template <int N>
__device__ __forceinline__ void load_unit(const float* p, float2* v) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const float4 f = *reinterpret_cast<const float4*>(p + 4 * i);
      v[2 * i] = make_float2(f.x, f.y);
      v[2 * i + 1] = make_float2(f.z, f.w);
    }
  } else {
    v[0] = *reinterpret_cast<const float2*>(p);
  }
}
__device__ __forceinline__ float2 widen(uint32_t w, __half) {
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
__device__ __forceinline__ float2 widen(uint32_t w, __nv_bfloat16) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <int N, typename T>
__device__ __forceinline__ void load_unit(const T* p, float2* v) {
  uint32_t w[N / 2];
  if constexpr (N == 8) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
  } else if constexpr (N == 4) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x, w[1] = u.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
#pragma unroll
  for (int i = 0; i < N / 2; ++i) v[i] = widen(w[i], T());
}
__device__ __forceinline__ uint32_t narrow(float2 f, __half) {
  const __half2 h = __floats2half2_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t narrow(float2 f, __nv_bfloat16) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int N>
__device__ __forceinline__ void store_unit(float* p, float2* v) {
  if constexpr (N >= 4) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *reinterpret_cast<float4*>(p + 4 * i) = make_float4(v[2 * i].x, v[2 * i].y, v[2 * i + 1].x, v[2 * i + 1].y);
  } else {
    *reinterpret_cast<float2*>(p) = v[0];
  }
}
// Stores the values rounded to T, and leaves the rounded ones in v; p may be null (rounding only).
template <int N, typename T>
__device__ __forceinline__ void store_unit(T* p, float2* v) {
  uint32_t w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    w[i] = narrow(v[i], T());
    v[i] = widen(w[i], T());
  }
  if (p == nullptr) return;
  if constexpr (N == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  } else if constexpr (N == 4) {
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  } else {
    *reinterpret_cast<uint32_t*>(p) = w[0];
  }
}

// A row's place among the CTA's warps, and sums and maxima over it.  Every thread of the CTA makes the same calls.
struct RowGroup {
  float* slots;  // [kSlots][kMaxWarps]
  int warps, first;  // of the row
  __device__ __forceinline__ float sum(float v, int slot) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (warps == 1) return v;
    float* const s = slots + slot * kMaxWarps;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    v = s[first];
    for (int i = 1; i < warps; ++i) v += s[first + i];  // one order for every thread
    return v;
  }
  // The largest; NaN if one is (bit patterns of non-negative floats order like the numbers, NaN above infinity).
  __device__ __forceinline__ float max(float v, int slot) const {
    unsigned int w = __reduce_max_sync(0xffffffffu, __float_as_uint(v));
    if (warps == 1) return __uint_as_float(w);
    float* const s = slots + slot * kMaxWarps;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = __uint_as_float(w);
    __syncthreads();
    for (int i = 0; i < warps; ++i) w = ::max(w, __float_as_uint(s[first + i]));
    return __uint_as_float(w);
  }
};

// v to (v - mean) / sqrt(var + eps), or v / sqrt(mean v^2 + eps); the variance from the deviations, in a second pass over the
// registers.  Channels that are not there hold 0 and are left 0.
template <typename Valid>
__device__ __forceinline__ void normalize(float2 (&v)[16], const RowGroup& row, int slot, bool layer, float inv_k, float eps, Valid valid) {
  if (layer) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += v[i].x + v[i].y;
    const float mean = row.sum(s, slot) * inv_k;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (valid(i)) v[i] = make_float2(v[i].x - mean, v[i].y - mean);
  }
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; ++i) s = fmaf(v[i].x, v[i].x, fmaf(v[i].y, v[i].y, s));
  const float var = row.sum(s, slot + 1) * inv_k + eps;
  const float scale = 1.0f / sqrtf(var);
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = make_float2(v[i].x * scale, v[i].y * scale);
}

__device__ __forceinline__ void butterflies(float2 (&v)[16], int distance) {  // between registers `distance` apart
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if ((i & distance) == 0) rq::bfly2(v[i], v[i + distance]);
}

__device__ __forceinline__ void sts_quad(uint32_t a, const float2* v) {
  asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(a), "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y) : "memory");
}
__device__ __forceinline__ void lds_quad(uint32_t a, float2* v) {
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[0].x), "=f"(v[0].y), "=f"(v[1].x), "=f"(v[1].y) : "r"(a) : "memory");
}
__device__ __forceinline__ void sts_half(uint32_t a, float2 v) {
  asm volatile("st.shared.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(v.x), "f"(v.y) : "memory");
}

// R: the residual's type (Norm only); T: the rows', or the branch's and the outputs'.  kQuant: codes leave (else h only).
template <typename R, typename T, bool kNorm, bool kQuant, int kLayout, int kFmt>
__global__ void __launch_bounds__(kRowThreads, kNorm ? 1 : 2) rows_kernel(const RowsArgs a) {
  constexpr int kUnit = kLayout == kSixteen ? 2 : kLayout == kEight ? 4 : 8;  // channels a load moves
  constexpr int kUnits = 32 / kUnit, kPer = kUnit / 2;
  extern __shared__ __align__(128) uint8_t row_smem[];  // a line of 128 bytes per thread
  __shared__ float s_red[kSlots * kMaxWarps];

  const int tpr = a.row_warps * 32;
  const int rloc = static_cast<int>(threadIdx.x) / tpr, j = static_cast<int>(threadIdx.x) - rloc * tpr;
  const RowGroup row = {s_red, a.row_warps, rloc * a.row_warps};
  const int m = blockIdx.x * a.rows_per_cta + rloc;
  const bool here = m < a.M;
  const bool active = here && (kLayout == kPieces || j * 32 < a.K);

  // channel of unit u: first of kUnit consecutive ones
  const int log_c = a.log_b - 8;                        // kEight: index bits above a 256-channel group
  const int keep = kLayout == kEight ? 3 - log_c : 0;   // line bits that a thread keeps
  int base = 0;
  if constexpr (kLayout == kPlain) base = j * 32;
  if constexpr (kLayout == kFour) base = (j & ~3) * 32 + (j & 3) * 8;
  if constexpr (kLayout == kEight) {
    const int group = 8 << log_c;
    base = (j & ~(group - 1)) * 32 + (((j >> 3) & ((1 << log_c) - 1)) << (keep + 5)) + (j & 7) * 4;
  }
  if constexpr (kLayout == kSixteen) base = (j & ~127) * 32 + ((j >> 4) & 7) * 32 + (j & 15) * 2;
  auto channel = [&](int u) {
    if constexpr (kLayout == kPieces) return (j + u * tpr) * 8;
    if constexpr (kLayout == kPlain) return base + u * 8;
    if constexpr (kLayout == kFour) return base + u * 32;
    if constexpr (kLayout == kEight) return base + (u >> keep) * 256 + (u & ((1 << keep) - 1)) * 32;
    return base + u * 256;
  };
  auto valid = [&](int u) { return kLayout == kPieces ? here && channel(u) < a.K : active; };

  bool write = active;  // of codes: 32 channels of a row that is there

  griddep_wait();  // rows come from the previous kernel, which may still read what this one writes
  griddep_launch_dependents();

  float2 v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = make_float2(0.0f, 0.0f);
  if constexpr (!kNorm) {
    const T* const src = static_cast<const T*>(a.x) + static_cast<size_t>(m) * a.x_stride;
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
      if (valid(u)) load_unit<kUnit>(src + channel(u), v + u * kPer);
  } else {
    const float inv_k = 1.0f / static_cast<float>(a.K);
    const bool layer = a.norm.layer != 0;
    auto there = [&](int i) { return valid(i / kPer); };
    const R* const r = static_cast<const R*>(a.x) + static_cast<size_t>(m) * a.x_stride;
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
      if (valid(u)) load_unit<kUnit>(r + channel(u), v + u * kPer);
    // the token's row of the conditioning
    size_t mod = 0;
    bool mod_ok = here;
    if (a.norm.gate != nullptr || a.norm.scale != nullptr || a.norm.shift != nullptr) {
      int c = 0;
      if (here) c = a.norm.mod_index != nullptr ? a.norm.mod_index[m] : m / a.norm.mod_tokens;
      if (c < 0 || c >= a.norm.mod_rows) {
        mod_ok = false;
        if (here && j == 0) atomicOr(&g_error_word, kErrIndex);
      } else {
        mod = static_cast<size_t>(c) * a.norm.mod_stride;
      }
    }
    const bool live = mod_ok;  // a token whose index is out of range is skipped: nothing of it is written
    const T* const gate = static_cast<const T*>(a.norm.gate);
    const T* const scale = static_cast<const T*>(a.norm.scale);
    const T* const shift = static_cast<const T*>(a.norm.shift);
    const float off = a.norm.weight_offset;
    if (a.y != nullptr) {
      float2 w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = make_float2(0.0f, 0.0f);
      const T* const y = static_cast<const T*>(a.y) + static_cast<size_t>(m) * a.y_stride;
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
        if (valid(u)) load_unit<kUnit>(y + channel(u), w + u * kPer);
      if (a.norm.post_norm) normalize(w, row, 0, layer, inv_k, a.norm.eps, there);
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        if (!valid(u) || !live) continue;
        float2 t[kPer];
        if (a.norm.post_weight != nullptr) {
          load_unit<kUnit>(static_cast<const T*>(a.norm.post_weight) + channel(u), t);
#pragma unroll
          for (int i = 0; i < kPer; ++i) w[u * kPer + i] = make_float2(w[u * kPer + i].x * (t[i].x + off), w[u * kPer + i].y * (t[i].y + off));
        }
        if (gate != nullptr) {
          load_unit<kUnit>(gate + mod + channel(u), t);
#pragma unroll
          for (int i = 0; i < kPer; ++i) w[u * kPer + i] = make_float2(w[u * kPer + i].x * t[i].x, w[u * kPer + i].y * t[i].y);
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        v[i] = make_float2(fmaf(a.norm.residual_scale, v[i].x, w[i].x), fmaf(a.norm.residual_scale, v[i].y, w[i].y));
    } else if (a.norm.residual_scale != 1.0f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = make_float2(a.norm.residual_scale * v[i].x, a.norm.residual_scale * v[i].y);
    }
    R* const out = static_cast<R*>(a.residual_out) + static_cast<size_t>(m) * a.x_stride;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (!valid(u)) continue;
      if constexpr (sizeof(R) == 4) {
        if (a.residual_out != nullptr && live) store_unit<kUnit>(out + channel(u), v + u * kPer);
      } else {
        store_unit<kUnit>(a.residual_out != nullptr && live ? out + channel(u) : static_cast<R*>(nullptr), v + u * kPer);
      }
    }
    if (!kQuant && a.h == nullptr) return;  // the residual alone (the same for every thread)
    normalize(v, row, 2, layer, inv_k, a.norm.eps, there);
    T* const h = static_cast<T*>(a.h) + static_cast<size_t>(m) * a.K;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      if (!valid(u) || !live) continue;
      float2 t[kPer];
      float2* const p = v + u * kPer;
      if (a.norm.pre_weight != nullptr) {
        load_unit<kUnit>(static_cast<const T*>(a.norm.pre_weight) + channel(u), t);
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = make_float2(p[i].x * (t[i].x + off), p[i].y * (t[i].y + off));
      }
      if (a.norm.pre_bias != nullptr) {
        load_unit<kUnit>(static_cast<const T*>(a.norm.pre_bias) + channel(u), t);
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = make_float2(p[i].x + t[i].x, p[i].y + t[i].y);
      }
      if (scale != nullptr) {
        load_unit<kUnit>(scale + mod + channel(u), t);
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = make_float2(p[i].x * (1.0f + t[i].x), p[i].y * (1.0f + t[i].y));
      }
      if (shift != nullptr) {
        load_unit<kUnit>(shift + mod + channel(u), t);
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = make_float2(p[i].x + t[i].x, p[i].y + t[i].y);
      }
      store_unit<kUnit>(a.h != nullptr ? h + channel(u) : static_cast<T*>(nullptr), p);  // the quantiser reads what is stored
    }
    if (!live) {
#pragma unroll
      for (int i = 0; i < 16; ++i) v[i] = make_float2(0.0f, 0.0f);
      write = false;
    }
  }
  if constexpr (!kQuant) return;

  // ---- rotation, to 32 consecutive channels a thread ----
  const uint32_t lines = smem_u32(row_smem) + static_cast<uint32_t>(rloc * tpr * 128);  // of this row
  if constexpr (kLayout == kFour) {
    if (a.log_b == 7) butterflies(v, 8);
    butterflies(v, 4);
    // quad i of line t at piece i ^ f(t), f = 0 2 4 6 1 3 5 7 over 8 lines: two groups' pieces fall on all eight
    const int g = (j >> 2) & 1;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t line = lines + static_cast<uint32_t>(((j & ~3) + u) * 128);
      const int f = 2 * u + g, p = 2 * (j & 3);
      sts_quad(line + ((p ^ f) << 4), v + 4 * u);
      sts_quad(line + (((p + 1) ^ f) << 4), v + 4 * u + 2);
    }
    __syncwarp();
    const uint32_t own = lines + static_cast<uint32_t>(j * 128);
    const int f = 2 * (j & 3) + g;
#pragma unroll
    for (int i = 0; i < 8; ++i) lds_quad(own + ((i ^ f) << 4), v + 2 * i);
  }
  if constexpr (kLayout == kEight || kLayout == kSixteen) {
    const int q = j & 7;
    if (kLayout == kSixteen) {
#pragma unroll
      for (int s = 3; s >= 0; --s) butterflies(v, 1 << s);
      const int l = (j >> 4) & 7, qq = (j >> 1) & 7;
      const uint32_t at = lines + static_cast<uint32_t>(((j & ~127) + l) * 128 + ((qq ^ l) << 4) + (j & 1) * 8);
#pragma unroll
      for (int h = 0; h < 16; ++h) sts_half(at + h * 1024, v[h]);
      __syncthreads();
    } else if (log_c > 0) {
      // stages over the group index, whose bits lie above the kept line bits of the unit
      butterflies(v, 8);
      if (log_c > 1) butterflies(v, 4);
      if (log_c > 2) butterflies(v, 2);
      const int group = 8 << log_c, la = ((j >> 3) & ((1 << log_c) - 1)) << keep;
      const uint32_t block = lines + static_cast<uint32_t>((j & ~(group - 1)) * 128);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int l = la | (u & ((1 << keep) - 1));
        sts_quad(block + static_cast<uint32_t>(((u >> keep) * 8 + l) * 128 + ((q ^ l) << 4)), v + 2 * u);
      }
      if (log_c > 2) {  // a block of 2048 is two warps
        __syncthreads();
      } else {
        __syncwarp();
      }
    }
    const uint32_t grp = lines + static_cast<uint32_t>((j & ~7) * 128);
    if (kLayout == kSixteen || log_c > 0) {
#pragma unroll
      for (int l = 0; l < 8; ++l) lds_quad(grp + static_cast<uint32_t>(l * 128 + ((q ^ l) << 4)), v + 2 * l);
    }
    butterflies(v, 8);
    butterflies(v, 4);
    butterflies(v, 2);
#pragma unroll
    for (int l = 0; l < 8; ++l) sts_quad(grp + static_cast<uint32_t>(l * 128 + ((q ^ l) << 4)), v + 2 * l);
    __syncwarp();
    const uint32_t own = lines + static_cast<uint32_t>(j * 128);
#pragma unroll
    for (int i = 0; i < 8; ++i) lds_quad(own + ((i ^ q) << 4), v + 2 * i);
  }
  if (a.log_b > 0) {
    const int n = kLayout == kPlain ? a.log_b : 5;  // stages among a thread's 32 channels
    if (n > 4) butterflies(v, 8);
    if (n > 3) butterflies(v, 4);
    if (n > 2) butterflies(v, 2);
    if (n > 1) butterflies(v, 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float s = v[i].x + v[i].y, d = v[i].x - v[i].y;
      v[i] = make_float2(s * a.inv_sqrt_b, d * a.inv_sqrt_b);
    }
  }

  // ---- scales and codes ----
  float top[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    float t = 0.0f;
#pragma unroll
    for (int i = 8 * b; i < 8 * b + 8; ++i) t = rq::max_nan(t, rq::max_nan(fabsf(v[i].x), fabsf(v[i].y)));
    top[b] = t;
  }
  uint32_t code[4];
  if constexpr (kFmt == kMx) {
    const uint32_t t = __float_as_uint(rq::max_nan(top[0], top[1]));
    uint32_t byte = 0;
    float to_codes = 0.0f;  // 2^-e
    if (t >= 0x7F800000u) {
      byte = 255u;  // an infinity or NaN: the block has no values
    } else if (t != 0u) {
      // floor(log2) - 2, of a subnormal below the clamp at -127 anyway
      const int e = max(static_cast<int>(t >> 23) - 127 - 2, -127);
      byte = static_cast<uint32_t>(e + 127);
      to_codes = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);  // (e <= 125; e = -127 gives 2^127)
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {  // the products are exact
      float2 s[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = make_float2(v[4 * c + i].x * to_codes, v[4 * c + i].y * to_codes);
      code[c] = e2m1x8(s[0], s[1], s[2], s[3]);
    }
    // the four threads of a tile's group hand their bytes to the first
    uint32_t w = byte << (8 * (j & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    if (write && (j & 3) == 0) *reinterpret_cast<uint32_t*>(a.scales + scale_offset(m, j, a.K >> 7)) = w;
  } else {
    float delta;
    if (a.step_scale != nullptr) {
      delta = __ldg(a.step_scale);
    } else {
      delta = __fdiv_rn(row.max(rq::max_nan(top[0], top[1]), 4), kRowMax);
      if (isinf(delta)) delta = __int_as_float(0x7FC00000);
    }
    if (write && j == 0) a.row_scale[m] = delta;
    uint32_t bytes = 0;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t s = delta > 0.0f && !isinf(delta) ? block_scale_e4m3(top[b], delta) : 0u;
      bytes |= s << (8 * b);
      const float d = e4m3_value(s) * delta;
      const bool easy = d >= 8.673617379884035e-19f && d <= 1.152921504606846976e18f;  // 2^-60 .. 2^60
      const float r = easy ? __frcp_rn(d) : 0.0f;
      // The float32 quotient is within 2^-22 of the exact one: where it rounds alike moved up and down by 2^-20 it decides.
      const float up = r * 1.00000095367431640625f, dn = r * 0.99999904632568359375f;
#pragma unroll
      for (int c = 2 * b; c < 2 * b + 2; ++c) {
        float2 h[4], l[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          h[i] = make_float2(v[4 * c + i].x * up, v[4 * c + i].y * up);
          l[i] = make_float2(v[4 * c + i].x * dn, v[4 * c + i].y * dn);
        }
        uint32_t w = e2m1x8(h[0], h[1], h[2], h[3]);
        if (w != e2m1x8(l[0], l[1], l[2], l[3]) || (!easy && d > 0.0f)) {
          w = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            w |= (code_exact(v[4 * c + i].x, d) << (8 * i)) | (code_exact(v[4 * c + i].y, d) << (8 * i + 4));
        }
        code[c] = w;
      }
    }
    uint32_t w = bytes << (16 * (j & 1));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    if (write && (j & 1) == 0) *reinterpret_cast<uint32_t*>(a.scales + scale_offset(m, 2 * j, a.K >> 6)) = w;
  }
  if (write) *reinterpret_cast<uint4*>(a.codes + static_cast<size_t>(m) * (a.K >> 1) + j * 16) = make_uint4(code[0], code[1], code[2], code[3]);
}

template <typename R, typename T, bool kNorm, bool kQuant, int kLayout, int kFmt>
cudaError_t launch_rows(RowsArgs a) {
  const int threads = kLayout == kPieces ? (a.K + 31) / 32 : a.K / 32;
  a.row_warps = (threads + 31) / 32;
  int rows = a.row_warps >= 8 ? 1 : 8 / a.row_warps;
  while (rows > 1 && (a.M + rows - 1) / rows < a.num_sms) rows /= 2;  // few rows: more CTAs
  a.rows_per_cta = rows;
  const int tpb = rows * a.row_warps * 32;
  auto kern = rows_kernel<R, T, kNorm, kQuant, kLayout, kFmt>;
  const size_t smem = kQuant && kLayout != kPlain && kLayout != kPieces ? static_cast<size_t>(tpb) * 128 : 0;
  if (smem > 40 * 1024) {
    static std::atomic<unsigned long long> raised{0};  // devices whose limit has been raised to the most any K asks for
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = 1ull << (dev & 63);
    if (!(raised.load() & bit)) {
      e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRowThreads * 128);
      if (e != cudaSuccess) return e;
      raised.fetch_or(bit);
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.M + rows - 1) / rows));
  cfg.blockDim = dim3(static_cast<unsigned>(tpb));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;  // may overlap the previous kernel
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kern, a);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <typename R, typename T, bool kNorm, int kFmt>
cudaError_t launch_quant_layout(const RowsArgs& a) {
  if (a.log_b <= 5) return launch_rows<R, T, kNorm, true, kPlain, kFmt>(a);
  if (a.log_b <= 7) return launch_rows<R, T, kNorm, true, kFour, kFmt>(a);
  if (a.log_b <= 11) return launch_rows<R, T, kNorm, true, kEight, kFmt>(a);
  return launch_rows<R, T, kNorm, true, kSixteen, kFmt>(a);
}

template <typename R, typename T, bool kNorm>
cudaError_t launch_quant(const RowsArgs& a) {
  return a.fmt == kMx ? launch_quant_layout<R, T, kNorm, kMx>(a) : launch_quant_layout<R, T, kNorm, kNv>(a);
}

}  // namespace fp4
}  // namespace qvla
