// What runs between two quantised products, a row at a time: the residual's update and the norms around a block, the Hadamard
// rotation and the quantiser to 4-bit floating point, in one pass over memory.
//
//   branch   u = y, or norm(y) (post_w + offset);  r' = R(a r + g u), R the residual's type
//   norm     h = T(norm(r') (pre_w + offset) + pre_b), with conditioning T((...)(1 + scale) + shift)
//   rotation z = h BlockDiag(H_b / sqrt b): float32 butterflies, the longest distance first, one product with 1/sqrt(b)
//   codes    MX and NV as in fp4.cuh
//
// The norm wants many loads in flight and few registers: 8 or 16 channels a thread, a row's operands asked for during the sums
// of the one before.  The rotation and the quantiser want many channels a thread: 32, the loads taking
// them as the rotation's first stages want them,
//   kPlain    b <= 32: 32 consecutive channels
//   kFour     b = 64, 128: of the 4 lines (32 channels each) of 128 channels, thread p of 4 holds quads 2p, 2p + 1 of each
//   256 ..    b = 256 to 2048: thread q of 8 holds quad q of 8 lines, which differ in the high bits of the block's index
//   4096      half a quad of 16 lines
// and one or two exchanges through shared memory (128 bytes a thread) end with 32 consecutive channels a thread, which is what
// the quantiser wants: one MX block or two NV blocks, 16 bytes of codes.  Running the stages from the longest distance
// down is what makes that the end and not the beginning.  Where both run, a group of threads norms 4 rows (2 beyond 8192
// channels) into shared memory, and then each quarter of it rotates and quantises one.
#pragma once

#include <algorithm>

#include "fp4.cuh"
#include "griddep.cuh"
#include "kernels.h"
#include "ptx.cuh"
#include "rotate_quant.cuh"

namespace qvla {
namespace fp4 {

// Layouts of the rotation by log2 of the block: 8 .. 12 stand for themselves.
constexpr int kPlain = 5, kFour = 7;

constexpr int kRowThreads = 512;   // most threads of a quantised row's CTA (K = 16384)
constexpr int kNormThreads = 1024;
constexpr int kMaxWarps = 32;

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
// Eight values as T; rounded to T and back; in memory.
template <typename T>
__device__ __forceinline__ uint4 pack_unit(const float2* v, T t) {
  return make_uint4(narrow(v[0], t), narrow(v[1], t), narrow(v[2], t), narrow(v[3], t));
}
template <typename T>
__device__ __forceinline__ void round_unit(float2* v, T t) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = widen(narrow(v[i], t), t);
}
template <typename T>
__device__ __forceinline__ void write_unit(T* p, const float2* v) {
  *reinterpret_cast<uint4*>(p) = pack_unit(v, T());
}
__device__ __forceinline__ void write_unit(float* p, const float2* v) {
  reinterpret_cast<float4*>(p)[0] = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
  reinterpret_cast<float4*>(p)[1] = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
}

// A row's place among the CTA's warps, and sums and maxima over it.  Every thread of the CTA makes the same calls.
struct RowGroup {
  float* slots;             // [slot][kMaxWarps]
  int warps, first, span;   // of the row: its warps, the first, and their number rounded up to a power of two
  __device__ __forceinline__ RowGroup(float* s, int w, int f) : slots(s), warps(w), first(f), span(1) {
    while (span < w) span *= 2;
  }
  __device__ __forceinline__ float sum(float v, int slot) const {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (warps == 1) return v;
    float* const s = slots + slot * kMaxWarps;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    // every warp adds the warps' sums in the same order
    const int w = static_cast<int>(threadIdx.x) & (span - 1);
    v = w < warps ? s[first + w] : 0.0f;
    for (int o = span >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
  }
  // The largest; NaN if one is (bit patterns of non-negative floats order like the numbers, NaN above infinity).
  __device__ __forceinline__ float max(float v, int slot) const {
    unsigned int w = __reduce_max_sync(0xffffffffu, __float_as_uint(v));
    if (warps == 1) return __uint_as_float(w);
    float* const s = slots + slot * kMaxWarps;
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = __uint_as_float(w);
    __syncthreads();
    const int lane = threadIdx.x & 31;
    return __uint_as_float(__reduce_max_sync(0xffffffffu, lane < warps ? __float_as_uint(s[first + lane]) : 0u));
  }
};

// ---- the norms ----------------------------------------------------------------------------------------------------------

// N 16-byte pieces of a row of T (float32: 2 N of them), 8 channels each, as they lie in memory.
template <typename T, int N>
struct Raw {
  static constexpr int kPer = sizeof(T) == 4 ? 2 : 1;
  uint4 q[N * kPer];
  __device__ __forceinline__ void load(int i, const T* p) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) q[i * kPer + k] = reinterpret_cast<const uint4*>(p)[k];
  }
  __device__ __forceinline__ float2 pair(int i) const {  // channels 2 i and 2 i + 1
    if constexpr (kPer == 2) {
      const uint4 w = q[i >> 1];
      return (i & 1) ? make_float2(__uint_as_float(w.z), __uint_as_float(w.w)) : make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    } else {
      const uint4 w = q[i >> 2];
      return widen((i & 3) == 0 ? w.x : (i & 3) == 1 ? w.y : (i & 3) == 2 ? w.z : w.w, T());
    }
  }
};

// v to v - mean with `layer`, and what it then has to be multiplied by: 1 / sqrt(mean v^2 + eps), the variance from the
// deviations in a second pass over the registers.  A thread without channels adds nothing, whatever it holds.  k: the channels,
// and their reciprocal.  (IEEE division and square root by every thread took 120 of a row's 430 instructions; the reciprocal square
// root is within 2^-22.)
template <int N>
__device__ __forceinline__ float sum_there(const float2 (&s)[N], const bool (&has)[N]) {
  float t = 0.0f;
#pragma unroll
  for (int i = 0; i < N; ++i) t += has[i] ? s[i].x + s[i].y : 0.0f;
  return t;
}
template <int N>
__device__ __forceinline__ float norm_scale(float2 (&v)[4 * N], const bool (&has)[N], const RowGroup& row, int slot, bool layer, float2 k, float eps) {
  float2 s[N];
  if (layer) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = __fadd2_rn(__fadd2_rn(v[4 * i], v[4 * i + 1]), __fadd2_rn(v[4 * i + 2], v[4 * i + 3]));
    const float sum = row.sum(sum_there<N>(s, has), slot), near = sum * k.y;
    const float mean = fmaf(fmaf(-near, k.x, sum), k.y, near);  // the quotient to its last bit: of equal channels it is their value
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) v[i] = __fadd2_rn(v[i], both(-mean));
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    s[i] = __fmul2_rn(v[4 * i], v[4 * i]);
#pragma unroll
    for (int q = 1; q < 4; ++q) s[i] = __ffma2_rn(v[4 * i + q], v[4 * i + q], s[i]);
  }
  return rsqrtf(fmaf(row.sum(sum_there<N>(s, has), slot + 1), k.y, eps));
}

// A group of threads takes rows m, m + step, ... (`rows` of them, those below M): thread j its pieces j, j + threads, ...  h goes
// to global memory where it is wanted, and with `store` (row number, channel, 8 values as T) to the caller.
// kMods, kPost: conditioning and branch norm may be there (without, their code is not).
template <typename R, typename T, int N, bool kMods, bool kPost, typename Store>
__device__ __forceinline__ void norm_rows(const RowsArgs& a, const RowGroup& row, int j, int m, int step, int rows, Store store) {
  const float2 width = make_float2(static_cast<float>(a.K), 1.0f / static_cast<float>(a.K));
  const float2 off = both(a.norm.weight_offset), alpha = both(a.norm.residual_scale);
  const bool layer = a.norm.layer != 0, norm_h = a.h != nullptr || a.codes != nullptr;
  const bool branch = a.y != nullptr, gated = kMods && branch && a.norm.gate != nullptr;
  const bool mods = kMods && (a.norm.gate != nullptr || a.norm.scale != nullptr || a.norm.shift != nullptr);
  // Channels of the thread's pieces.  A piece beyond the row reads the row's first one, so that loads need no branch (with branches
  // the values that are never there cost 200 to 400 bytes of spills), and adds nothing to sums.
  const int first = j * 8, apart = row.warps * 256;
  bool has[N];
  int at[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    has[i] = first + i * apart < a.K;
    at[i] = has[i] ? first + i * apart : 0;
  }
  // Weights and conditioning stay in registers from the row's start; with two pieces a thread they are loaded at their use.
  constexpr bool kHold = N == 1;
  auto take = [&](Raw<T, N>& to, const void* from, size_t mod) {
#pragma unroll
    for (int i = 0; i < N; ++i) to.load(i, static_cast<const T*>(from) + mod + at[i]);
  };
  // f(i, pair i) of a vector: held since the row's start, or loaded now
  size_t mod = 0;
  auto with = [&](const Raw<T, kHold ? N : 1>& held, const void* from, size_t place, auto f) {
    if constexpr (kHold) {
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) f(i, held.pair(i));
    } else {
      Raw<T, N> t;
      take(t, from, place);
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) f(i, t.pair(i));
    }
  };
  Raw<T, kHold ? N : 1> post_w, pre_w, pre_b;  // the same for every row
  griddep_wait();  // everything comes from earlier kernels, which may still read what this one writes
  griddep_launch_dependents();
  if constexpr (kHold) {
    if (kPost && a.norm.post_weight != nullptr) take(post_w, a.norm.post_weight, 0);
    if (a.norm.pre_weight != nullptr) take(pre_w, a.norm.pre_weight, 0);
    if (a.norm.pre_bias != nullptr) take(pre_b, a.norm.pre_bias, 0);
  }

  Raw<R, N> r;  // the operands of the row in work, soon those of the next
  Raw<T, N> y;
  auto fetch = [&](int number) {
    const R* const px = static_cast<const R*>(a.x) + static_cast<size_t>(number) * a.x_stride;
    const T* const py = static_cast<const T*>(a.y) + static_cast<size_t>(number) * a.y_stride;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      r.load(i, px + at[i]);
      if (branch) y.load(i, py + at[i]);
    }
  };
  if (m < a.M) fetch(m);
  for (int k = 0; k < rows; ++k) {
    const int slot = (k & 1) * 4;
    bool live = m < a.M;
    Raw<T, kHold ? N : 1> g, sc, sh;
    if (mods) {  // the token's row of the conditioning; a token whose index is out of range is skipped: nothing of it is written
      const int c = !live ? 0 : a.norm.mod_index != nullptr ? a.norm.mod_index[m] : m / a.norm.mod_tokens;
      if (c < 0 || c >= a.norm.mod_rows) {
        if (live && j == 0) atomicOr(&g_error_word, kErrIndex);
        live = false;
      }
      mod = live ? static_cast<size_t>(c) * a.norm.mod_stride : 0;
      if constexpr (kHold) {
        if (gated) take(g, a.norm.gate, mod);
        if (a.norm.scale != nullptr) take(sc, a.norm.scale, mod);
        if (a.norm.shift != nullptr) take(sh, a.norm.shift, mod);
      }
    }
    float2 v[4 * N];
    if (branch) {
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) v[i] = y.pair(i);
      if (kPost && a.norm.post_norm) {
        const float2 s = both(norm_scale<N>(v, has, row, slot, layer, width, a.norm.eps));
#pragma unroll
        for (int i = 0; i < 4 * N; ++i) v[i] = __fmul2_rn(v[i], s);
        if (a.norm.post_weight != nullptr) with(post_w, a.norm.post_weight, 0, [&](int i, float2 w) { v[i] = __fmul2_rn(v[i], __fadd2_rn(w, off)); });
      }
      if (gated) with(g, a.norm.gate, mod, [&](int i, float2 w) { v[i] = __fmul2_rn(v[i], w); });
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) v[i] = __ffma2_rn(alpha, r.pair(i), v[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4 * N; ++i) v[i] = __fmul2_rn(alpha, r.pair(i));
    }
    const bool write_r = a.residual_out != nullptr && live;
    R* const po = static_cast<R*>(a.residual_out) + static_cast<size_t>(m) * a.x_stride;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(R) == 2) round_unit(v + 4 * i, R());
      if (write_r && has[i]) write_unit(po + at[i], v + 4 * i);
    }
    T* const ph = static_cast<T*>(a.h) + static_cast<size_t>(m) * a.K;
    m += step;
    // (A caller may update the residual in place, and have h where y is: a thread has its pieces of a row in registers before it writes
    // them, another one reads them only where it has no channels and uses none, and other rows are other memory.)
    if (k + 1 < rows && m < a.M) fetch(m);
    if (!norm_h) continue;
    const float2 s = both(norm_scale<N>(v, has, row, slot + 2, layer, width, a.norm.eps));
#pragma unroll
    for (int i = 0; i < 4 * N; ++i) v[i] = __fmul2_rn(v[i], s);
    if (a.norm.pre_weight != nullptr) with(pre_w, a.norm.pre_weight, 0, [&](int i, float2 w) { v[i] = __fmul2_rn(v[i], __fadd2_rn(w, off)); });
    if (a.norm.pre_bias != nullptr) with(pre_b, a.norm.pre_bias, 0, [&](int i, float2 w) { v[i] = __fadd2_rn(v[i], w); });
    if (kMods && a.norm.scale != nullptr) with(sc, a.norm.scale, mod, [&](int i, float2 w) { v[i] = __fmul2_rn(v[i], __fadd2_rn(w, both(1.0f))); });
    if (kMods && a.norm.shift != nullptr) with(sh, a.norm.shift, mod, [&](int i, float2 w) { v[i] = __fadd2_rn(v[i], w); });
    const bool write_h = a.h != nullptr && live;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (!has[i]) continue;
      const uint4 h = pack_unit(v + 4 * i, T());
      if (write_h) *reinterpret_cast<uint4*>(ph + at[i]) = h;
      store(k, at[i], h, live);
    }
  }
}

// ---- rotation and quantiser -----------------------------------------------------------------------------------------------

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

// Where the thread's channels of a row lie ahead of the rotation.
template <int kLayout>
struct Place {
  static constexpr int kUnit = kLayout == 12 ? 2 : kLayout > kFour ? 4 : 8;  // channels a load moves
  static constexpr int kUnits = 32 / kUnit, kPer = kUnit / 2;
  static constexpr int kLogC = kLayout - 8, kKeep = kLayout > kFour && kLayout < 12 ? 3 - kLogC : 0;  // 256 ..: index bits above a 256-channel group, line bits that a thread keeps
  int base;
  __device__ __forceinline__ explicit Place(int j) {
    if constexpr (kLayout == kPlain) base = j * 32;
    if constexpr (kLayout == kFour) base = (j & ~3) * 32 + (j & 3) * 8;
    if constexpr (kLayout > kFour && kLayout < 12) {
      constexpr int kGroup = 8 << kLogC;
      base = (j & ~(kGroup - 1)) * 32 + (((j >> 3) & ((1 << kLogC) - 1)) << (kKeep + 5)) + (j & 7) * 4;
    }
    if constexpr (kLayout == 12) base = (j & ~127) * 32 + ((j >> 4) & 7) * 32 + (j & 15) * 2;
  }
  __device__ __forceinline__ int channel(int u) const {  // of unit u
    if constexpr (kLayout == kPlain) return base + u * 8;
    if constexpr (kLayout == kFour) return base + u * 32;
    if constexpr (kLayout == 12) return base + u * 256;
    return base + (u >> kKeep) * 256 + (u & ((1 << kKeep) - 1)) * 32;
  }
};

template <bool kNamed, int kThreads>
__device__ __forceinline__ void block_sync() {
  if constexpr (kNamed) {
    asm volatile("bar.sync %0, %1;" ::"r"(1 + static_cast<int>(threadIdx.x) / kThreads), "n"(kThreads) : "memory");
  } else {
    __syncthreads();
  }
}

// Thread j of a row holds v as Place<kLayout> says and leaves with its 32 consecutive channels, rotated; `lines` is the row's
// shared memory, 128 bytes a thread.  kNamed: at most 512 threads, so that the 64 or 128 of a block of 2048 or 4096 have a barrier of
// their own (1 and up); without, every thread of the CTA calls this.
template <int kLayout, bool kNamed>
__device__ __forceinline__ void rotate(int log_b, float inv_sqrt_b, int j, uint32_t lines, float2 (&v)[16]) {
  if constexpr (kLayout == kFour) {
    if (log_b == 7) butterflies(v, 8);
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
  if constexpr (kLayout > kFour) {
    const int q = j & 7;
    if constexpr (kLayout == 12) {
#pragma unroll
      for (int s = 3; s >= 0; --s) butterflies(v, 1 << s);
      const int l = (j >> 4) & 7, qq = (j >> 1) & 7;
      const uint32_t at = lines + static_cast<uint32_t>(((j & ~127) + l) * 128 + ((qq ^ l) << 4) + (j & 1) * 8);
#pragma unroll
      for (int h = 0; h < 16; ++h) sts_half(at + h * 1024, v[h]);
      block_sync<kNamed, 128>();
    } else if constexpr (kLayout > 8) {
      using P = Place<kLayout>;
      constexpr int log_c = P::kLogC, keep = P::kKeep;
      // stages over the group index, whose bits lie above the kept line bits of the unit
      butterflies(v, 8);
      if constexpr (log_c > 1) butterflies(v, 4);
      if constexpr (log_c > 2) butterflies(v, 2);
      constexpr int group = 8 << log_c;
      const int la = ((j >> 3) & ((1 << log_c) - 1)) << keep;
      const uint32_t block = lines + static_cast<uint32_t>((j & ~(group - 1)) * 128);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int l = la | (u & ((1 << keep) - 1));
        sts_quad(block + static_cast<uint32_t>(((u >> keep) * 8 + l) * 128 + ((q ^ l) << 4)), v + 2 * u);
      }
      if constexpr (log_c > 2) {  // a block of 2048 is two warps
        block_sync<kNamed, 64>();
      } else {
        __syncwarp();
      }
    }
    const uint32_t grp = lines + static_cast<uint32_t>((j & ~7) * 128);
    if constexpr (kLayout > 8) {
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
  if (log_b > 0) {
    const int n = kLayout == kPlain ? log_b : 5;  // stages among a thread's 32 channels
    if (n > 4) butterflies(v, 8);
    if (n > 3) butterflies(v, 4);
    if (n > 2) butterflies(v, 2);
    if (n > 1) butterflies(v, 1);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      v[i] = __fmul2_rn(make_float2(v[i].x + v[i].y, v[i].x - v[i].y), both(inv_sqrt_b));
    }
  }
}

// The largest magnitude of each half of a thread's channels, NaN if one is.
__device__ __forceinline__ void magnitudes(const float2 (&v)[16], float (&top)[2]) {
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    float t = 0.0f;
#pragma unroll
    for (int i = 8 * b; i < 8 * b + 8; ++i) t = rq::max_nan(t, rq::max_nan(fabsf(v[i].x), fabsf(v[i].y)));
    top[b] = t;
  }
}

// A thread's MX block: its scale's byte.
__device__ __forceinline__ uint32_t encode_mx(const float2 (&v)[16], const float (&top)[2], uint32_t (&code)[4]) {
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
    for (int i = 0; i < 4; ++i) s[i] = __fmul2_rn(v[4 * c + i], both(to_codes));
    code[c] = e2m1x8(s[0], s[1], s[2], s[3]);
  }
  return byte;
}

// A row's scale by its largest magnitude.
__device__ __forceinline__ float row_scale(float most) {
  const float delta = __fdiv_rn(most, kRowMax);
  return isinf(delta) ? __int_as_float(0x7FC00000) : delta;
}

// A thread's two NV blocks: their scales' bytes, the first in the low one.
__device__ __forceinline__ uint32_t encode_nv(const float2 (&v)[16], const float (&top)[2], float delta, uint32_t (&code)[4]) {
  uint32_t bytes = 0;
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    const uint32_t s = delta > 0.0f && !isinf(delta) ? block_scale_e4m3(top[b], delta) : 0u;
    bytes |= s << (8 * b);
    const float d = e4m3_value(s) * delta;
    const bool easy = d >= 8.673617379884035e-19f && d <= 1.152921504606846976e18f;  // 2^-60 .. 2^60
    const float r = easy ? near_reciprocal(d) : 0.0f;
    // The float32 quotient is within 2^-22 of the exact one: where it rounds alike moved up and down by 2^-20 it decides.
    const float up = r * 1.00000095367431640625f, dn = r * 0.99999904632568359375f;
#pragma unroll
    for (int c = 2 * b; c < 2 * b + 2; ++c) {
      float2 h[4], l[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        h[i] = __fmul2_rn(v[4 * c + i], both(up));
        l[i] = __fmul2_rn(v[4 * c + i], both(dn));
      }
      uint32_t w = e2m1x8(h[0], h[1], h[2], h[3]);
      const uint32_t low = e2m1x8(l[0], l[1], l[2], l[3]);
      if (w != low) w = decide_codes(low, w, v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3], d);
      if (!easy && d > 0.0f) w = codes_exact(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3], d);
      code[c] = w;
    }
  }
  return bytes;
}

// Rotates v (as above) and leaves codes, block scales and the row's.  write: the row and the thread's channels are there.  Every thread
// of the CTA calls this.
template <int kLayout, int kFmt, bool kNamed>
__device__ __forceinline__ void rotate_quantize(const RowsArgs& a, const RowGroup& row, int slot, int j, int m, bool write, uint32_t lines,
                                                float2 (&v)[16]) {
  rotate<kLayout, kNamed>(a.log_b, a.inv_sqrt_b, j, lines, v);
  float top[2];
  magnitudes(v, top);
  uint32_t code[4];
  if constexpr (kFmt == kMx) {
    // the four threads of a tile's group hand their bytes to the first
    uint32_t w = encode_mx(v, top, code) << (8 * (j & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    if (write && (j & 3) == 0) *reinterpret_cast<uint32_t*>(a.scales + scale_offset(m, j, a.K >> 7)) = w;
  } else {
    const float delta = a.step_scale != nullptr ? *a.step_scale : row_scale(row.max(rq::max_nan(top[0], top[1]), slot));
    if (write && j == 0) a.row_scale[m] = delta;
    uint32_t w = encode_nv(v, top, delta, code) << (16 * (j & 1));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    if (write && (j & 1) == 0) *reinterpret_cast<uint32_t*>(a.scales + scale_offset(m, 2 * j, a.K >> 6)) = w;
  }
  if (write) *reinterpret_cast<uint4*>(a.codes + static_cast<size_t>(m) * (a.K >> 1) + j * 16) = make_uint4(code[0], code[1], code[2], code[3]);
}

template <typename T, int kLayout, int kFmt>
__global__ void __launch_bounds__(kRowThreads, 2) quantize_rows_kernel(const RowsArgs a) {
  using P = Place<kLayout>;
  extern __shared__ __align__(128) uint8_t row_smem[];
  __shared__ float s_red[kMaxWarps];
  const int tpr = a.row_warps * 32;
  const int rloc = static_cast<int>(threadIdx.x) / tpr, j = static_cast<int>(threadIdx.x) - rloc * tpr;
  const RowGroup row(s_red, a.row_warps, rloc * a.row_warps);
  const int m = blockIdx.x * a.group_rows + rloc;
  const bool active = m < a.M && j * 32 < a.K;
  const P place(j);
  griddep_wait();  // rows come from the previous kernel, which may still read what this one writes
  griddep_launch_dependents();
  float2 v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = make_float2(0.0f, 0.0f);
  if (active) {
    const T* const src = static_cast<const T*>(a.x) + static_cast<size_t>(m) * a.x_stride;
#pragma unroll
    for (int u = 0; u < P::kUnits; ++u) load_unit<P::kUnit>(src + place.channel(u), v + u * P::kPer);
  }
  rotate_quantize<kLayout, kFmt, true>(a, row, 0, j, m, active, smem_u32(row_smem) + static_cast<uint32_t>(rloc * tpr * 128), v);
}

// Norm, rotation and quantiser.  A group of a.row_warps warps norms a.group_rows rows into shared memory (as T), one after the
// other; then the CTA's warps are dealt to the rows anew, K / 32 threads each.
template <typename R, typename T, int N, bool kPlainNorm, int kLayout, int kFmt>
__global__ void __launch_bounds__(kNormThreads, 1) norm_quantize_kernel(const RowsArgs a) {
  using P = Place<kLayout>;
  extern __shared__ __align__(128) uint8_t row_smem[];  // the rows as T; then a line of 128 bytes per thread
  __shared__ float s_red[8 * kMaxWarps];
  const int tpg = a.row_warps * 32;
  const int g = static_cast<int>(threadIdx.x) / tpg, j1 = static_cast<int>(threadIdx.x) - g * tpg;
  const int groups = static_cast<int>(blockDim.x) / tpg, m0 = blockIdx.x * groups * a.group_rows;
  T* const hs = reinterpret_cast<T*>(row_smem);
  __shared__ unsigned int s_live;  // rows that are there and whose conditioning is
  if (threadIdx.x == 0) s_live = 0u;
  __syncthreads();
  {
    const RowGroup group(s_red, a.row_warps, g * a.row_warps);
    // (rows of a group lie next to one another)
    norm_rows<R, T, N, !kPlainNorm, !kPlainNorm>(a, group, j1, m0 + g * a.group_rows, 1, a.group_rows, [&](int k, int channel, uint4 h, bool live) {
      const int r = g * a.group_rows + k;
      *reinterpret_cast<uint4*>(hs + static_cast<size_t>(r) * a.K + channel) = h;
      if (channel == 0 && live) atomicOr(&s_live, 1u << r);
    });
  }
  __syncthreads();
  // the second dealing: quant_warps warps a row
  const int quant_warps = (a.K + 1023) / 1024, tpr = quant_warps * 32;
  const int rloc = static_cast<int>(threadIdx.x) / tpr, j = static_cast<int>(threadIdx.x) - rloc * tpr;
  const RowGroup row(s_red, quant_warps, rloc * quant_warps);
  const bool active = rloc < groups * a.group_rows && ((s_live >> (rloc & 31)) & 1u) && j * 32 < a.K;
  const P place(j);
  float2 v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = make_float2(0.0f, 0.0f);
  if (active) {
    const T* const src = hs + static_cast<size_t>(rloc) * a.K;
#pragma unroll
    for (int u = 0; u < P::kUnits; ++u) load_unit<P::kUnit>(src + place.channel(u), v + u * P::kPer);
  }
  __syncthreads();  // the rows have been read: their place now takes the rotation's lines
  rotate_quantize<kLayout, kFmt, false>(a, row, 0, j, m0 + rloc, active, smem_u32(row_smem) + static_cast<uint32_t>(rloc * tpr * 128), v);
}

// Norm alone: the CTAs that run at once go through the rows.
template <typename R, typename T, int N, bool kMods, bool kPost>
__global__ void __launch_bounds__(kNormThreads, 1) norm_kernel(const RowsArgs a) {
  __shared__ float s_red[8 * kMaxWarps];
  const int tpg = a.row_warps * 32;
  const int g = static_cast<int>(threadIdx.x) / tpg, j = static_cast<int>(threadIdx.x) - g * tpg;
  const int groups = static_cast<int>(blockDim.x) / tpg, step = static_cast<int>(gridDim.x) * groups;
  const RowGroup group(s_red, a.row_warps, g * a.row_warps);
  const int first = blockIdx.x * groups;  // every group of the CTA makes as many turns
  norm_rows<R, T, N, kMods, kPost>(a, group, j, first + g, step, first < a.M ? (a.M - first + step - 1) / step : 0, [](int, int, uint4, bool) {});
}

// ---- launches -----------------------------------------------------------------------------------------------------------------

template <typename K>
cudaError_t start(K kern, const RowsArgs& a, int grid, int threads, size_t smem) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(grid));
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
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

// Raises the kernel's limit of dynamic shared memory once per device; `done` holds the devices where it is.
template <typename K>
cudaError_t raise_limit(K kern, size_t smem, size_t most, std::atomic<unsigned long long>* done) {
  if (smem <= 40 * 1024) return cudaSuccess;  // (48 KB without it, the kernel's own few words included)
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (done->load() & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(most));
  if (e == cudaSuccess) done->fetch_or(bit);
  return e;
}

template <typename T, int kLayout, int kFmt>
cudaError_t launch_quantize(RowsArgs a) {
  a.row_warps = (a.K / 32 + 31) / 32;
  int rows = a.row_warps >= 8 ? 1 : 8 / a.row_warps;
  while (rows > 1 && (a.M + rows - 1) / rows < a.num_sms) rows /= 2;  // few rows: more CTAs
  a.group_rows = rows;
  const int threads = rows * a.row_warps * 32;
  auto kern = quantize_rows_kernel<T, kLayout, kFmt>;
  const size_t smem = kLayout != kPlain ? static_cast<size_t>(threads) * 128 : 0;
  static std::atomic<unsigned long long> raised{0};
  if (cudaError_t e = raise_limit(kern, smem, kRowThreads * 128, &raised)) return e;
  return start(kern, a, (a.M + rows - 1) / rows, threads, smem);
}

template <typename R, typename T, int N, bool kPlainNorm, int kLayout, int kFmt>
cudaError_t launch_norm_quantize(RowsArgs a) {
  a.row_warps = (a.K + N * 256 - 1) / (N * 256);
  const int quant_warps = (a.K + 1023) / 1024;
  // Rows of a CTA: as many as its warps quantise at once; fewer where that would leave SMs without any.
  int groups = a.row_warps >= 8 ? 1 : 8 / a.row_warps;
  a.group_rows = a.row_warps / quant_warps;
  while (groups > 1 && (a.M + groups * a.group_rows - 1) / (groups * a.group_rows) < a.num_sms) groups /= 2;
  while (a.group_rows > 1 && (a.M + groups * a.group_rows - 1) / (groups * a.group_rows) < 2 * a.num_sms) a.group_rows /= 2;
  const int threads = groups * a.row_warps * 32, rows = groups * a.group_rows;
  auto kern = norm_quantize_kernel<R, T, N, kPlainNorm, kLayout, kFmt>;
  const size_t lines = kLayout != kPlain ? static_cast<size_t>(threads) * 128 : 0, kept = static_cast<size_t>(rows) * a.K * sizeof(T);
  const size_t smem = std::max(lines, kept);
  static std::atomic<unsigned long long> raised{0};
  if (cudaError_t e = raise_limit(kern, smem, kNormThreads * 128, &raised)) return e;
  return start(kern, a, (a.M + rows - 1) / rows, threads, smem);
}

template <typename R, typename T, int N>
cudaError_t launch_norm_only(RowsArgs a) {
  a.row_warps = (a.K + N * 256 - 1) / (N * 256);
  int groups = a.row_warps >= 8 ? 1 : 8 / a.row_warps;
  while (groups > 1 && (a.M + groups - 1) / groups < a.num_sms) groups /= 2;
  const int threads = groups * a.row_warps * 32, blocks = (a.M + groups - 1) / groups;
  const int at_once = a.num_sms * (threads >= 1024 ? 1 : 1024 / threads);
  const int grid = blocks < at_once ? blocks : at_once;
  const bool mods = a.norm.gate != nullptr || a.norm.scale != nullptr || a.norm.shift != nullptr, post = a.norm.post_norm != 0;
  if (mods) return post ? start(norm_kernel<R, T, N, true, true>, a, grid, threads, 0) : start(norm_kernel<R, T, N, true, false>, a, grid, threads, 0);
  return post ? start(norm_kernel<R, T, N, false, true>, a, grid, threads, 0) : start(norm_kernel<R, T, N, false, false>, a, grid, threads, 0);
}

template <typename R, typename T, int N, bool kPlainNorm, int kFmt>
cudaError_t launch_norm_layout(const RowsArgs& a) {
  if (a.log_b <= 5) return launch_norm_quantize<R, T, N, kPlainNorm, kPlain, kFmt>(a);
  if (a.log_b <= 7) return launch_norm_quantize<R, T, N, kPlainNorm, kFour, kFmt>(a);
  switch (a.log_b) {
    case 8: return launch_norm_quantize<R, T, N, kPlainNorm, 8, kFmt>(a);
    case 9: return launch_norm_quantize<R, T, N, kPlainNorm, 9, kFmt>(a);
    case 10: return launch_norm_quantize<R, T, N, kPlainNorm, 10, kFmt>(a);
    case 11: return launch_norm_quantize<R, T, N, kPlainNorm, 11, kFmt>(a);
    default: return launch_norm_quantize<R, T, N, kPlainNorm, 12, kFmt>(a);
  }
}

template <typename R, typename T, int N, int kFmt>
cudaError_t launch_norm_kind(const RowsArgs& a) {
  const bool plain = a.norm.gate == nullptr && a.norm.scale == nullptr && a.norm.shift == nullptr && a.norm.post_norm == 0;
  return plain ? launch_norm_layout<R, T, N, true, kFmt>(a) : launch_norm_layout<R, T, N, false, kFmt>(a);
}

// R: the residual's type, T: everything else's.  Two pieces a thread where one would need more than 1024 threads, and with a
// 16-bit residual on many rows (6528 x 2048 14.8 us against 16.6 with one, conditioned 25.0 against 28.5; a float32 residual
// 29.3 against 25.1; 50 x 1024 1.9 against 1.7).
template <typename R, typename T>
cudaError_t launch_norm(const RowsArgs& a) {
  if (a.K > 8192 || (sizeof(R) == 2 && a.K >= 512 && a.M >= 2 * a.num_sms)) {
    if (a.codes == nullptr) return launch_norm_only<R, T, 2>(a);
    return a.fmt == kMx ? launch_norm_kind<R, T, 2, kMx>(a) : launch_norm_kind<R, T, 2, kNv>(a);
  }
  if (a.codes == nullptr) return launch_norm_only<R, T, 1>(a);
  return a.fmt == kMx ? launch_norm_kind<R, T, 1, kMx>(a) : launch_norm_kind<R, T, 1, kNv>(a);
}

template <typename T, int kFmt>
cudaError_t launch_quantize_layout(const RowsArgs& a) {
  if (a.log_b <= 5) return launch_quantize<T, kPlain, kFmt>(a);
  if (a.log_b <= 7) return launch_quantize<T, kFour, kFmt>(a);
  switch (a.log_b) {
    case 8: return launch_quantize<T, 8, kFmt>(a);
    case 9: return launch_quantize<T, 9, kFmt>(a);
    case 10: return launch_quantize<T, 10, kFmt>(a);
    case 11: return launch_quantize<T, 11, kFmt>(a);
    default: return launch_quantize<T, 12, kFmt>(a);
  }
}

template <typename T>
cudaError_t launch_quantize_fmt(const RowsArgs& a) {
  return a.fmt == kMx ? launch_quantize_layout<T, kMx>(a) : launch_quantize_layout<T, kNv>(a);
}

}  // namespace fp4
}  // namespace qvla
