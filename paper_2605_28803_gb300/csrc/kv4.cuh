// Device helpers of the attention operators: packed sequences, the 4-bit cache's pages, rotated heads.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

#include "kernels.h"
#include "ptx.cuh"

namespace qvla {

// An offset or length; kL2: past the first-level cache, where the kernel has not waited for the previous one yet.
template <bool kL2>
__device__ __forceinline__ int read_index(const int32_t* p) {
  if constexpr (kL2) return __ldcg(p);
  return __ldg(p);
}

// The sequence of packed row t: the last b with cu[b] <= t, found by the whole warp, 32 offsets a round.  False when t lies in
// no sequence.  Any contents of cu are safe: b stays in [0, batch).
template <bool kL2 = false>
__device__ __forceinline__ bool find_sequence(const int32_t* __restrict__ cu, int batch, int t, int& b, int& first) {
  const int lane = threadIdx.x & 31;
  int lo = 0, n = batch;
  while (n > 1) {
    const int step = (n + 31) >> 5;
    const bool at_or_before = lane * step < n && read_index<kL2>(cu + lo + lane * step) <= t;
    const int c = max(1, __popc(__ballot_sync(0xffffffffu, at_or_before)));
    lo += (c - 1) * step;
    n = min(step, n - (c - 1) * step);
  }
  b = lo;
  first = read_index<kL2>(cu + lo);
  return first <= t && t < read_index<kL2>(cu + lo + 1);
}

__device__ __forceinline__ void report_index() { atomicOr(&g_error_word, kErrIndex); }

// Reports offsets that begin below 0, decrease or pass `total`; one warp of every CTA, which take 32 offsets in turn.  (What the kernels
// make of them is safe without it: they are cut to [0, total], and a sequence whose offsets decrease has no tokens.)  Made ahead of
// the search for the sequence and finished after it, so that its loads run beside the search's.
struct OffsetsCheck {
  const int32_t* cu;
  int batch, total, at, next;
  int64_t i;
  __device__ __forceinline__ OffsetsCheck(const int32_t* cu_, int batch_, int total_) : cu(cu_), batch(batch_), total(total_) {
    i = static_cast<int64_t>(blockIdx.x) * 32 + (threadIdx.x & 31);
    load();
  }
  __device__ __forceinline__ void load() {
    at = i <= batch ? __ldg(cu + i) : 0;
    next = i < batch ? __ldg(cu + i + 1) : i == batch ? total : 0;
  }
  __device__ __forceinline__ void finish() {
    bool bad = at < 0 || next < at;
    while ((i += static_cast<int64_t>(gridDim.x) * 32) <= batch) {
      load();
      bad |= at < 0 || next < at;
    }
    if (bad) report_index();
  }
};

// Bytes of one head's tokens of a page, and the place of its parts.
__device__ __forceinline__ size_t kv4_block_bytes(const Kv4Pool& p) { return static_cast<size_t>(p.head_dim + 8) << p.log_page; }

// The block that holds position pos of sequence b for a head; null (and reported) when the table or the page is left.
__device__ __forceinline__ uint8_t* kv4_block(const Kv4Pool& p, const int32_t* __restrict__ table, int max_pages, int b, int64_t pos,
                                              int head) {
  if (pos < 0 || (pos >> p.log_page) >= max_pages) {
    report_index();
    return nullptr;
  }
  const int page = __ldg(table + static_cast<size_t>(b) * max_pages + (pos >> p.log_page));
  if (page < 0 || page >= p.num_pages) {
    report_index();
    return nullptr;
  }
  return p.base + (static_cast<size_t>(page) * p.kv_heads + head) * kv4_block_bytes(p);
}

// x . H / sqrt(D) for heads spread over teams of kTeam = D / 8 adjacent lanes, n heads a team at once.  Distances within a lane's
// 8 channels are butterflies in registers.  For the others two lanes first exchange a half of their registers, so that both ends of a
// distance lie in one lane (4 shuffles a level and head where exchanging all would take 8).  That turns the order of the channels:
// a lane has either channels 8 l to 8 l + 7 or channels 4 l to 4 l + 3 and those D / 2 further on (the halves' order).
template <int n>
__device__ __forceinline__ void butterflies(float (&y)[n][8], int h) {
#pragma unroll
  for (int j = 0; j < n; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if ((i & h) == 0) {
        const float a = y[j][i], b = y[j][i + h];
        y[j][i] = a + b;
        y[j][i + h] = a - b;
      }
}
template <int n>
__device__ __forceinline__ void swap_halves(float (&y)[n][8], int h) {
  const bool high = (threadIdx.x & h) != 0;
#pragma unroll
  for (int j = 0; j < n; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float got = __shfl_xor_sync(0xffffffffu, high ? y[j][i] : y[j][i + 4], h);
      y[j][i] = high ? got : y[j][i];
      y[j][i + 4] = high ? y[j][i + 4] : got;
    }
}
template <int kTeam, int n>
__device__ __forceinline__ void scale_rotated(float (&y)[n][8]) {
  constexpr float f = kTeam == 8 ? 0.125f : kTeam == 16 ? 0.08838834764831845f : 0.0625f;  // float32(1 / sqrt(8 kTeam))
#pragma unroll
  for (int j = 0; j < n; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) y[j][i] *= f;
}
// from the halves' order
template <int kTeam, int n>
__device__ __forceinline__ void rotate_from_halves(float (&y)[n][8]) {
  butterflies(y, 1);
  butterflies(y, 2);
  butterflies(y, 4);
#pragma unroll
  for (int h = kTeam / 2; h > 0; h /= 2) {
    swap_halves(y, h);
    butterflies(y, 4);
  }
  scale_rotated<kTeam>(y);
}
// to the halves' order
template <int kTeam, int n>
__device__ __forceinline__ void rotate_to_halves(float (&y)[n][8]) {
  butterflies(y, 1);
  butterflies(y, 2);
  butterflies(y, 4);
#pragma unroll
  for (int h = 1; h < kTeam; h *= 2) {
    swap_halves(y, h);
    butterflies(y, 4);
  }
  scale_rotated<kTeam>(y);
}

// (w & mask) ^ flip in one instruction.  Only one of its operands can be an immediate: `flip` comes from a register that the
// compiler cannot see through (hidden_constant), or it would take two instructions with an immediate each.
__device__ __forceinline__ uint32_t and_xor(uint32_t w, uint32_t mask, uint32_t flip) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(r) : "r"(w), "r"(mask), "r"(flip));
  return r;
}
template <uint32_t kValue>
__device__ __forceinline__ uint32_t hidden_constant() {
  uint32_t r;
  asm volatile("mov.u32 %0, %1;" : "=r"(r) : "n"(kValue));
  return r;
}

// Of a word of 8 codes: the codes at nibbles 0 and 4, and at 1 and 5, as float16 pairs.  The bits 0x6408 ^ code read 1032 + code
// and 0x5480 ^ (code << 4) read 72 + code, from which one exact addition takes the offset.
struct CodeBits {
  uint32_t low = hidden_constant<0x64086408u>(), high = hidden_constant<0x54805480u>();
  __device__ __forceinline__ uint32_t codes_04(uint32_t w) const {
    w = and_xor(w, 0x000f000fu, low);
    const __half2 v = __hadd2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0xe408)));  // -1032
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  __device__ __forceinline__ uint32_t codes_15(uint32_t w) const {
    w = and_xor(w, 0x00f000f0u, high);
    const __half2 v = __hadd2(*reinterpret_cast<const __half2*>(&w), __half2half2(__ushort_as_half(0xd480)));  // -72
    return *reinterpret_cast<const uint32_t*>(&v);
  }
};

// Two float32 operations an instruction, each rounded like the single one.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t&>(r))
      : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)), "l"(reinterpret_cast<const uint64_t&>(c)));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t&>(r)) : "l"(reinterpret_cast<const uint64_t&>(a)), "l"(reinterpret_cast<const uint64_t&>(b)));
  return r;
}

template <typename T>
struct Pair;
template <>
struct Pair<__half> {
  using V = __half2;
  static __device__ __forceinline__ float2 to_float(V v) { return __half22float2(v); }
  static __device__ __forceinline__ V from_float(float a, float b) { return __floats2half2_rn(a, b); }
};
template <>
struct Pair<__nv_bfloat16> {
  using V = __nv_bfloat162;
  static __device__ __forceinline__ float2 to_float(V v) { return __bfloat1622float2(v); }
  static __device__ __forceinline__ V from_float(float a, float b) { return __floats2bfloat162_rn(a, b); }
};

// 8 consecutive 16-bit values at a 16-byte aligned address.
template <typename T>
__device__ __forceinline__ void unpack8(const uint4& v, float (&y)[8]) {
  const typename Pair<T>::V* h = reinterpret_cast<const typename Pair<T>::V*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = Pair<T>::to_float(h[i]);
    y[2 * i] = f.x;
    y[2 * i + 1] = f.y;
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&y)[8]) {
  uint4 v;
  typename Pair<T>::V* h = reinterpret_cast<typename Pair<T>::V*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = Pair<T>::from_float(y[2 * i], y[2 * i + 1]);
  return v;
}
// A lane's 8 channels of a head, in the halves' order where they have been rotated.
template <int kTeam, typename T>
__device__ __forceinline__ void store_head(T* head, const float (&y)[8], bool halves) {
  const uint4 v = pack8<T>(y);
  const int tl = threadIdx.x % kTeam;
  if (halves) {
    *reinterpret_cast<uint2*>(head + tl * 4) = make_uint2(v.x, v.y);
    *reinterpret_cast<uint2*>(head + kTeam * 4 + tl * 4) = make_uint2(v.z, v.w);
  } else {
    *reinterpret_cast<uint4*>(head + tl * 8) = v;
  }
}

}  // namespace qvla
