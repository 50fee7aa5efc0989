// Microscaled 4-bit floating point: E2M1 codes with E8M0 scales of 32 channels (MX) or E4M3 scales of 16 and a float32 scale
// a row (NV).  The formats and the rounding decisions that the row kernels and the products share.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace qvla {
namespace fp4 {

constexpr int kMx = 0, kNv = 1;  // qvla_fp4_format

constexpr float kMaxCode = 6.0f;            // E2M1
constexpr float kRowMax = 6.0f * 448.0f;    // E2M1 times E4M3: a row's largest entry stands there

// Scales lie in tiles of 128 rows x 4 blocks, 512 bytes: the order in which tcgen05 takes them (row % 32 is the lane, row / 32
// the column, a column's four bytes the blocks).  `groups` is the number of tiles side by side (blocks of a row / 4).
__host__ __device__ __forceinline__ size_t scale_offset(int row, int block, int groups) {
  return (static_cast<size_t>(row >> 7) * groups + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// Eight values as E2M1 codes, the first in the lowest nibble: to nearest, ties to even, +-6 beyond.
__device__ __forceinline__ uint32_t e2m1x8(float2 a, float2 b, float2 c, float2 d) {
  uint32_t r;
  asm("{\n.reg .b8 p, q, r, s;\n"
      "cvt.rn.satfinite.e2m1x2.f32 p, %2, %1;\n"  // the second operand is the low nibble
      "cvt.rn.satfinite.e2m1x2.f32 q, %4, %3;\n"
      "cvt.rn.satfinite.e2m1x2.f32 r, %6, %5;\n"
      "cvt.rn.satfinite.e2m1x2.f32 s, %8, %7;\n"
      "mov.b32 %0, {p, q, r, s};\n}\n"
      : "=r"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y), "f"(d.x), "f"(d.y));
  return r;
}

// Two values as E4M3 bytes (to nearest, ties to even, 448 beyond, NaN 0x7F), the first in the low byte.
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(b), "f"(a));
  return r;
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// The value of a non-negative E4M3 byte: 1.mmm 2^(e - 7), or 0.mmm 2^-6 with e = 0.
__device__ __forceinline__ float e4m3_value(uint32_t c) {
  if (c == 0x7Fu) return __int_as_float(0x7FC00000);
  // the byte's fields as a float's, whose exponent is then 120 too small; the product also makes its subnormals right
  return __uint_as_float(c << 20) * __uint_as_float((127u + 120u) << 23);
}

// 2^(byte - 127); byte 255 is NaN.
__device__ __forceinline__ float e8m0_value(uint32_t b) {
  return b == 255u ? __int_as_float(0x7FC00000) : b == 0u ? __uint_as_float(1u << 22) : __uint_as_float(b << 23);
}

// The product of code and a power-of-two shift of 1/2: codes 0 .. 7 are 0, .5, 1, 1.5, 2, 3, 4, 6.
__device__ __forceinline__ float e2m1_value(uint32_t c) {
  const uint32_t m = c & 7u;  // exponent and mantissa bit of a float whose exponent is 126 too small
  const float v = __uint_as_float(m << 22) * __uint_as_float((127u + 126u) << 23);
  return (c & 8u) ? -v : v;
}

// Two float32 numbers scaled by one power of two into the range where quotients and products of them lose nothing.
__device__ __forceinline__ void bring_near(float& a, float& d) {
  const float up = 1.2089258196146292e24f, down = 8.271806125530277e-25f;  // 2^80, 2^-80
  if (d < 8.673617379884035e-19f) {  // 2^-60
    a *= up;
    d *= up;
  } else if (d > 1.152921504606846976e18f) {
    a *= down;
    d *= down;
  }
}

// 1 / x within 2^-23 of it, x and the quotient normal numbers.
__device__ __forceinline__ float near_reciprocal(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// The E4M3 byte nearest the exact quotient a / (6 delta), ties to the even byte; 448 at most.  a >= 0, delta > 0 finite.
// The float32 quotient is within 2^-21 of the exact one: where its neighbours 2^-20 away round alike it decides; else the
// midpoint between both bytes does, by the sign of a - midpoint * 6 delta (exact in one FMA: a midpoint has 5 bits, 6 of
// them with the factor 3, and float32 holds the factor).
__device__ __forceinline__ uint32_t block_scale_e4m3(float a, float delta) {
  bring_near(a, delta);
  const float t = a * near_reciprocal(6.0f * delta);
  const uint32_t both = e4m3x2(t * 0.99999904632568359375f, t * 1.00000095367431640625f);
  const uint32_t lo = both & 0xFFu, hi = both >> 8;
  if (lo == hi) return lo;
  const float mid6 = 3.0f * (e4m3_value(lo) + e4m3_value(hi));
  const float d = fmaf(-mid6, delta, a);
  if (d == 0.0f) return (lo & 1u) ? hi : lo;
  return d > 0.0f ? hi : lo;
}

// Where two candidate words of codes (each value's quotient moved down and up a little) differ, the codes nearest the exact
// quotients z / d, ties to the even code; d > 0 finite.  The two candidates of a value are neighbours, and the sign of
// |z| - midpoint * d, exact in one FMA, decides between them.  A few values of a thread at most come here, but among bfloat16
// rows without a rotation about one in 200 does: a channel at a power of two of the row's largest stands one rounding of
// Delta from a tie.
static __device__ __noinline__ uint32_t decide_codes(uint32_t down, uint32_t up, float2 a, float2 b, float2 c, float2 e, float d) {
  uint32_t diff = down ^ up;
  diff |= diff >> 2;
  diff |= diff >> 1;
  diff &= 0x11111111u;  // one bit a code
  while (diff != 0u) {
    const int at = __ffs(static_cast<int>(diff)) - 1, i = at >> 2;
    diff &= diff - 1;
    const float2 p = (i & 4) ? ((i & 2) ? e : c) : ((i & 2) ? b : a);
    float z = fabsf((i & 1) ? p.y : p.x), unit = d;
    bring_near(z, unit);
    const uint32_t lo = (down >> at) & 7u;
    // the number halfway to the next code has one bit more: as a float its fields are 126 exponents low
    const float mid = __uint_as_float((2u * lo + 1u) << 21) * __uint_as_float((127u + 126u) << 23);
    const float r = fmaf(-mid, unit, z);
    const uint32_t take = r > 0.0f || (r == 0.0f && (lo & 1u)) ? lo + 1u : lo;
    up = (up & ~(7u << at)) | (take << at);
  }
  return up;
}

// All eight by comparison with every midpoint: for units so large or small that an approximate quotient says nothing.
static __device__ __noinline__ uint32_t codes_exact(float2 a, float2 b, float2 c, float2 e, float d) {
  const float z[8] = {a.x, a.y, b.x, b.y, c.x, c.y, e.x, e.y};
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float v = fabsf(z[i]), unit = d;
    bring_near(v, unit);
    uint32_t k = 0;
    const float mid[7] = {0.25f, 0.75f, 1.25f, 1.75f, 2.5f, 3.5f, 5.0f};
#pragma unroll
    for (int m = 0; m < 7; ++m) {
      const float r = fmaf(-mid[m], unit, v);
      k += (r > 0.0f || (r == 0.0f && (m & 1))) ? 1u : 0u;  // a tie goes up where the upper code is even
    }
    w |= (k | ((__float_as_uint(z[i]) >> 28) & 8u)) << (4 * i);
  }
  return w;
}

}  // namespace fp4
}  // namespace qvla
