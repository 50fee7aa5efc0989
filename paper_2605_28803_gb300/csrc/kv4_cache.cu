// The 4-bit key/value cache: tokens in (rotate, quantise, store to their pages) and tokens out.
//
// Per token and key/value head: y = x . H / sqrt(D) (or x), Delta = max |y| / 7, codes clamp(round(y / Delta), -7, 7), round half
// to even on the exact quotient; out again, x^ = (Delta / sqrt(D)) (q . H), rounded to the output's type.  q . H is a vector of
// integers of at most 7 D = 1792: exact in float16, so on the way out the rotation is float16 arithmetic, two channels an
// instruction and a shuffle, without a rounding.
//
// Both move 2 D bytes of values one way and D / 2 + 4 of codes the other way per head, and HBM would be the bound; the rotation's
// log2 D sums a channel and its exchanges between lanes come close to it.  So a head is a team of only D / 32 lanes with four
// groups of 8 channels each, group k of lane l at channel 8 (k team + l): of the butterflies' distances 1, 2, 4 and the two
// largest stay in registers, two channels an instruction, and 1 to 3 are shuffles; a team's 16-byte accesses are contiguous.
// A warp takes `sets` sets of 32 / team heads in a row, keys and then values of each (which lie in the same block of the cache), and
// loads the next pass's data ahead of the present one's arithmetic; the search for the first token's sequence is made once.
//
// Measured, 8 heads of 128 channels: 7194 tokens in and out 24.8 us (on the way in the latency of a head's shuffles, maximum and rounding,
// with the 20 warps an SM that registers allow: issue 52%, DRAM 18%); 49611 tokens out 48.9 us, 203 MB written at 4.2 TB/s (a plain fill writes at 3.9).  Keys and
// values of a head by the same warp, which finds their block once, took 49611 tokens from 50.5 to 48.6 and 3000 tokens of 8 heads of
// 256 from 9.9 to 7.8 us.
#include <cuda_runtime.h>

#include "griddep.cuh"
#include "kv4.cuh"

namespace qvla {
namespace {

constexpr int kThreads = 128;
constexpr int kSets = 4;          // of a warp, at most
constexpr int kWarpsPerSm = 48;   // below this many warps an SM, a warp takes fewer sets (of 7194 tokens in and out: 40 warps 27.3 us, 48 24.6, 64 24.6)

template <int kTeam>
constexpr float kNorm = kTeam == 2 ? 0.125f : kTeam == 4 ? 0.08838834764831845f : 0.0625f;  // float32(1 / sqrt(32 kTeam))

// q . H for codes (or sums of them) spread over kTeam lanes as above: v[k] holds channels 0 and 4, 1 and 5, 2 and 6, 3 and 7 of
// group k's eight.  Every sum is exact.
template <int kTeam>
__device__ __forceinline__ void rotate_codes(__half2 (&v)[4][4]) {
  const int lane = threadIdx.x & 31;
  const __half2 split = __halves2half2(__ushort_as_half(0x3c00), __ushort_as_half(0xbc00));  // 1, -1
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int h = 1; h < 4; h *= 2)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((i & h) == 0) {
          const __half2 a = v[k][i], b = v[k][i + h];
          v[k][i] = __hadd2(a, b);
          v[k][i + h] = __hsub2(a, b);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[k][i] = __hfma2(v[k][i], split, __lowhigh2highlow(v[k][i]));
  }
#pragma unroll
  for (int h = 1; h < kTeam; h *= 2) {
    const __half2 sign = __half2half2(__ushort_as_half((lane & h) != 0 ? 0xbc00 : 0x3c00));
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) v[k][i] = __hfma2(v[k][i], sign, __shfl_xor_sync(0xffffffffu, v[k][i], h));
  }
#pragma unroll
  for (int h = 1; h < 4; h *= 2)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((k & h) == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const __half2 a = v[k][i], b = v[k + h][i];
          v[k][i] = __hadd2(a, b);
          v[k + h][i] = __hsub2(a, b);
        }
}

// x . H / sqrt(32 kTeam) for a head spread over kTeam lanes as above; distances 1, 2, 4, ... in this order (another one rounds differently).
template <int kTeam>
__device__ __forceinline__ void rotate_groups(float2 (&y)[4][4]) {
  const float2 minus = make_float2(-1.0f, -1.0f);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[k][i] = make_float2(y[k][i].x + y[k][i].y, y[k][i].x - y[k][i].y);
#pragma unroll
    for (int h = 1; h < 4; h *= 2)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if ((i & h) == 0) {
          const float2 a = y[k][i], b = y[k][i + h];
          y[k][i] = add2(a, b);
          y[k][i + h] = fma2(b, minus, a);
        }
  }
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int h = 1; h < kTeam; h *= 2) {
    const float sign = (lane & h) != 0 ? -1.0f : 1.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 o = make_float2(__shfl_xor_sync(0xffffffffu, y[k][i].x, h), __shfl_xor_sync(0xffffffffu, y[k][i].y, h));
        y[k][i] = fma2(y[k][i], make_float2(sign, sign), o);  // a + b, or a - b in the upper lane
      }
  }
  constexpr float f = kNorm<kTeam>;
#pragma unroll
  for (int h = 1; h < 4; h *= 2)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((k & h) == 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 a = y[k][i], b = y[k + h][i];
          y[k][i] = add2(a, b);
          y[k + h][i] = fma2(b, minus, a);
        }
#pragma unroll
  for (int k = 0; k < 4; ++k)
#pragma unroll
    for (int i = 0; i < 4; ++i) y[k][i] = mul2(y[k][i], make_float2(f, f));
}

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

// kApart: a warp takes the keys or the values of one set, for calls of few tokens; else `sets` sets, keys and values.
template <typename T, int kTeam, bool kAppend, bool kApart>
__global__ void __launch_bounds__(kThreads) kv4_rows_kernel(const __grid_constant__ Kv4RowsArgs a, int sets) {
  constexpr int kDim = 32 * kTeam, kHeads = 32 / kTeam;  // heads of a warp's pass
  const int lane = threadIdx.x & 31, team = lane / kTeam, tl = lane % kTeam;
  const int heads = a.pool.kv_heads;
  const int64_t all = static_cast<int64_t>(a.total) * heads;
  const int64_t warp = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) >> 5;
  const int side = kApart ? static_cast<int>(warp & 1) : 0;
  const int64_t id0 = (kApart ? warp >> 1 : warp * sets) * kHeads;
  griddep_wait();  // tokens, cache, tables and offsets may come from the previous kernel, which may still read the outputs
  griddep_launch_dependents();
  if (id0 >= all) return;  // (not a CTA's first warp)
  OffsetsCheck offsets(a.cu, a.batch, a.total);
  // this team's token and head, and what they move on by from set to set (no division by `heads` there)
  const int64_t id = id0 + team;
  int t = static_cast<int>(all >> 31 ? id / heads : static_cast<uint32_t>(id) / static_cast<uint32_t>(heads));
  int head = static_cast<int>(id - static_cast<int64_t>(t) * heads), b, first, next;
  find_sequence(a.cu, a.batch, __shfl_sync(0xffffffffu, t, 0), b, first);
  next = __ldg(a.cu + b + 1);
  if (threadIdx.x < 32) offsets.finish();
  const int t_on = kHeads / heads, head_on = kHeads % heads;
  const int plane = (kDim / 2) << a.pool.log_page;  // bytes of a block's key codes

  // a team's head in the cache: its key's codes and scale at the token (null: none), the value's a plane further on
  bool here = false;
  uint8_t* codes = nullptr;
  float* scale = nullptr;
  auto find = [&]() {
    here = false;
    codes = nullptr;
    if (t >= a.total) return;
    while (t >= next && b + 1 < a.batch) {  // (tokens come in order)
      first = next;
      ++b;
      next = __ldg(a.cu + b + 1);
    }
    if (t < first || t >= next) return;
    here = true;
    const int64_t pos = static_cast<int64_t>(a.start ? __ldg(a.start + b) : 0) + (t - max(first, 0));
    uint8_t* const at = kv4_block(a.pool, a.table, a.max_pages, b, pos, head);
    if (at == nullptr) return;
    const int slot = static_cast<int>(pos) & ((1 << a.pool.log_page) - 1);
    codes = at + slot * (kDim / 2) + tl * 4;
    scale = reinterpret_cast<float*>(at + 2 * plane) + slot;
  };
  struct Head {
    uint8_t* at;    // its codes in the cache; null: none
    float* scale;
    T* out;         // gather's output, append's input; null: nothing to do
    uint4 x[4];     // append: the token's values; gather: the codes of group k in x[0].xyzw
    float d;
  };
  auto load = [&](Head& h, int value) {
    h.out = nullptr;
    h.at = nullptr;
    h.d = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) h.x[k] = make_uint4(0, 0, 0, 0);
    if (!here) return;
    h.out = static_cast<T*>(value ? a.v : a.k) + t * (value ? a.v_stride : a.k_stride) + head * kDim + tl * 8;
    if (codes == nullptr) return;
    h.at = codes + (value ? plane : 0);
    h.scale = scale + (value << a.pool.log_page);
    if constexpr (kAppend) {
#pragma unroll
      for (int k = 0; k < 4; ++k) h.x[k] = __ldg(reinterpret_cast<const uint4*>(h.out + k * 8 * kTeam));
    } else {
      h.x[0].x = __ldg(reinterpret_cast<const unsigned int*>(h.at));
      h.x[0].y = __ldg(reinterpret_cast<const unsigned int*>(h.at + 4 * kTeam));
      h.x[0].z = __ldg(reinterpret_cast<const unsigned int*>(h.at + 8 * kTeam));
      h.x[0].w = __ldg(reinterpret_cast<const unsigned int*>(h.at + 12 * kTeam));
      h.d = __ldg(h.scale);
    }
  };
  auto finish = [&](const Head& h) {
    float2 y[4][4];
    if constexpr (kAppend) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const typename Pair<T>::V* v = reinterpret_cast<const typename Pair<T>::V*>(&h.x[k]);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[k][i] = Pair<T>::to_float(v[i]);
      }
      if (a.pool.rotate) rotate_groups<kTeam>(y);
      uint32_t m = 0;  // the largest magnitude by its bits: a NaN stands above every number
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          m = max(m, max(__float_as_uint(y[k][i].x) & 0x7fffffffu, __float_as_uint(y[k][i].y) & 0x7fffffffu));
#pragma unroll
      for (int s = 1; s < kTeam; s *= 2) m = max(m, __shfl_xor_sync(0xffffffffu, m, s));
      if (h.at == nullptr) return;
      const float d = m < 0x7f800000u ? __fdiv_rn(__uint_as_float(m), 7.0f) : __uint_as_float(0x7fffffffu);
      // y / d is at most 7 (1 + 2^-24) by the choice of d, so codes need no clamp.  1.5 2^23 + y r rounds to half even in the last place, whose
      // byte is the code; where that lies within 1e-5 of a tie (or r is no number to use) the exact decision is taken.
      const float r = __frcp_rn(d);
      const float2 r2 = make_float2(r, r), big = make_float2(12582912.0f, 12582912.0f), neg = make_float2(-12582912.0f, -12582912.0f);
      float far = 0.0f;  // from the code, at most
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        uint32_t e[4], o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 n = fma2(y[k][i], r2, big), c = add2(n, neg), rest = fma2(y[k][i], r2, make_float2(-c.x, -c.y));
          far = fmaxf(far, fmaxf(fabsf(rest.x), fabsf(rest.y)));
          e[i] = __float_as_uint(n.x);
          o[i] = __float_as_uint(n.y);
        }
        const uint32_t even = __byte_perm(__byte_perm(e[0], e[1], 0x0040), __byte_perm(e[2], e[3], 0x0040), 0x5410);
        const uint32_t odd = __byte_perm(__byte_perm(o[0], o[1], 0x0040), __byte_perm(o[2], o[3], 0x0040), 0x5410);
        w[k] = (even & 0x0f0f0f0fu) | ((odd << 4) & 0xf0f0f0f0u);
      }
      const bool tiny = d < 1e-28f;  // the remainder of a quotient could leave the numbers: decide on scaled values
      if (!(far < 0.49999f) || tiny || !(d > 0.0f)) {
        const float up = tiny ? 0x1p64f : 1.0f, ds = d * up, rs = __frcp_rn(ds);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          w[k] = 0;
          if (d > 0.0f) {  // (not zero, not NaN)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              w[k] |= (static_cast<uint32_t>(code_of(y[k][i].x * up, ds, rs)) & 15u) << (8 * i);
              w[k] |= (static_cast<uint32_t>(code_of(y[k][i].y * up, ds, rs)) & 15u) << (8 * i + 4);
            }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) *reinterpret_cast<uint32_t*>(h.at + k * 4 * kTeam) = w[k];
      if (tl == 0) *h.scale = d;
    } else {
      const CodeBits bits;
      __half2 v[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t w = k == 0 ? h.x[0].x : k == 1 ? h.x[0].y : k == 2 ? h.x[0].z : h.x[0].w;
        *reinterpret_cast<uint32_t*>(&v[k][0]) = bits.codes_04(w);
        *reinterpret_cast<uint32_t*>(&v[k][1]) = bits.codes_15(w);
        *reinterpret_cast<uint32_t*>(&v[k][2]) = bits.codes_04(w >> 8);
        *reinterpret_cast<uint32_t*>(&v[k][3]) = bits.codes_15(w >> 8);
      }
      if (a.pool.rotate) rotate_codes<kTeam>(v);
      if (h.out == nullptr) return;
      const float f = a.pool.rotate ? h.d * kNorm<kTeam> : h.d;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 c = mul2(__half22float2(v[k][i]), make_float2(f, f));
          y[i] = c.x;
          y[i + 4] = c.y;
        }
        *reinterpret_cast<uint4*>(h.out + k * 8 * kTeam) = pack8<T>(y);
      }
    }
  };
  Head now;
  find();
  load(now, side);
  if constexpr (kApart) {
    finish(now);
  } else {
    for (int i = 0; i < 2 * sets; ++i) {  // a set's keys, then its values
      if (id0 + static_cast<int64_t>(i / 2) * kHeads >= all) break;  // (the whole warp)
      Head ahead;
      if ((i & 1) && i + 1 < 2 * sets) {
        t += t_on;
        head += head_on;
        if (head >= heads) {
          head -= heads;
          ++t;
        }
        find();
      }
      if (i + 1 < 2 * sets) load(ahead, (i + 1) & 1);
      finish(now);
      now = ahead;
    }
  }
}

template <typename T, int kTeam, bool kAppend>
cudaError_t launch_rows(const Kv4RowsArgs& a) {
  const int64_t all = (static_cast<int64_t>(a.total) * a.pool.kv_heads + 32 / kTeam - 1) / (32 / kTeam);
  const int64_t fill = static_cast<int64_t>(a.num_sms) * kWarpsPerSm;
  const int sets = static_cast<int>(all >= fill * kSets ? kSets : all <= fill ? 1 : (all + fill - 1) / fill);
  const bool apart = 2 * all <= fill;
  const int64_t warps = apart ? 2 * all : (all + sets - 1) / sets;
  const int64_t blocks = (warps * 32 + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(blocks));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, apart ? kv4_rows_kernel<T, kTeam, kAppend, true> : kv4_rows_kernel<T, kTeam, kAppend, false>, a, sets);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

template <bool kAppend>
cudaError_t launch_rows(const Kv4RowsArgs& a) {
  const int d = a.pool.head_dim;
  if (a.dt == 0) {
    return d == 64 ? launch_rows<__half, 2, kAppend>(a) : d == 128 ? launch_rows<__half, 4, kAppend>(a) : launch_rows<__half, 8, kAppend>(a);
  }
  return d == 64 ? launch_rows<__nv_bfloat16, 2, kAppend>(a)
                 : d == 128 ? launch_rows<__nv_bfloat16, 4, kAppend>(a) : launch_rows<__nv_bfloat16, 8, kAppend>(a);
}

}  // namespace

cudaError_t launch_kv4_append(const Kv4RowsArgs& a) { return launch_rows<true>(a); }
cudaError_t launch_kv4_gather(const Kv4RowsArgs& a) { return launch_rows<false>(a); }

cudaError_t read_and_clear_error_word_kv4(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess || *out == 0) return e;  // (cleared only where it is set: the check goes through every unit's word)
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

}  // namespace qvla
