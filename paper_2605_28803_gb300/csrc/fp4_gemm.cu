// Product of two matrices in 4-bit floating point with block scales, on tcgen05.mma with block scaling.
//
//   acc[m, n] = sum_k (c s)_x[m, k] (c s)_w[n, k]     codes and block scales multiplied by the tensor cores, float32 sums
//   y = fma(acc, xscale[m] wscale[n], bias[n]), or for a gated layer gelu_tanh(gate) up, rounded once
//
// A tile is 128 tokens x 128 weight rows; its k-blocks of 256 codes (128 bytes a row under the 128-byte swizzle) come by TMA
// through a ring, the scales beside them as whole tiles (fp4.cuh), which tcgen05.cp spreads over TMEM ahead of the products.
#include "fp4.cuh"
#include "gemm_kernel.cuh"

namespace qvla {
namespace {

constexpr int kF4Bm = 128, kF4Bn = 128;
constexpr int kF4Row = 128;                      // bytes of a row of a k-block: 256 codes
constexpr int kF4TileA = kF4Bm * kF4Row, kF4TileB = kF4Bn * kF4Row;
constexpr int kF4ScaleMax = 2048;                // bytes of scales of 128 rows and a k-block (NV; MX has half)
constexpr int kF4Stage = kF4TileA + kF4TileB + 2 * kF4ScaleMax;
constexpr int kF4Stages = 5;
constexpr int kF4Smem = kF4Stages * kF4Stage + 1024;
constexpr int kF4Threads = 6 * 32;               // 4 epilogue warps, MMA, TMA

struct F4Params {
  const uint8_t *xs, *ws;
  const float *xrow, *wrow, *bias;
  void* y;
  int M, N, K;
};

// Descriptor of scales for tcgen05.cp: 32 rows of 16 bytes, 8-row groups 128 bytes apart, no swizzle.
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128 >> 4) << 32) | (static_cast<uint64_t>(1) << 46);
}
// 128 rows' scales of four blocks (512 bytes) to four TMEM columns, for each of the four lane quadrants.
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}

// Instruction descriptor: A = B = E2M1, both K-major, shape M x N, K = 64; scales E8M0 (MX) or E4M3.
__host__ __device__ constexpr uint32_t idesc_e2m1_f32(int fmt, int m, int n) {
  return (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (fmt == fp4::kMx ? 1u << 23 : 0u) |
         (static_cast<uint32_t>(m >> 7) << 27);
}

// 64 codes of K.  MX: two scales a row, bytes `id` and id + 1 (id = 0 or 2) of the column; NV: all four.
template <int kFmt>
__device__ __forceinline__ void mma_e2m1(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa, uint32_t sb,
                                         uint32_t accumulate) {
  if constexpr (kFmt == fp4::kMx) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  } else {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  }
}

template <int kFmt, bool kGated, typename OutT>
__global__ void __launch_bounds__(kF4Threads, 1) fp4_gemm_kernel(const __grid_constant__ CUtensorMap tmap_x,
                                                                 const __grid_constant__ CUtensorMap tmap_w, F4Params p) {
  extern __shared__ uint8_t dyn_smem[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bar_full[kF4Stages], bar_empty[kF4Stages], bar_done;
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  __shared__ __align__(16) float s_ws[kF4Bn], s_b[kF4Bn];

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int m0 = blockIdx.x * kF4Bm, n0 = blockIdx.y * kF4Bn;
  const int nkb = (p.K + 255) / 256;
  constexpr int kTileCodes = kFmt == fp4::kMx ? 128 : 64;  // codes that a scale tile covers
  constexpr int kTiles = 256 / kTileCodes;                 // scale tiles of a k-block
  const int groups = p.K / kTileCodes;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kF4Stages; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    mbar_init(smem_u32(&bar_done), 1);
    mbar_init_fence();
    s_abort = 0;
  }
  if (warp == 4) tmem_alloc<256>(smem_u32(&s_tmem_base));
  if (threadIdx.x < kF4Bn) {
    const int n = n0 + static_cast<int>(threadIdx.x);
    s_ws[threadIdx.x] = n < p.N ? p.wrow[n] : 0.0f;
    s_b[threadIdx.x] = n < p.N ? p.bias[n] : 0.0f;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem_base, t_sa = tmem + 128, t_sb = tmem + 160;
  griddep_wait();
  griddep_launch_dependents();

  if (warp == 5) {
    bool ok = *const_cast<volatile int*>(&g_debug_hold_loads) == 0;
    int it = 0;
    for (; it < nkb && ok; ++it) {
      const int s = it % kF4Stages;
      const uint32_t ph = static_cast<uint32_t>(it / kF4Stages) & 1u;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_empty[s]), ph ^ 1u))) { ok = false; break; }
      if (elect_one()) {
        const uint32_t bar = smem_u32(&bar_full[s]), dst = smem_u32(smem + s * kF4Stage);
        const int tiles = min(kTiles, groups - it * kTiles);
        mbar_arrive_expect_tx(bar, static_cast<uint32_t>(kF4TileA + kF4TileB + 2 * tiles * 512));
        tma_load_2d(dst, &tmap_x, it * kF4Row, m0, bar);
        tma_load_2d(dst + kF4TileA, &tmap_w, it * kF4Row, n0, bar);
        bulk_load(dst + kF4TileA + kF4TileB, p.xs + (static_cast<size_t>(blockIdx.x) * groups + it * kTiles) * 512, tiles * 512, bar);
        bulk_load(dst + kF4TileA + kF4TileB + kF4ScaleMax, p.ws + (static_cast<size_t>(blockIdx.y) * groups + it * kTiles) * 512, tiles * 512, bar);
      }
      __syncwarp();
    }
    for (int i = max(0, it - kF4Stages); i < it; ++i) mbar_wait(smem_u32(&bar_full[i % kF4Stages]), static_cast<uint32_t>(i / kF4Stages) & 1u);
  } else if (warp == 4) {
    constexpr uint32_t idesc = idesc_e2m1_f32(kFmt, kF4Bm, kF4Bn);
    bool ok = true;
    for (int it = 0; it < nkb; ++it) {
      const int s = it % kF4Stages;
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_full[s]), static_cast<uint32_t>(it / kF4Stages) & 1u))) { ok = false; break; }
      tc_fence_after();
      if (elect_one()) {
        const uint32_t base = smem_u32(smem + s * kF4Stage);
        const int tiles = min(kTiles, groups - it * kTiles);
        for (int t = 0; t < tiles; ++t) {
          copy_scales(t_sa + 4 * t, scale_desc(base + kF4TileA + kF4TileB + t * 512));
          copy_scales(t_sb + 4 * t, scale_desc(base + kF4TileA + kF4TileB + kF4ScaleMax + t * 512));
        }
        const uint64_t da = smem_desc_sw128(base), db = smem_desc_sw128(base + kF4TileA);
        const int steps = tiles * (kTileCodes / 64);
        for (int k = 0; k < steps; ++k) {
          const uint32_t col = kFmt == fp4::kMx ? 4 * (k >> 1) : 4 * k;
          const uint32_t id = kFmt == fp4::kMx ? 2u * (k & 1) : 0u;
          mma_e2m1<kFmt>(tmem, da + 2 * k, db + 2 * k, idesc | (id << 4) | (id << 29), t_sa + col, t_sb + col, (it | k) != 0 ? 1u : 0u);
        }
        mma_commit(smem_u32(&bar_empty[s]));
      }
      __syncwarp();
    }
    if (elect_one()) {
      if (!ok) *const_cast<volatile int*>(&s_abort) = 1;
      __threadfence_block();
      mma_commit(smem_u32(&bar_done));  // also after a wait ran out: what was issued is waited for
    }
    __syncwarp();
  } else {
    const bool done = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_done), 0) && *const_cast<volatile int*>(&s_abort) == 0);
    __syncwarp();
    tc_fence_after();
    const int m = m0 + warp * 32 + lane;
    const int ldy = kGated ? p.N / 2 : p.N;
    const float xs = m < p.M && p.xrow != nullptr ? p.xrow[m] : 1.0f;
    OutT* const yrow = static_cast<OutT*>(p.y) + static_cast<size_t>(m) * ldy;
    const uint32_t taddr = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    for (int c0 = 0; c0 < kF4Bn && done; c0 += kGated ? 64 : 32) {
      uint32_t r[32], u[32];
      __syncwarp();
      tmem_ld32(taddr + c0, r);
      if constexpr (kGated) tmem_ld32(taddr + c0 + 32, u);
      tmem_ld_wait();
      if (m >= p.M) continue;
      const int col = kGated ? (n0 + c0) / 2 : n0 + c0;
#pragma unroll
      for (int i = 0; i < 32; i += 8) {
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float v[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int c = i + 2 * k + e;
            v[e] = fmaf(__uint_as_float(r[c]), xs * s_ws[c0 + c], s_b[c0 + c]);
            if constexpr (kGated) v[e] = gelu_tanh(v[e]) * fmaf(__uint_as_float(u[c]), xs * s_ws[c0 + 32 + c], s_b[c0 + 32 + c]);
          }
          w[k] = pack2<OutT>(v[0], v[1]);
        }
        if (col + i < ldy) *reinterpret_cast<uint4*>(yrow + col + i) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 4) tmem_dealloc<256>(tmem);
}

template <int kFmt, bool kGated, typename OutT>
cudaError_t launch_f4(const Fp4GemmArgs& a) {
  auto kern = fp4_gemm_kernel<kFmt, kGated, OutT>;
  cudaError_t e = prepare_kernel(reinterpret_cast<const void*>(kern), kF4Smem);
  if (e != cudaSuccess) return e;
  CUtensorMap tx = {}, tw = {};
  e = make_tmap_bytes(&tx, a.xq, a.M, a.K / 2, kF4Bm);
  if (e == cudaSuccess) e = make_tmap_bytes(&tw, a.wq, a.N, a.K / 2, kF4Bn);
  if (e != cudaSuccess) return e;
  F4Params p = {a.xs, a.ws, a.xrow, a.wrow, a.bias, a.y, a.M, a.N, a.K};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.M + kF4Bm - 1) / kF4Bm), static_cast<unsigned>((a.N + kF4Bn - 1) / kF4Bn));
  cfg.blockDim = dim3(kF4Threads);
  cfg.dynamicSmemBytes = kF4Smem;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, kern, tx, tw, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int kFmt, bool kGated>
cudaError_t launch_f4_t(const Fp4GemmArgs& a) {
  return a.ydt == 0 ? launch_f4<kFmt, kGated, __half>(a) : launch_f4<kFmt, kGated, __nv_bfloat16>(a);
}

}  // namespace

cudaError_t launch_fp4_gemm(const Fp4GemmArgs& a) {
  if (a.fmt == fp4::kMx) return a.gated ? launch_f4_t<fp4::kMx, true>(a) : launch_f4_t<fp4::kMx, false>(a);
  return a.gated ? launch_f4_t<fp4::kNv, true>(a) : launch_f4_t<fp4::kNv, false>(a);
}

cudaError_t read_and_clear_error_word_fp4(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess || *out == 0) return e;
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

cudaError_t set_debug_hooks_fp4(unsigned long long wait_limit_ns, int hold_loads) { return set_debug_hooks(wait_limit_ns, hold_loads); }

}  // namespace qvla
