// Product of two matrices in 4-bit floating point with block scales, on tcgen05.mma with block scaling.
//
//   acc[m, n] = sum_k (c s)_x[m, k] (c s)_w[n, k]     codes and block scales multiplied by the tensor cores, float32 sums
//   y = fma(acc, xscale[m] wscale[n], bias[n]), or for a gated layer gelu_tanh(gate) up, rounded once
//
// Both kernels take the product weight-major, D[weight row, token]: the weights are the MMA's M side, whose 128 or 256 rows a
// layer always has, and the tokens its N side, which may be any multiple of 16.  k-blocks of 256 codes (128 bytes a row
// under the 128-byte swizzle) come by TMA through a ring, the scales beside them as whole tiles (fp4.cuh), which tcgen05.cp
// spreads over TMEM ahead of the products.
//
// Many tokens: persistent CTA pairs, tiles of 256 weight rows by 64 to 256 tokens.  Few: clusters of 1 to 8 CTAs that split a
// tile's K.
//
// us in a graph of calls (MX unless noted), one 128 x 128 tile a CTA on one SM before and these: 8192 x 2048 -> 16384 342
// and 94 (5.8 PFLOP/s); 816 x 2048 -> 2 x 16384 gated, NV, 81 and 28; 1187 x 4096 -> 2576 17.4 and 8.9; one token of 16384 ->
// 2048 24 and 5.5.  What bounds the large ones: without the epilogue's stores 8192 x 2048 -> 16384 takes 83 us, without the
// epilogue 79, at K = 64 an instruction (27 tiles a pair, 5600 cycles each at 1.9 GHz against 4350 of tensor work, 700 of them the hand-over of
// the one accumulator that fits); the 268 MB of outputs leave at 2.8 TB/s beside it.
// Tried and dropped: clusters of two pairs that share the tokens by multicast (102 us to 106: four-CTA clusters leave 8 of the
// 152 SMs idle, and the loads were not the bound), 16 epilogue warps (101 to 103), a second set of scale columns (the same),
// output lines of 64 bytes (the same), an evict-first hint on the stores (the same), token tiles of even width instead of whole
// ones and a remainder (816 tokens: 28.3 to 30.3), weights held in shared memory over the token tiles (K 2048: 95 to 110; with 512 as
// much faster as the order of units alone makes it), two pairs a tile with half of K each (816 x 16384 -> 2048, NV, 15.4 to 18.4: fewer
// stages a CTA, and the loads are the bound there), the gated epilogue without its GELU (0.7 us of 28).
#include "fp4_mma.cuh"

namespace qvla {
namespace {

// ---- many tokens: CTA pairs, persistent -------------------------------------------------------------------------------

// Warps: the epilogue's (two to a quadrant of 32 TMEM lanes; four to a quadrant took 103 us against 101 at 8192 x 2048 -> 16384),
// then one each for the products, the weights' loads and the tokens'.
constexpr int kPEpiWarps = 8, kPMma = 8, kPTmaW = 9, kPTmaX = 10, kPThreads = 11 * 32;
constexpr int kPMaxStages = 6;
constexpr int kPOutChunk = 32 * 128;            // 32 tokens of 64 channels
constexpr int kPOut = 2 * 2 * 2 * kPOutChunk;   // [half of the warps][64 channels of a CTA's][two in turn]

struct PairParams {
  const float *xrow, *wrow, *bias;
  int M, N, K;  // N weight rows
  int tiles_m, tiles_n;
  int bn_last;  // columns of the last token tile: its tokens rounded up to 16
  int by_tokens;  // the order of work units
  // Work unit u.  By weights: first the whole token tiles, weight tile by weight tile, then the last one's where it is narrower (in plain
  // order a pair could meet whole tiles only: 816 tokens are 4 tiles of 256 or fewer, and 4 divides 76 pairs), so that weights come from
  // memory once.  By tokens: what the pairs write at a time are whole rows of y nearly, so that outputs leave faster.
  __device__ __forceinline__ void unit(int u, int& ta, int& tb, int bn) const {
    const int whole = tiles_m - (bn_last < bn ? 1 : 0);
    if (!by_tokens && u < whole * tiles_n) {
      tb = u / whole;
      ta = u - tb * whole;
    } else {
      ta = u / tiles_n;
      tb = u - ta * tiles_n;
    }
  }
};

__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const void* tmap, int x, int y, int z, uint32_t cluster_bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(x), "r"(y), "r"(z), "r"(cluster_bar)
      : "memory");
}
// In both CTAs of the pair, each from its own shared memory to its own TMEM.
__device__ __forceinline__ void copy_scales_pair(uint32_t taddr, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <int kFmt>
__device__ __forceinline__ void mma_e2m1_pair(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t sa, uint32_t sb,
                                              uint32_t accumulate) {
  if constexpr (kFmt == fp4::kMx) {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  } else {
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.b32 p, %6, 0;\n"
        "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d_tmem),
        "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate)
        : "memory");
  }
}

template <int kBn, int kFmt>
struct PairCfg {
  static constexpr int kTileCodes = kFmt == fp4::kMx ? 128 : 64;  // codes that a scale tile covers
  static constexpr int kKb = kBn <= 128 ? 2 : 1;                  // k-blocks of 256 codes a stage
  static constexpr int kTiles = kKb * 256 / kTileCodes;           // scale tiles of a stage
  static constexpr int kAtoms = (kBn + 127) / 128;                // 128-token groups of scales that a token tile meets
  static constexpr int kA1 = 128 * 128, kB1 = kBn / 2 * 128;      // bytes of a k-block
  static constexpr int kA = kKb * kA1, kB = kKb * kB1, kSa = kTiles * 512, kSb = kAtoms * kTiles * 512;
  static constexpr int kStage = (kA + kB + kSa + kSb + 1023) / 1024 * 1024;
  // (a second set of columns, so that a stage's scales need not wait for the products before, gained nothing)
  static constexpr int kScaleCols = 4 * kTiles * (1 + kAtoms);
  static constexpr int kBufs = 2 * kBn + kScaleCols <= 512 ? 2 : 1;
  static constexpr int kChunks = kBn / 64;  // 32-token chunks of an epilogue warp: every second one
  static constexpr int kStagesRaw = (220 * 1024 - kPOut) / kStage;
  static constexpr int kStages = kStagesRaw > kPMaxStages ? kPMaxStages : kStagesRaw;
  static constexpr int kSmem = kStages * kStage + kPOut + 1024;
};

// D[weight row, token] = W X^T on a pair: 256 weight rows (128 a CTA, the lanes of its TMEM) by kBn tokens (columns; half of
// them in each CTA's shared memory).
template <int kBn, int kFmt, bool kGated, typename OutT>
__global__ void __launch_bounds__(kPThreads, 1) fp4_pair_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_xs,
                                                                const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws,
                                                                const __grid_constant__ CUtensorMap tmap_y, const PairParams p) {
  using C = PairCfg<kBn, kFmt>;
  constexpr int S = C::kStages;
  extern __shared__ uint8_t dyn_smem[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bar_full[S];   // leader: both CTAs' loads of the stage have landed
  __shared__ __align__(8) uint64_t bar_empty[S];  // the products have read it (in both CTAs)
  __shared__ __align__(8) uint64_t bar_tfull[C::kBufs], bar_tempty[C::kBufs], bar_done;
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_left[4];

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int nkb = (p.K + 255) / 256;
  const int units = p.tiles_m * p.tiles_n;
  const int unit0 = static_cast<int>(blockIdx.x >> 1), ustep = static_cast<int>(gridDim.x >> 1);
  uint8_t* const out_smem = smem + S * C::kStage;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 2);  // both loading warps' expected bytes
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    for (int i = 0; i < C::kBufs; ++i) {
      mbar_init(smem_u32(&bar_tfull[i]), 1);
      mbar_init(smem_u32(&bar_tempty[i]), 2 * kPEpiWarps);
    }
    mbar_init(smem_u32(&bar_done), 1);
    mbar_init_fence();
    for (int i = 0; i < 4; ++i) s_left[i] = 0;
  }
  if (warp == kPMma) tmem_alloc_pair<512>(smem_u32(&s_tmem_base));
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // both CTAs' barriers exist before any arrival crosses the pair
  tc_fence_after();
  const uint32_t tmem = s_tmem_base, t_sa = tmem + C::kBufs * kBn, t_sb = t_sa + 4 * C::kTiles;
  if (threadIdx.x == 0) griddep_launch_dependents();

  if (warp == kPTmaW || warp == kPTmaX) {
    // one warp loads the weights, one the tokens
    bool ok = *const_cast<volatile int*>(&g_debug_hold_loads) == 0;  // test hook: issue nothing
    if (warp == kPTmaX) griddep_wait();  // (no earlier kernel writes the weights)
    int it = 0, s = 0;
    uint32_t ph = 0;
    for (int u = unit0; u < units && ok; u += ustep) {
      int ta, tb;
      p.unit(u, ta, tb, kBn);
      const int n = ta == p.tiles_m - 1 ? p.bn_last : kBn;
      const int token = ta * kBn + static_cast<int>(rank) * (n / 2), row = tb * 256 + static_cast<int>(rank) * 128;
      for (int kb = 0; kb < nkb; kb += C::kKb, ++it) {
        if (warp == kPTmaW && it == S) griddep_wait();  // (the ring is full until there are tokens)
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_empty[s]), ph ^ 1u))) { ok = false; break; }
        const uint32_t full = smem_u32(&bar_full[s]), lead = mapa_shared(full, 0), dst = smem_u32(smem + s * C::kStage);
        if (elect_one()) {
          if (warp == kPTmaW) {
            if (rank == 0) mbar_arrive_expect_tx(full, 2 * (C::kA + C::kSa));
#pragma unroll
            for (int h = 0; h < C::kKb; ++h) tma_load_2d_pair(dst + h * C::kA1, &tmap_w, (kb + h) * 128, row, lead);
            tma_load_3d_pair(dst + C::kA + C::kB, &tmap_ws, 0, kb * (256 / C::kTileCodes), row / 128, lead);
          } else {
            if (rank == 0) mbar_arrive_expect_tx(full, 2 * (C::kB + C::kSb));
            const int t0 = kb * (256 / C::kTileCodes), g0 = ta * kBn / 128;
#pragma unroll
            for (int h = 0; h < C::kKb; ++h) tma_load_2d_pair(dst + C::kA + h * C::kB1, &tmap_x, (kb + h) * 128, token, lead);
            tma_load_3d_pair(dst + C::kA + C::kB + C::kSa, &tmap_xs, 0, t0, g0, lead);
          }
        }
        __syncwarp();
        if (++s == S) { s = 0; ph ^= 1u; }
      }
    }
    // before leaving, let every load land: the products that read a stage release it
    if (warp == kPTmaW && it < S) griddep_wait();
    for (int i = 0; i < S && i < it; ++i) {
      if (--s < 0) { s = S - 1; ph ^= 1u; }
      ok = ok && mbar_wait(smem_u32(&bar_empty[s]), ph);  // (after a time-out nothing will release the rest)
    }
    __syncwarp();
  } else if (warp == kPMma) {
    griddep_wait();  // (nothing of its own to wait for: it would poll for tokens beside a kernel that is still running)
    if (rank == 0) {
      int s = 0, tile_iter = 0;
      uint32_t ph = 0;
      bool ok = true;
      for (int u = unit0; u < units && ok; u += ustep, ++tile_iter) {
        int ta, tb;
        p.unit(u, ta, tb, kBn);
        const int buf = tile_iter % C::kBufs;
        const uint32_t idesc = idesc_e2m1_f32(kFmt, 256, ta == p.tiles_m - 1 ? p.bn_last : kBn);
        if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_tempty[buf]), (static_cast<uint32_t>(tile_iter / C::kBufs) & 1u) ^ 1u))) break;
        tc_fence_after();
        const uint32_t d = tmem + static_cast<uint32_t>(buf * kBn);
        const uint32_t sb0 = t_sb + static_cast<uint32_t>((ta * kBn % 128) / 32);  // a tile may start in the middle of its first group (0 or 2)
        for (int kb = 0; kb < nkb; kb += C::kKb) {
          if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_full[s]), ph))) { ok = false; break; }
          tc_fence_after();
          if (elect_one()) {
            const uint32_t base = smem_u32(smem + s * C::kStage);
            const uint32_t sa = base + C::kA + C::kB, sb = sa + C::kSa;
#pragma unroll
            for (int t = 0; t < C::kTiles; ++t) {
              copy_scales_pair(t_sa + 4 * t, scale_desc(sa + t * 512));
#pragma unroll
              for (int g = 0; g < C::kAtoms; ++g)
                copy_scales_pair(t_sb + 4 * (t * C::kAtoms + g), scale_desc(sb + (g * C::kTiles + t) * 512));
            }
            const uint64_t da = smem_desc_sw128(base), db = smem_desc_sw128(base + C::kA);
            const int steps = min(4 * C::kKb, (p.K - kb * 256) / 64);
#pragma unroll
            for (int k = 0; k < 4 * C::kKb; ++k) {
              if (k >= steps) break;
              const int t = kFmt == fp4::kMx ? k >> 1 : k;
              const uint32_t id = kFmt == fp4::kMx ? 2u * (k & 1) : 0u;
              mma_e2m1_pair<kFmt>(d, da + (k >> 2) * (C::kA1 >> 4) + 2 * (k & 3), db + (k >> 2) * (C::kB1 >> 4) + 2 * (k & 3), idesc | (id << 4) | (id << 29), t_sa + 4 * t, sb0 + 4 * t * C::kAtoms,
                                  (kb | k) != 0 ? 1u : 0u);
            }
            mma_commit_pair(smem_u32(&bar_empty[s]), 3);
          }
          __syncwarp();
          if (++s == S) { s = 0; ph ^= 1u; }
        }
        if (!ok) break;
        if (elect_one()) mma_commit_pair(smem_u32(&bar_tfull[buf]), 3);
        __syncwarp();
      }
      if (elect_one()) {
        mma_commit_pair(smem_u32(&bar_done), 1);  // every product issued above is complete once this flips
        mbar_wait(smem_u32(&bar_done), 0);
      }
    }
    __syncwarp();
  } else {
    // A thread reads the accumulator as matrix fragments: of its quadrant's lanes 8 j + lane / 4 (j < 4) the token columns
    // 2 (lane % 4) and the next of every 8.  A gated layer's lanes 0-15 are gate rows and 16-31 the up rows of the same units.
    constexpr int kChunks = C::kChunks;
    const int quad = warp & 3, half = warp >> 2;
    const int r0 = lane >> 2;
    // The warps that write 64 channels of the same tokens together, whole 128-byte lines of y: two of them, of a gated layer
    // all four of a half.
    constexpr int kTogether = kGated ? 4 : 2;
    const int set = kGated ? half : half * 2 + (quad >> 1);
    const bool storer = quad % kTogether == 0 && lane == 0;
    auto meet = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(1 + set), "n"(kTogether * 32) : "memory"); };
    uint8_t* const out = out_smem + set * (2 * kPOutChunk);
    griddep_wait();  // xrow comes from the previous kernel, which may still read y
    int tile_iter = 0, chunk_iter = 0;
    for (int u = unit0; u < units; u += ustep, ++tile_iter) {
      int ta, tb;
      p.unit(u, ta, tb, kBn);
      const int buf = tile_iter % C::kBufs;
      const int row = tb * 256 + static_cast<int>(rank) * 128 + quad * 32;  // of the weights, this warp's first
      float ws[4], bs[4], xs[kChunks];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int n = min(row + 8 * j + r0, p.N - 1);
        ws[j] = __ldg(p.wrow + n);
        bs[j] = __ldg(p.bias + n);
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
        xs[c] = kFmt == fp4::kMx ? 1.0f : p.xrow[min(ta * kBn + (2 * c + half) * 32 + lane, p.M - 1)];
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_tfull[buf]), static_cast<uint32_t>(tile_iter / C::kBufs) & 1u)) && lane == 0)
        *const_cast<volatile int*>(&s_left[set]) = 1;
      meet();
      // every warp of a set leaves, or none (the next write comes seconds later at the earliest, when the next wait runs out)
      if (*const_cast<volatile int*>(&s_left[set])) break;
      tc_fence_after();
      const uint32_t taddr = tmem + (static_cast<uint32_t>(quad * 32) << 16) + static_cast<uint32_t>(buf * kBn + half * 32);
      uint32_t r[kChunks][32];  // [16 g + 4 c + 2 i + k]: lane 16 g + 8 i + r0, token 8 c + 2 (lane % 4) + k of the chunk
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        tmem_ld_16x256b_x4(taddr + c * 64, r[c]);
        tmem_ld_16x256b_x4(taddr + (16u << 16) + c * 64, r[c] + 16);
      }
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {  // the accumulator may be overwritten
        if (rank == 0) {
          mbar_arrive(smem_u32(&bar_tempty[buf]));
        } else {
          mbar_arrive_peer(mapa_shared(smem_u32(&bar_tempty[buf]), 0));
        }
      }
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        const int m = ta * kBn + (2 * c + half) * 32;
        if (m >= p.M) break;
        uint8_t* const dst = out + (chunk_iter & 1) * kPOutChunk;
        ++chunk_iter;
        uint32_t pk[4][4];  // [8-token group][row block j]
        uint32_t hk[4][2];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float x0 = kFmt == fp4::kMx ? 1.0f : __shfl_sync(0xffffffffu, xs[c], 8 * g + 2 * (lane & 3));
          const float x1 = kFmt == fp4::kMx ? 1.0f : __shfl_sync(0xffffffffu, xs[c], 8 * g + 2 * (lane & 3) + 1);
          float y[4][2];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int i = 16 * (j >> 1) + 4 * g + 2 * (j & 1);
            y[j][0] = fmaf(__uint_as_float(r[c][i]), x0 * ws[j], bs[j]);
            y[j][1] = fmaf(__uint_as_float(r[c][i + 1]), x1 * ws[j], bs[j]);
          }
          if constexpr (kGated) {
#pragma unroll
            for (int j = 0; j < 2; ++j) hk[g][j] = pack2<OutT>(gelu_fast(y[j][0]) * y[j + 2][0], gelu_fast(y[j][1]) * y[j + 2][1]);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) pk[g][j] = pack2<OutT>(y[j][0], y[j][1]);
          }
        }
        if (storer) bulk_wait_read_but<1>();  // the store before the last has read this buffer
        meet();
        // rows of 64 channels (128 bytes) under the 128-byte swizzle: 16-byte piece q of token t at q ^ t % 8
        const int t = lane & 7;
        if constexpr (kGated) {
          const uint32_t at = smem_u32(dst) + static_cast<uint32_t>((lane >> 4) * 1024 + t * 128 + (((2 * quad + ((lane >> 3) & 1)) ^ t) << 4));
#pragma unroll
          for (int g = 0; g < 4; g += 2) {
            const uint32_t h[4] = {hk[g][0], hk[g][1], hk[g + 1][0], hk[g + 1][1]};
            stmatrix_x4_trans(at + static_cast<uint32_t>(g * 1024), h);
          }
        } else {
          const uint32_t at = smem_u32(dst) + static_cast<uint32_t>(t * 128 + (((4 * (quad & 1) + (lane >> 3)) ^ t) << 4));
#pragma unroll
          for (int g = 0; g < 4; ++g) stmatrix_x4_trans(at + static_cast<uint32_t>(g * 1024), pk[g]);
        }
        fence_proxy_async_smem();  // the stores are read by the async proxy
        meet();
        if (storer) {  // tokens past M and channels past N are clipped
          const int n = kGated ? row / 2 : row;
          if (n < (kGated ? p.N / 2 : p.N)) tma_store_2d(&tmap_y, n, m, smem_u32(dst));
          bulk_commit();
        }
      }
    }
    if (storer) bulk_wait_all();
    __syncwarp();
  }

  tc_fence_before();
  __syncthreads();
  cluster_sync();  // the leader's products on this CTA's shared memory and TMEM are complete
  tc_fence_after();
  if (warp == kPMma) tmem_dealloc_pair<512>(tmem);
}

// The output [M][width] of 16-bit values, written in boxes of 64 channels x 32 tokens from 128-byte swizzled rows.
cudaError_t make_tmap_y(CUtensorMap* m, void* base, int rows, int width) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(width), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(width) * 2};
  const cuuint32_t box[2] = {64, 32};
  const cuuint32_t estr[2] = {1, 1};
  CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int kBn, int kFmt, bool kGated, typename OutT>
cudaError_t launch_pair(const Fp4GemmArgs& a) {
  using C = PairCfg<kBn, kFmt>;
  auto kern = fp4_pair_kernel<kBn, kFmt, kGated, OutT>;
  static std::atomic<unsigned long long> raised{0};
  cudaError_t e = raise_smem(reinterpret_cast<const void*>(kern), C::kSmem, &raised);
  if (e != cudaSuccess) return e;
  CUtensorMap tx = {}, txs = {}, ty = {};
  const CUtensorMap &tw = weight_map(a, 0), &tws = weight_map(a, C::kKb);
  const int tiles = a.K / C::kTileCodes;
  e = make_tmap_bytes(&tx, a.xq, a.M, a.K / 2, kBn / 2);
  if (e == cudaSuccess) e = make_tmap_scales(&txs, a.xs, (a.M + 127) / 128, tiles, C::kTiles, C::kAtoms);
  static_assert(C::kSmem >= 161 * 1024, "no CTA of a cluster of the split kernel beside this one (its launch says why)");
  if (e == cudaSuccess) e = make_tmap_y(&ty, a.y, a.M, kGated ? a.N / 2 : a.N);
  if (e != cudaSuccess) return e;
  // By tokens where the outputs are more than 8 times the weights.  Both orders at 192 shapes (816 to 8192 tokens, K 256 to 4096, 1024 to
  // 16384 outputs, gated ones among them, MX and NV, other weights in every call): where the rule takes it, 4.4% faster in the mean, 24% at
  // best (4096 x 256 -> 16384, MX, 26.1 us against 32.4; 8192 x 1024 -> 16384 58.5 against 62.6; 8192 x 2048 -> 16384 the same) and 3% slower at
  // worst (2048 x 512 -> 1024, NV, 5.1 against 5.0); where it does not, it would be 10% faster to 4% slower (816 x 2048 -> 2 x 16384 29.7 against 28.5).
  const bool by_tokens = 2ll * a.M * (kGated ? a.N / 2 : a.N) > 8ll * a.N * (a.K / 2);
  PairParams p = {a.xrow, a.wrow, a.bias, a.M, a.N, a.K, (a.M + kBn - 1) / kBn, (a.N + 255) / 256, 0, by_tokens};
  p.bn_last = (a.M - (p.tiles_m - 1) * kBn + 15) / 16 * 16;
  const int units = p.tiles_m * p.tiles_n, pairs = a.num_sms / 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * (units < pairs ? units : pairs)));
  cfg.blockDim = dim3(kPThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  e = cudaLaunchKernelEx(&cfg, kern, tx, txs, tw, tws, ty, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// ---- few tokens: a tile's K split over a cluster ------------------------------------------------------------------------

constexpr int kSEpiWarps = 4, kSMma = 4, kSTma = 5, kSThreads = 6 * 32;
constexpr int kSMaxStages = 12;

struct F4SplitParams {
  const float *xrow, *wrow, *bias;
  void* y;
  int M, N, K;
  int stages;  // of the ring
};

template <int kBn, int kFmt>
struct SplitCfg {
  static constexpr int kTileCodes = kFmt == fp4::kMx ? 128 : 64;
  static constexpr int kTiles = 256 / kTileCodes;
  static constexpr int kA = 128 * 128, kB = kBn * 128, kScale = kTiles * 512;
  static constexpr int kBytes = kA + kB + 2 * kScale;
  static constexpr int kStage = (kBytes + 1023) / 1024 * 1024;
  static constexpr int kRecv = 128 * kBn * 4;  // partial sums from the cluster's CTAs
  static constexpr int kColumns = kBn + 8 * kTiles;
  static constexpr uint32_t kTmem = kColumns <= 64 ? 64 : kColumns <= 128 ? 128 : 256;
};

// D[weight row, token]: 128 weight rows by kBn tokens a cluster, whose CTAs (kSplit) take equal parts of K.  Every CTA keeps
// kBn / kSplit tokens and sends the others' partial sums to the CTAs that keep those, with stores that complete on the
// receiver's barrier; it adds the parts in the order of K.
template <int kBn, int kSplit, int kFmt, bool kGated, typename OutT>
__global__ void __launch_bounds__(kSThreads, 1) fp4_split_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_xs,
                                                                 const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws,
                                                                 const F4SplitParams p) {
  using C = SplitCfg<kBn, kFmt>;
  constexpr int kKeep = kBn / kSplit;  // tokens of a CTA
  static_assert(kBn == 32 || kBn % 64 == 0, "tiles begin at even columns of the scales");
  static_assert(kKeep % 4 == 0, "four tokens travel together");
  extern __shared__ uint8_t dyn_smem[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bar_full[kSMaxStages], bar_empty[kSMaxStages], bar_done, bar_recv;
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int S = p.stages;
  const int rank = kSplit > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int tb = static_cast<int>(blockIdx.x) / kSplit, ta = static_cast<int>(blockIdx.y);
  const int nkb = (p.K + 255) / 256;
  const int ka = nkb * rank / kSplit, kz = nkb * (rank + 1) / kSplit;
  uint8_t* const recv = smem + S * C::kStage;  // [part][token / 4][128 rows] float4

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    mbar_init(smem_u32(&bar_done), 1);
    mbar_init(smem_u32(&bar_recv), 1);
    mbar_init_fence();
    s_abort = 0;
    if (kSplit > 1) mbar_arrive_expect_tx(smem_u32(&bar_recv), (kSplit - 1) * kKeep * 128 * 4);
  }
  if (warp == kSMma) tmem_alloc<C::kTmem>(smem_u32(&s_tmem_base));
  tc_fence_before();
  __syncthreads();
  if (kSplit > 1) cluster_arrive_relaxed();  // waited for ahead of the first store to another CTA
  tc_fence_after();
  const uint32_t tmem = s_tmem_base, t_sa = tmem + kBn, t_sb = t_sa + 4 * C::kTiles;
  griddep_launch_dependents();

  if (warp == kSTma) {
    bool ok = *const_cast<volatile int*>(&g_debug_hold_loads) == 0;  // test hook: issue nothing
    auto weights = [&](int kb, int s) {  // no earlier kernel writes them
      const uint32_t full = smem_u32(&bar_full[s]), dst = smem_u32(smem + s * C::kStage);
      mbar_arrive_expect_tx(full, C::kBytes);
      tma_load_2d(dst, &tmap_w, kb * 128, tb * 128, full);
      tma_load_3d(dst + C::kA + C::kB, &tmap_ws, 0, kb * C::kTiles, tb, full);
    };
    auto tokens = [&](int kb, int s) {
      const uint32_t full = smem_u32(&bar_full[s]), dst = smem_u32(smem + s * C::kStage);
      tma_load_2d(dst + C::kA, &tmap_x, kb * 128, ta * kBn, full);
      tma_load_3d(dst + C::kA + C::kB + C::kScale, &tmap_xs, 0, kb * C::kTiles, ta * kBn / 128, full);
    };
    const int first = min(S, kz - ka);
    if (ok && elect_one())
      for (int i = 0; i < first; ++i) weights(ka + i, i);
    __syncwarp();
    griddep_wait();
    if (ok && elect_one())
      for (int i = 0; i < first; ++i) tokens(ka + i, i);
    __syncwarp();
    int it = ok ? first : 0, s = first == S ? 0 : first;
    uint32_t ph = first == S ? 1 : 0;
    for (int kb = ka + first; kb < kz && ok; ++kb, ++it) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_empty[s]), ph ^ 1u))) { ok = false; break; }
      if (elect_one()) {
        weights(kb, s);
        tokens(kb, s);
      }
      __syncwarp();
      if (++s == S) { s = 0; ph ^= 1u; }
    }
    // before leaving, let every load land
    for (int i = max(0, it - S); i < it; ++i) mbar_wait(smem_u32(&bar_full[i % S]), static_cast<uint32_t>(i / S) & 1u);
    __syncwarp();
  } else if (warp == kSMma) {
    griddep_wait();  // (it would only poll)
    const int tokens = min(p.M - ta * kBn, kBn);
    const uint32_t idesc = idesc_e2m1_f32(kFmt, 128, (tokens + 15) / 16 * 16);
    // The address of scales in TMEM has to be even (an odd one is a misaligned address): tiles of 32 tokens begin at token 0.
    const uint32_t sb0 = t_sb + static_cast<uint32_t>((ta * kBn % 128) / 64 * 2);
    bool ok = true;
    int s = 0;
    uint32_t ph = 0;
    for (int kb = ka; kb < kz; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_full[s]), ph))) { ok = false; break; }
      tc_fence_after();
      if (elect_one()) {
        const uint32_t base = smem_u32(smem + s * C::kStage);
        const uint32_t sa = base + C::kA + C::kB, sb = sa + C::kScale;
#pragma unroll
        for (int t = 0; t < C::kTiles; ++t) {
          copy_scales(t_sa + 4 * t, scale_desc(sa + t * 512));
          copy_scales(t_sb + 4 * t, scale_desc(sb + t * 512));
        }
        const uint64_t da = smem_desc_sw128(base), db = smem_desc_sw128(base + C::kA);
        const int steps = min(4, (p.K - kb * 256) / 64);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k >= steps) break;
          const int t = kFmt == fp4::kMx ? k >> 1 : k;
          const uint32_t id = kFmt == fp4::kMx ? 2u * (k & 1) : 0u;
          mma_e2m1<kFmt>(tmem, da + 2 * k, db + 2 * k, idesc | (id << 4) | (id << 29), t_sa + 4 * t, sb0 + 4 * t, (kb != ka || k != 0) ? 1u : 0u);
        }
        mma_commit(smem_u32(&bar_empty[s]));
      }
      __syncwarp();
      if (++s == S) { s = 0; ph ^= 1u; }
    }
    if (elect_one()) {
      if (!ok) *const_cast<volatile int*>(&s_abort) = 1;
      __threadfence_block();
      mma_commit(smem_u32(&bar_done));  // also after a wait ran out: what was issued is waited for
    }
    __syncwarp();
  } else {
    const int n = tb * 128 + warp * 32 + lane;  // this thread's weight row
    const int nc = min(n, p.N - 1);
    const float ws = __ldg(p.wrow + nc), bs = __ldg(p.bias + nc);
    griddep_wait();  // xrow comes from the previous kernel (so no read-only load of it), which may still read y
    const int m0 = ta * kBn + rank * kKeep;  // the first token that this CTA keeps
    const int row = warp * 32 + lane;
    bool done = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_done), 0) && *const_cast<volatile int*>(&s_abort) == 0);
    __syncwarp();
    tc_fence_after();
    const uint32_t taddr = tmem + (static_cast<uint32_t>(warp * 32) << 16);
    if (kSplit > 1) cluster_wait();  // every CTA's barrier exists
    // partial sums of the tokens that others keep
    if (kSplit > 1 && done) {
#pragma unroll 1
      for (int c0 = 0; c0 < kBn; c0 += 32) {
        uint32_t r[32];
        __syncwarp();
        tmem_ld32(taddr + c0, r);
        tmem_ld_wait();
#pragma unroll
        for (int g = 0; g < 8; ++g) {
          const int t = c0 + 4 * g, to = t / kKeep;
          if (to == rank) continue;
          const uint32_t at = smem_u32(recv) + static_cast<uint32_t>(((rank * (kKeep / 4) + (t - to * kKeep) / 4) * 128 + row) * 16);
          st_async_v4(mapa_shared(at, to), make_float4(__uint_as_float(r[4 * g]), __uint_as_float(r[4 * g + 1]), __uint_as_float(r[4 * g + 2]), __uint_as_float(r[4 * g + 3])),
                      mapa_shared(smem_u32(&bar_recv), to));
        }
      }
      done = __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&bar_recv), 0));
    }
    const int ldy = kGated ? p.N / 2 : p.N;
    const int col = kGated ? tb * 64 + warp * 16 + (lane & 15) : n;
    const bool store = done && (kGated ? lane < 16 : n < p.N);
    OutT* const y = static_cast<OutT*>(p.y) + col;
    constexpr int kChunk = kKeep < 32 ? kKeep : 32;
#pragma unroll 1
    for (int c0 = 0; c0 < kKeep && m0 + c0 < p.M && done; c0 += kChunk) {
      float v[kChunk];
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kChunk; i += 4) {
        uint32_t r[4];
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(taddr + rank * kKeep + c0 + i));
        tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i + k] = __uint_as_float(r[k]);
      }
      if (kSplit > 1) {
#pragma unroll
        for (int i = 0; i < kChunk; i += 4) {
          float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
          for (int q = 0; q < kSplit; ++q) {
            float4 a = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            if (q != rank) a = *reinterpret_cast<const float4*>(recv + ((q * (kKeep / 4) + (c0 + i) / 4) * 128 + row) * 16);
            sum = make_float4(sum.x + a.x, sum.y + a.y, sum.z + a.z, sum.w + a.w);
          }
          v[i] = sum.x, v[i + 1] = sum.y, v[i + 2] = sum.z, v[i + 3] = sum.w;
        }
      }
#pragma unroll
      for (int i = 0; i < kChunk; ++i) {
        const int m = m0 + c0 + i;
        const float xs = kFmt == fp4::kMx ? 1.0f : p.xrow[min(m, p.M - 1)];
        float a = fmaf(v[i], xs * ws, bs);
        if constexpr (kGated) a = gelu_fast(a) * __shfl_down_sync(0xffffffffu, a, 16);
        if (store && m < p.M) {
          const uint32_t h = pack2<OutT>(a, 0.0f);
          *reinterpret_cast<uint16_t*>(y + static_cast<size_t>(m) * ldy) = static_cast<uint16_t>(h);
        }
      }
    }
  }
  if (kSplit > 1 && warp >= kSEpiWarps) cluster_wait();
  tc_fence_before();
  __syncthreads();
  if (kSplit > 1) cluster_sync();  // no CTA leaves while another may still send to it (after a wait ran out)
  tc_fence_after();
  if (warp == kSMma) tmem_dealloc<C::kTmem>(tmem);
}

template <int kBn, int kSplit, int kFmt, bool kGated, typename OutT>
cudaError_t launch_split(const Fp4GemmArgs& a) {
  using C = SplitCfg<kBn, kFmt>;
  if (kBn == 32 && a.M > 32) return cudaErrorInvalidValue;  // (see the kernel)
  auto kern = fp4_split_kernel<kBn, kSplit, kFmt, kGated, OutT>;
  constexpr int kRecv = kSplit > 1 ? C::kRecv : 0;
  constexpr int kMost = std::min(kSMaxStages, (220 * 1024 - kRecv) / C::kStage), kHalf = (110 * 1024 - kRecv) / C::kStage;
  static std::atomic<unsigned long long> raised{0};
  cudaError_t e = raise_smem(reinterpret_cast<const void*>(kern), kMost * C::kStage + kRecv + 1024, &raised);
  if (e != cudaSuccess) return e;
  CUtensorMap tx = {}, txs = {};
  const CUtensorMap &tw = weight_map(a, 0), &tws = weight_map(a, 1);
  const int tiles = a.K / C::kTileCodes, nkb = (a.K + 255) / 256;
  e = make_tmap_bytes(&tx, a.xq, a.M, a.K / 2, kBn);
  if (e == cudaSuccess) e = make_tmap_scales(&txs, a.xs, (a.M + 127) / 128, tiles, C::kTiles, 1);
  if (e != cudaSuccess) return e;
  const int range = (nkb + kSplit - 1) / kSplit;
  const unsigned weight_tiles = static_cast<unsigned>((a.N + 127) / 128), token_tiles = static_cast<unsigned>((a.M + kBn - 1) / kBn);
  // One CTA an SM while all clusters run at once so; clusters of 4 and 8 leave SMs of their GPC over.
  const unsigned at_once = static_cast<unsigned>(a.num_sms) * (kSplit == 8 ? 3u : kSplit == 4 ? 15u : 16u) / (kSplit == 8 ? 4u : 16u) / kSplit;
  const int most = weight_tiles * token_tiles <= at_once ? kMost : kHalf;
  F4SplitParams p = {a.xrow, a.wrow, a.bias, a.y, a.M, a.N, a.K, range < most ? range : most};
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(weight_tiles * kSplit, token_tiles);
  cfg.blockDim = dim3(kSThreads);
  // CTAs that wait for one another must not wait for TMEM too, which a CTA of another stream's kernel could hold while it waits
  // for one that these keep out: with 68 KB at least, none of them shares an SM with a kernel that takes all columns (the least
  // of them the prompt attention's of 64 channels, 161 KB), and the three that fit an SM find theirs (128 at most).
  const size_t smem = static_cast<size_t>(p.stages) * C::kStage + kRecv + 1024;
  static_assert(C::kTmem <= 128, "three CTAs' columns");
  cfg.dynamicSmemBytes = kSplit > 1 ? std::max(smem, size_t{68} << 10) : smem;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kSplit;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kSplit > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, kern, tx, txs, tw, tws, p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

// ---- the choice -------------------------------------------------------------------------------------------------------

struct F4Plan {
  int bn, split;  // split 0: CTA pairs with tiles of bn tokens; else clusters of `split` CTAs
};

// Estimated time (ns) of the pair kernel: a fixed part, the pairs at work, and what the pair with most to do spends: for every
// tile its k-blocks and the hand-over to the epilogue (which at 2048 channels also holds the wait for the memory's writes).
// Fitted, like the next one, to launches of 1 to 4096 tokens, K 512 to 16384, 512 to 16384 outputs on a GB300: the choice was
// 1.5% above the best of the eleven variants in the mean, 17% at worst (200 x 16384 -> 2048).
long pair_estimate(const Fp4GemmArgs& a, int bn) {
  const long pairs = a.num_sms / 2, nkb = (a.K + 255) / 256, tiles_m = (a.M + bn - 1) / bn, tiles_n = (a.N + 255) / 256;
  const long last = (a.M - (tiles_m - 1) * bn + 15) / 16 * 16;
  auto tile = [&](long columns) {
    long kb = a.fmt == fp4::kMx ? 112 + 68 * columns / 100 : 120 + 78 * columns / 100;
    if (bn > 128 && kb < 200) kb = 200;  // a round of loads and products for every k-block; up to 128 columns for two
    return nkb * kb + 100 + 33 * columns / 10;
  };
  const long whole = (tiles_m - (last < bn ? 1 : 0)) * tiles_n, units = tiles_m * tiles_n;
  auto worst = [&](long pair) {  // its units are pair, pair + pairs, ...: whole tiles first
    const long n = pair < whole ? (whole - pair + pairs - 1) / pairs : 0;
    const long next = n * pairs + pair, rest = next < units ? (units - next + pairs - 1) / pairs : 0;
    return n * tile(bn) + rest * tile(last);
  };
  const long most = std::max(worst(0), whole % pairs < units ? worst(whole % pairs) : 0);
  return 2300 + 22 * bn / 10 + most + 14 * std::min(units, pairs);
}

// The same of the split kernel: k-blocks of a CTA, slower where several share an SM, and the exchange of the partial sums.
long split_estimate(const Fp4GemmArgs& a, int bn, int split) {
  const long nkb = (a.K + 255) / 256, ctas = static_cast<long>((a.N + 127) / 128) * ((a.M + bn - 1) / bn) * split;
  long t = (split == 1 ? 2300 : 2500) + (bn == 64 ? 700 : 0) + 250 * ((nkb + split - 1) / split) * std::max(ctas, 140l) / 140;
  if (split > 1) t += 16l * bn * (split - 1) / split * std::max(ctas, 50l) / 100;
  return ctas > 273 ? t * ctas / 273 : t;
}

F4Plan plan_gemm(const Fp4GemmArgs& a) {
  F4Plan best = {64, 0};
  long t = pair_estimate(a, 64);
  auto offer = [&](long other, F4Plan p) {
    if (other < t) {
      t = other;
      best = p;
    }
  };
  for (int bn = 128; bn <= 256; bn += 64) offer(pair_estimate(a, bn), {bn, 0});
  const int nkb = (a.K + 255) / 256;
  for (int split = 1; split <= 8 && split <= nkb; split *= 2) {  // every CTA has a k-block
    if (a.M <= 32) offer(split_estimate(a, 32, split), {32, split});
    if (a.M > 32 && split > 1) offer(split_estimate(a, 64, split), {64, split});
  }
  return best;
}

template <int kFmt, bool kGated, typename OutT>
cudaError_t launch_any(const Fp4GemmArgs& a) {
  const F4Plan p = plan_gemm(a);
  switch (p.split * 1000 + p.bn) {
    case 256: return launch_pair<256, kFmt, kGated, OutT>(a);
    case 192: return launch_pair<192, kFmt, kGated, OutT>(a);
    case 128: return launch_pair<128, kFmt, kGated, OutT>(a);
    case 1032: return launch_split<32, 1, kFmt, kGated, OutT>(a);
    case 2032: return launch_split<32, 2, kFmt, kGated, OutT>(a);
    case 4032: return launch_split<32, 4, kFmt, kGated, OutT>(a);
    case 8032: return launch_split<32, 8, kFmt, kGated, OutT>(a);
    case 2064: return launch_split<64, 2, kFmt, kGated, OutT>(a);
    case 4064: return launch_split<64, 4, kFmt, kGated, OutT>(a);
    case 8064: return launch_split<64, 8, kFmt, kGated, OutT>(a);
    default: return launch_pair<64, kFmt, kGated, OutT>(a);
  }
}

template <int kFmt, bool kGated>
cudaError_t launch_f4_t(const Fp4GemmArgs& a) {
  return a.ydt == 0 ? launch_any<kFmt, kGated, __half>(a) : launch_any<kFmt, kGated, __nv_bfloat16>(a);
}

}  // namespace

static_assert(sizeof(CUtensorMap) <= kFp4MapBytes && alignof(CUtensorMap) <= kFp4MapBytes, "a map's place");

cudaError_t fp4_weight_maps(const uint8_t* wq, const uint8_t* ws, int fmt, int N, int K, void* maps) {
  uint8_t* const at = static_cast<uint8_t*>(maps);
  const int codes = fmt == fp4::kMx ? 128 : 64, groups = (N + 255) / 256 * 2;
  cudaError_t e = make_tmap_bytes(reinterpret_cast<CUtensorMap*>(at), wq, N, K / 2, 128);
  for (int i = 1; i < kFp4Maps && e == cudaSuccess; ++i)
    e = make_tmap_scales(reinterpret_cast<CUtensorMap*>(at + i * kFp4MapBytes), ws, groups, K / codes, i * 256 / codes, 1);
  return e;
}

int fp4_split(const Fp4GemmArgs& a) {
  const F4Plan p = plan_gemm(a);
  return p.bn == 32 ? p.split : 0;
}

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
