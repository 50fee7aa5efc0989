// One launch for the linear of 1 to 4 tokens in 4-bit floating point: rotation, quantiser and product.
//
// The clusters of the split product (fp4_gemm.cu), whose CTAs take equal parts of K.  Here each makes the codes of its own part: it
// loads the channels of the rotation's blocks that the part touches (they may reach into its neighbours', which rotate them too), rotates
// them, trades the rows' largest magnitudes with the cluster (NV without a step's scale), and writes codes and block scales to shared
// memory as the product takes them, while its weights are on their way.  Codes, scales and the order of sums are those of the quantiser and
// the product one after the other, and so are the outputs, to the bit.
//
// us in a graph of calls, one launch and two: a token of 16384 -> 2048, b 2048, NV 7.2 and 8.6, MX 5.6 and 7.6; 2048 -> 2048 5.0 and 5.3; 1024
// -> 4096, b 64, MX 3.3 and 4.4; 4096 -> 4096, b 4096 (whose parts of 512 channels each rotate all) 6.0 and 6.0; and one launch less of the
// host's time (2).  What is left is a chain: the row's load, rotation, exchange (1.2 us, NV), codes, 8 k-blocks of products, join.
#include "fp4_mma.cuh"
#include "fp4_rows.cuh"

namespace qvla {
namespace {

using namespace fp4;

constexpr int kTokens = 4;           // at most
constexpr int kTWorkWarps = 4;       // quantise, and then read the sums out
constexpr int kTMma = 4, kTTma = 5, kTThreads = 6 * 32, kTMaxStages = 12;
// The product takes 16 token rows of 256 codes (two groups of 8, 1024 bytes each) and scale tiles of 32 rows, of which the first 4 count:
// k-blocks and tiles lie closer, and what the rows behind the tokens hold (the next ones' bytes) stays in sums that nobody reads.
constexpr int kTOperand = 8 * 128, kTTile = kTokens * 16;

struct TokenParams {
  const void* x;
  const float *step, *wrow, *bias;
  void* y;
  float inv_sqrt_b;
  int M, N, K, log_b, gated;
  int threads;  // of a row
  int stages, most;  // of the weights' ring; k-blocks of a CTA at most
};

template <int kFmt>
struct TokenCfg {
  static constexpr int kTiles = kFmt == kMx ? 2 : 4;  // scale tiles of 256 codes
  static constexpr int kA = 128 * 128, kScale = kTiles * 512, kStage = (kA + kScale + 1023) / 1024 * 1024;
  static constexpr int kTmem = 64;  // sums of 16 tokens (of 32 columns), 8 kTiles of scales
};

__device__ __forceinline__ void work_sync() { asm volatile("bar.sync 7, %0;" ::"n"(kTWorkWarps * 32) : "memory"); }

template <int kLayout, typename T>
__device__ __forceinline__ void load_rotated(const TokenParams& p, const T* src, int j, bool there, uint32_t lines, float2 (&v)[16]) {
  using P = Place<kLayout>;
  const P place(j);
  if (there) {
#pragma unroll
    for (int u = 0; u < P::kUnits; ++u) load_unit<P::kUnit>(src + place.channel(u), v + u * P::kPer);
  }
  rotate<kLayout, true>(p.log_b, p.inv_sqrt_b, j, lines, v);
}

template <int kSplit, int kFmt, typename T>
__global__ void __launch_bounds__(kTThreads, 1) fp4_token_kernel(const __grid_constant__ CUtensorMap tmap_w, const __grid_constant__ CUtensorMap tmap_ws,
                                                                 const TokenParams p) {
  using C = TokenCfg<kFmt>;
  extern __shared__ uint8_t dyn_smem[];
  uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_smem) + 1023) & ~uintptr_t(1023));
  __shared__ __align__(8) uint64_t bar_full[kTMaxStages], bar_empty[kTMaxStages], bar_tokens, bar_done, bar_most, bar_recv;
  __shared__ __align__(16) float s_peers[kSplit][kTokens];  // the rows' largest magnitudes in each CTA's channels
  __shared__ float s_warps[kTWorkWarps], s_delta[kTokens];
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;

  const int warp = warp_index(), lane = threadIdx.x & 31;
  const int S = p.stages;
  const int rank = kSplit > 1 ? static_cast<int>(cluster_ctarank()) : 0;
  const int tb = static_cast<int>(blockIdx.x) / kSplit;
  const int nkb = (p.K + 255) / 256;
  const int ka = nkb * rank / kSplit, kz = nkb * (rank + 1) / kSplit;
  uint8_t* const operand = smem + S * C::kStage;                   // [k-block][8 tokens][128 bytes], 128-byte swizzled, and 8 rows more
  uint8_t* const scales = operand + (p.most + 1) * kTOperand;      // [k-block][tile][64 bytes], and 512 more
  uint8_t* const recv = scales + p.most * C::kTiles * kTTile + 512;  // of the first CTA: [part][128 rows] float4
  uint8_t* const lines = recv + (kSplit > 1 ? kSplit * 2048 : 0);  // the rotation's exchanges: 128 bytes a thread
  const bool trade = kFmt == kNv && kSplit > 1 && p.step == nullptr;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S; ++s) {
      mbar_init(smem_u32(&bar_full[s]), 1);
      mbar_init(smem_u32(&bar_empty[s]), 1);
    }
    mbar_init(smem_u32(&bar_tokens), kTWorkWarps);
    mbar_init(smem_u32(&bar_done), 1);
    mbar_init(smem_u32(&bar_most), 1);
    mbar_init(smem_u32(&bar_recv), 1);
    mbar_init_fence();
    s_abort = 0;
    if (trade) mbar_arrive_expect_tx(smem_u32(&bar_most), kSplit * 16);
    if (kSplit > 1 && rank == 0) mbar_arrive_expect_tx(smem_u32(&bar_recv), (kSplit - 1) * 128 * 16);
  }
  if (warp == kTMma) tmem_alloc<C::kTmem>(smem_u32(&s_tmem_base));
  tc_fence_before();
  __syncthreads();
  if (kSplit > 1) cluster_arrive_relaxed();  // waited for ahead of the first store to another CTA
  tc_fence_after();
  const uint32_t tmem = s_tmem_base, t_sa = tmem + 32, t_sb = t_sa + 4 * C::kTiles;
  griddep_launch_dependents();

  if (warp == kTTma) {  // the weights, which no earlier kernel writes
    bool ok = *const_cast<volatile int*>(&g_debug_hold_loads) == 0;  // test hook: issue nothing
    int it = 0, s = 0;
    uint32_t ph = 0;
    for (int kb = ka; kb < kz && ok; ++kb, ++it) {
      if (it == S) griddep_wait();  // (the ring is full until there are tokens: the wait's limit is not for the previous kernel)
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_empty[s]), ph ^ 1u))) break;
      if (elect_one()) {
        const uint32_t full = smem_u32(&bar_full[s]), dst = smem_u32(smem + s * C::kStage);
        mbar_arrive_expect_tx(full, C::kA + C::kScale);
        tma_load_2d(dst, &tmap_w, kb * 128, tb * 128, full);
        tma_load_3d(dst + C::kA, &tmap_ws, 0, kb * C::kTiles, tb, full);
      }
      __syncwarp();
      if (++s == S) { s = 0; ph ^= 1u; }
    }
    // before leaving, let every load land
    for (int i = max(0, it - S); i < it; ++i) mbar_wait(smem_u32(&bar_full[i % S]), static_cast<uint32_t>(i / S) & 1u);
    __syncwarp();
  } else if (warp == kTMma) {
    griddep_wait();  // (it would only poll)
    bool ok = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_tokens), 0) && *const_cast<volatile int*>(&s_abort) == 0);
    const uint32_t idesc = idesc_e2m1_f32(kFmt, 128, 16);
    int s = 0;
    uint32_t ph = 0;
    for (int kb = ka; kb < kz && ok; ++kb) {
      if (!__all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_full[s]), ph))) { ok = false; break; }
      tc_fence_after();
      if (elect_one()) {
        const uint32_t base = smem_u32(smem + s * C::kStage), tok = smem_u32(operand + (kb - ka) * kTOperand), sc = smem_u32(scales + (kb - ka) * C::kTiles * kTTile);
#pragma unroll
        for (int t = 0; t < C::kTiles; ++t) {
          copy_scales(t_sa + 4 * t, scale_desc(base + C::kA + t * 512));
          copy_scales(t_sb + 4 * t, scale_desc(sc + t * kTTile));
        }
        const uint64_t da = smem_desc_sw128(base), db = smem_desc_sw128(tok);
        const int steps = min(4, (p.K - kb * 256) / 64);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (k >= steps) break;
          const int t = kFmt == kMx ? k >> 1 : k;
          const uint32_t id = kFmt == kMx ? 2u * (k & 1) : 0u;
          mma_e2m1<kFmt>(tmem, da + 2 * k, db + 2 * k, idesc | (id << 4) | (id << 29), t_sa + 4 * t, t_sb + 4 * t, (kb != ka || k != 0) ? 1u : 0u);
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
    const int row = warp * 32 + lane, n = tb * 128 + row;  // this thread's weight row
    const int nc = min(n, p.N - 1);
    const float ws = __ldg(p.wrow + nc), bs = __ldg(p.bias + nc);
    // The rotation's blocks that this CTA's channels c0 .. c1 - 1 touch begin at `start`.
    const int c0 = 256 * ka, c1 = min(p.K, 256 * kz), b = 1 << p.log_b;
    const int start = c0 & ~(b - 1), end = min(p.K, (c1 + b - 1) & ~(b - 1));
    const int token = static_cast<int>(threadIdx.x) / p.threads, j = static_cast<int>(threadIdx.x) - token * p.threads;
    const bool there = token < p.M && start + j * 32 < end;
    const uint32_t own = smem_u32(lines) + static_cast<uint32_t>(token * p.threads * 128);
    griddep_wait();  // x comes from the previous kernel, which may still read y
    const T* const src = static_cast<const T*>(p.x) + static_cast<size_t>(token) * p.K + start;
    float2 v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = make_float2(0.0f, 0.0f);
    if (p.log_b <= 5) {
      load_rotated<kPlain, T>(p, src, j, there, own, v);
    } else if (p.log_b <= 7) {
      load_rotated<kFour, T>(p, src, j, there, own, v);
    } else if (p.log_b == 8) {
      load_rotated<8, T>(p, src, j, there, own, v);
    } else if (p.log_b == 9) {
      load_rotated<9, T>(p, src, j, there, own, v);
    } else if (p.log_b == 10) {
      load_rotated<10, T>(p, src, j, there, own, v);
    } else if (p.log_b == 11) {
      load_rotated<11, T>(p, src, j, there, own, v);
    } else {
      load_rotated<12, T>(p, src, j, there, own, v);
    }
    float top[2];
    magnitudes(v, top);
    if (kSplit > 1) cluster_wait();  // every CTA's barriers exist
    bool ok = true;
    float delta = 1.0f;
    if constexpr (kFmt == kNv) {
      if (p.step != nullptr) {
        delta = *p.step;
      } else {
        const uint32_t m = __reduce_max_sync(0xffffffffu, __float_as_uint(rq::max_nan(top[0], top[1])));
        if (lane == 0) s_warps[warp] = __uint_as_float(m);
        work_sync();
        auto of_row = [&](int t) {  // the largest of token t's warps (bit patterns order like the numbers, NaN above all)
          uint32_t w = 0;
          for (int i = t * p.threads / 32; i < (t + 1) * p.threads / 32 && i < kTWorkWarps; ++i) w = max(w, __float_as_uint(s_warps[i]));
          return __uint_as_float(w);
        };
        float most;
        if constexpr (kSplit > 1) {
          if (threadIdx.x < kSplit && *const_cast<volatile int*>(&g_debug_hold_loads) == 0)
            st_async_v4(mapa_shared(smem_u32(&s_peers[rank][0]), threadIdx.x), make_float4(of_row(0), of_row(1), of_row(2), of_row(3)),
                        mapa_shared(smem_u32(&bar_most), threadIdx.x));
          __syncwarp();
          ok = __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&bar_most), 0));
          uint32_t w = 0;
#pragma unroll
          for (int q = 0; q < kSplit; ++q) w = max(w, __float_as_uint(s_peers[q][min(token, kTokens - 1)]));
          most = __uint_as_float(w);
        } else {
          most = of_row(min(token, kTokens - 1));
        }
        delta = row_scale(most);
      }
      if (j == 0 && token < p.M) s_delta[token] = delta;
    }
    uint32_t code[4], bytes;
    if constexpr (kFmt == kMx) {
      bytes = encode_mx(v, top, code);
    } else {
      bytes = encode_nv(v, top, delta, code);
    }
    const int c = start + j * 32;
    if (there && c >= c0 && c < c1) {
      const int kb = c / 256 - ka, piece = c / 32 % 8;
      *reinterpret_cast<uint4*>(operand + kb * kTOperand + token * 128 + ((piece ^ token) << 4)) = make_uint4(code[0], code[1], code[2], code[3]);
      if constexpr (kFmt == kMx) {
        scales[(kb * C::kTiles + (piece >> 2)) * kTTile + token * 16 + (piece & 3)] = static_cast<uint8_t>(bytes);
      } else {
        *reinterpret_cast<uint16_t*>(scales + (kb * C::kTiles + (piece >> 1)) * kTTile + token * 16 + 2 * (piece & 1)) = static_cast<uint16_t>(bytes);
      }
    }
    if (!ok && lane == 0) *const_cast<volatile int*>(&s_abort) = 1;
    fence_proxy_async_smem();  // the tensor cores read them
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bar_tokens));
    work_sync();  // (for s_delta)

    bool done = __all_sync(0xffffffffu, mbar_wait(smem_u32(&bar_done), 0) && *const_cast<volatile int*>(&s_abort) == 0);
    __syncwarp();
    tc_fence_after();
    uint32_t r[4];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(tmem + (static_cast<uint32_t>(warp * 32) << 16)));
    tmem_ld_wait();
    float4 sum = make_float4(__uint_as_float(r[0]), __uint_as_float(r[1]), __uint_as_float(r[2]), __uint_as_float(r[3]));
    if constexpr (kSplit > 1) {  // the first CTA adds the parts, in the order of K
      if (rank != 0) {
        if (done) st_async_v4(mapa_shared(smem_u32(recv) + static_cast<uint32_t>((rank * 128 + row) * 16), 0), sum, mapa_shared(smem_u32(&bar_recv), 0));
        done = false;
      } else if (done) {
        done = __all_sync(0xffffffffu, mbar_wait_cluster(smem_u32(&bar_recv), 0));
        const float4 first = sum;
        sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int q = 0; q < kSplit; ++q) {
          const float4 a = q == 0 ? first : *reinterpret_cast<const float4*>(recv + (q * 128 + row) * 16);
          sum = make_float4(sum.x + a.x, sum.y + a.y, sum.z + a.z, sum.w + a.w);
        }
      }
    }
    const int ldy = p.gated ? p.N / 2 : p.N;
    T* const y = static_cast<T*>(p.y) + (p.gated ? tb * 64 + warp * 16 + (lane & 15) : n);
    const bool store = done && (p.gated ? lane < 16 : n < p.N);
#pragma unroll
    for (int m = 0; m < kTokens; ++m) {
      const float xs = kFmt == kMx ? 1.0f : s_delta[min(m, p.M - 1)];
      float a = fmaf(m == 0 ? sum.x : m == 1 ? sum.y : m == 2 ? sum.z : sum.w, xs * ws, bs);
      const float up = __shfl_down_sync(0xffffffffu, a, 16);
      if (p.gated) a = gelu_fast(a) * up;
      if (store && m < p.M) {
        const uint32_t h = pack2<T>(a, 0.0f);
        *reinterpret_cast<uint16_t*>(y + static_cast<size_t>(m) * ldy) = static_cast<uint16_t>(h);
      }
    }
  }
  if (kSplit > 1 && warp >= kTWorkWarps) cluster_wait();
  tc_fence_before();
  __syncthreads();
  if (kSplit > 1) cluster_sync();  // no CTA leaves while another may still send to it (after a wait ran out)
  tc_fence_after();
  if (warp == kTMma) tmem_dealloc<C::kTmem>(tmem);
}

template <int kSplit, int kFmt, typename T>
cudaError_t launch_token(const Fp4GemmArgs& a, TokenParams p, bool* taken) {
  using C = TokenCfg<kFmt>;
  // Threads of a row, the same in every CTA, by the widest of the parts with the blocks that it touches.
  const int nkb = (a.K + 255) / 256, b = 1 << p.log_b;
  int widest = 0;
  for (int rank = 0; rank < kSplit; ++rank) {
    const int ka = nkb * rank / kSplit, kz = nkb * (rank + 1) / kSplit;
    const int c0 = 256 * ka, c1 = std::min(a.K, 256 * kz);
    widest = std::max(widest, std::min(a.K, (c1 + b - 1) / b * b) - c0 / b * b);
    p.most = std::max(p.most, kz - ka);
  }
  p.threads = (widest + 1023) / 1024 * 32;
  const int tiles = (a.N + 127) / 128;
  // One CTA an SM while all clusters run at once so (as at the launch of the split product), two, or no fused call.
  const int at_once = a.num_sms * (kSplit == 8 ? 12 : kSplit == 4 ? 15 : 16) / 16 / kSplit;
  if (a.M * p.threads > kTWorkWarps * 32 || tiles > 2 * at_once) return cudaSuccess;
  const int fixed = (p.most + 1) * kTOperand + p.most * C::kTiles * kTTile + 512 + (kSplit > 1 ? kSplit * 2048 : 0) + kTWorkWarps * 32 * 128 + 1024;
  p.stages = std::min(std::min(p.most, kTMaxStages), ((tiles <= at_once ? 220 : 110) * 1024 - fixed) / C::kStage);
  auto kern = fp4_token_kernel<kSplit, kFmt, T>;
  static std::atomic<unsigned long long> raised{0};
  cudaError_t e = raise_smem(reinterpret_cast<const void*>(kern), 220 * 1024, &raised);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles * kSplit));
  cfg.blockDim = dim3(kTThreads);
  // (at least 68 KB, for the reason at the launch of the split product)
  cfg.dynamicSmemBytes = std::max(static_cast<size_t>(fixed) + static_cast<size_t>(p.stages) * C::kStage, size_t{68} << 10);
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
  *taken = true;
  e = cudaLaunchKernelEx(&cfg, kern, weight_map(a, 0), weight_map(a, 1), p);
  return e != cudaSuccess ? e : cudaGetLastError();
}

template <int kFmt, typename T>
cudaError_t launch_split(const Fp4GemmArgs& a, const TokenParams& p, int split, bool* taken) {
  switch (split) {
    case 1: return launch_token<1, kFmt, T>(a, p, taken);
    case 2: return launch_token<2, kFmt, T>(a, p, taken);
    case 4: return launch_token<4, kFmt, T>(a, p, taken);
    case 8: return launch_token<8, kFmt, T>(a, p, taken);
    default: return cudaSuccess;
  }
}

}  // namespace

cudaError_t launch_fp4_token(const Fp4GemmArgs& a, const void* x, int log_b, float inv_sqrt_b, const float* step, bool* taken) {
  *taken = false;
  if (a.M > kTokens) return cudaSuccess;
  const int split = fp4_split(a);
  const TokenParams p = {x, step, a.wrow, a.bias, a.y, inv_sqrt_b, a.M, a.N, a.K, log_b, a.gated, 0, 0, 0};
  if (a.fmt == kMx) return a.ydt == 0 ? launch_split<kMx, __half>(a, p, split, taken) : launch_split<kMx, __nv_bfloat16>(a, p, split, taken);
  return a.ydt == 0 ? launch_split<kNv, __half>(a, p, split, taken) : launch_split<kNv, __nv_bfloat16>(a, p, split, taken);
}

cudaError_t read_and_clear_error_word_fp4_token(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess || *out == 0) return e;
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

cudaError_t set_debug_hooks_fp4_token(unsigned long long wait_limit_ns, int hold_loads) { return set_debug_hooks(wait_limit_ns, hold_loads); }

}  // namespace qvla
