// Softmax attention over packed prompts: o_i = sum_j p_ij v_j, p_ij = exp(scale q_i.k_j) / sum exp, in one pass over the keys
// with a running maximum and sum, on the tensor cores.
//
// A CTA takes kTiles tiles of 128 query rows of one key/value head and runs them over the keys in blocks of kBlock.  A tile's
// rows are tokens x the query heads that share the key/value head, so grouped heads fill a tile that one head's tokens would
// leave half empty, and read K and V once.  Per block and tile:
//   S = Q K^T        tcgen05, operands from shared memory (TMA, 128-byte swizzle), S in TMEM
//   P = exp2(S c - m), rounded to 16 bits, over S's own columns in TMEM: a thread a row, no exchange between threads
//   O += P V         tcgen05 with A = P from TMEM and B = V as it lies (MN-major), O in TMEM
// While a warpgroup works out one tile's P, the tensor cores run the other tile's products; with 256 channels O takes half of
// TMEM, so there is one tile with two S buffers instead, and its next S is made while P is worked out.
// The maximum that P is taken against moves only when a row's maximum has grown by more than 2^8 (numerator and denominator use
// the same one, and both types hold the p that result), so O is rarely read back to be rescaled.
//
// Where a launch would leave SMs idle, a cluster of CTAs shares a group of tiles: each takes a run of the key blocks, and their O,
// maxima and sums are joined through distributed shared memory.
//
// Keys that some row of the CTA does not see (the diagonal's blocks, a sequence's last block) need care on the value side, where
// 0 * NaN would spread: two warps zero the rows behind the sequence's end and take NaN and infinities out of such
// blocks; a row that does see one of those gets it back, exactly, when it is written out.
//
// Measured: 8192 causal tokens, 16 heads of 128 channels on 4, 174 us (1580 TFLOP/s, tensor pipe 65% active, up to 189 us under the power cap: the exponentials
// take as long as the products); 816 tokens, 8 heads of 256 on one, 15.3 us (a CTA's 13 blocks at 0.65 us, on 51 SMs); packed prompts of
// up to 1500 over 2000 keys, 14 heads of 64 on 2, 22.2 us (the longest CTA's 16 blocks at 1.2 us).
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <atomic>
#include <mutex>
#include <type_traits>

#include "griddep.cuh"
#include "kv4.cuh"

namespace qvla {
namespace {

// Test hook: nonzero makes the load warp issue no copy (see qvla_debug.h).
static __device__ int g_debug_hold_loads;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRowsPerTile = 128;
constexpr float kGrowth = 8.0f;  // log2 of what a row's maximum may grow by before its O is rescaled
// P is taken against a reference below the maximum in float16, so that p reaches up to 2^15 there: of a key far below the leading one
// 2^-32 of the leading one's weight is resolved, where 2^-25 would lose what hundreds of thousands of such keys add up to.
template <typename T>
constexpr float kLift = std::is_same<T, __half>::value ? 7.0f : 0.0f;  // log2
constexpr int kLeastKeys = 256;  // of a CTA where a cluster shares a sequence's, which then has at least kSplitKeys
constexpr int kSplitKeys = 1024;
constexpr int kWarpLoad = 0, kWarpMma = 1, kWarpGuard = 2, kGuardWarps = 2, kWarpSoftmax = 4;

template <int kDim>
struct Shape {
  static constexpr int kTiles = kDim == 256 ? 1 : 2;
  static constexpr int kBlock = kDim == 256 ? 64 : 128;
  // Stages: a load takes about 2000 cycles from the release of its stage, as long as a block's products, and V passes the guard too.
  static constexpr int kStagesK = kDim == 64 ? 4 : kDim == 128 ? 2 : 3, kStagesV = kDim == 64 ? 4 : kDim == 128 ? 3 : 4;
  static constexpr bool kQTmem = kDim == 256;                 // Q in TMEM beside S and O (there is room with one tile only)
  static constexpr int kThreads = 32 * (kWarpSoftmax + 4 * kTiles);
  static constexpr int kQBytes = kQTmem ? 0 : kRowsPerTile * kDim * 2;  // one tile in shared memory
  static constexpr int kKvBytes = kBlock * kDim * 2;          // one block of K or V
  static constexpr int kStageAt = kStagesV - 2;               // with Q in TMEM: the stages of V that Q passes through
  static_assert(!kQTmem || 2 * kKvBytes == kRowsPerTile * kDim * 2, "a tile of Q takes two stages");
  static constexpr int kSmem = kTiles * kQBytes + (kStagesK + kStagesV) * kKvBytes + 1024;
  // a cluster's join: O in float32, rows kORow apart (which spreads a column over the banks), then maximum and sum of each row
  static constexpr int kORow = kDim + 4, kOBytes = kTiles * kRowsPerTile * kORow * 4;
  static_assert(kOBytes + kTiles * kRowsPerTile * 8 + 1024 <= kSmem, "the join fits over the operands");
  static constexpr int kOCol = 2 * kBlock, kQCol = kOCol + kTiles * kDim;  // TMEM: two S buffers, O of each tile, Q
};

struct PromptParams {
  const int32_t* cu_q;
  const int32_t* cu_k;
  void* o;
  const void* q;
  const void* v;
  int64_t q_stride, v_stride;
  int batch, total_q, total_k;
  int heads, kv_heads, group;  // group: query heads on a key/value head
  int chunk_heads, chunks;     // of them in one tile; tiles' head chunks
  int tokens;                  // tokens in one tile
  int causal;
  int split;                   // CTAs of a cluster, which share the keys of a group of tiles
  float c;                     // scale * log2(e)
};

struct Work {
  int q0, n, k0, keys;  // the sequence's first row, queries, first key and keys
  int token;            // first token of the CTA's first tile
  int kvh, head;        // key/value head; first query head
  int heads;            // query heads in the tile
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typename Pair<T>::V v = Pair<T>::from_float(a, b);
  return *reinterpret_cast<uint32_t*>(&v);
}

// Two 16-bit values of type T: the bits of those that are not finite, the others zero.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  constexpr uint32_t e = sizeof(T) == 2 && std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u;
  uint32_t m = 0;
  if ((w & e) == e) m |= 0xffffu;
  if (((w >> 16) & e) == e) m |= 0xffff0000u;
  return w & m;
}
template <typename T>
__device__ __forceinline__ bool any_not_finite(uint32_t w) {
  constexpr uint32_t e = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
  constexpr uint32_t one = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
  return (((w & e) + one) & 0x80008000u) != 0;  // an exponent of all ones carries into the sign's place
}

__device__ __forceinline__ float2 cluster_load2(uint32_t at) {  // of a CTA of the cluster (address from mapa_shared)
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ float4 cluster_load4(uint32_t at) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
  return v;
}
// 32 bytes of a row, in one access (a whole sector) where o's address allows: 0.3 to 0.5 us of a call against 16 bytes at a time.
__device__ __forceinline__ void store_row(void* dst, const uint32_t (&q)[8], bool wide) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst), "r"(q[0]), "r"(q[1]), "r"(q[2]), "r"(q[3]), "r"(q[4]),
                 "r"(q[5]), "r"(q[6]), "r"(q[7])
                 : "memory");
  } else {
    static_cast<uint4*>(dst)[0] = make_uint4(q[0], q[1], q[2], q[3]);
    static_cast<uint4*>(dst)[1] = make_uint4(q[4], q[5], q[6], q[7]);
  }
}
template <int kThreads>
__device__ __forceinline__ void softmax_sync() {  // the softmax warps meet
  asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
}

// Keys that query token i of its sequence sees.
__device__ __forceinline__ int seen_by(const Work& w, int causal, int i) {
  return causal ? max(0, min(w.keys, w.keys - w.n + i + 1)) : w.keys;
}

// The rows of a cluster's tiles that fall to CTA `rank` of it, four channels a thread: O, maxima and sums of up to kCtas CTAs
// are asked for at once, for kAhead places at a time (a row after the other took 8 us of a launch, this 3).
template <typename T, int kDim, int kCtas, int kAhead>
__device__ __forceinline__ void join(const PromptParams& p, const Work& w, const uint8_t* smem, int rank) {
  using C = Shape<kDim>;
  constexpr int kPer = kDim / 4, kRows = C::kTiles * kRowsPerTile;
  const int step = p.split * C::kThreads;
  uint32_t at[kCtas];
#pragma unroll
  for (int c = 0; c < kCtas; ++c) at[c] = mapa_shared(smem_u32(smem), static_cast<uint32_t>(min(c, p.split - 1)));
  for (int u0 = rank * C::kThreads + threadIdx.x; u0 < kRows * kPer; u0 += kAhead * step) {
    float2 ms[kAhead][kCtas];
    float4 v[kAhead][kCtas];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int u = min(u0 + a * step, kRows * kPer - 1), r = u / kPer, e = u % kPer * 4;
#pragma unroll
      for (int c = 0; c < kCtas; ++c) {
        ms[a][c] = cluster_load2(at[c] + C::kOBytes + r * 8);
        v[a][c] = cluster_load4(at[c] + static_cast<uint32_t>((r * C::kORow + e) * 4));
      }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int u = u0 + a * step, r = u / kPer, e = u % kPer * 4, t = r / kRowsPerTile, row = r % kRowsPerTile;
      const int token = w.token + t * p.tokens + row / p.chunk_heads, head = row % p.chunk_heads;
      bool live = u < kRows * kPer && row < p.tokens * p.chunk_heads && token < w.n && head < w.heads;
      float m = -INFINITY, sum = 0.0f, y[4] = {};
#pragma unroll
      for (int c = 0; c < kCtas; ++c) {
        if (c >= p.split || ms[a][c].y == 0.0f) continue;  // this CTA's keys are none that the row sees
        if (ms[a][c].y < 0.0f) live = false;               // a wait of that CTA ran out
        const float top = fmaxf(m, ms[a][c].x), keep = m == -INFINITY ? 0.0f : ex2(m - top), k = ex2(ms[a][c].x - top);
        m = top;
        sum = sum * keep + ms[a][c].y * k;
        y[0] = y[0] * keep + v[a][c].x * k;
        y[1] = y[1] * keep + v[a][c].y * k;
        y[2] = y[2] * keep + v[a][c].z * k;
        y[3] = y[3] * keep + v[a][c].w * k;
      }
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
      if (live)
        *reinterpret_cast<uint2*>(static_cast<T*>(p.o) + (static_cast<size_t>(w.q0 + token) * p.heads + w.head + head) * kDim + e) =
            make_uint2(pack2<T>(y[0] * inv, y[1] * inv), pack2<T>(y[2] * inv, y[3] * inv));
    }
  }
}

template <typename T, int kDim, bool kSplit>
__global__ void __launch_bounds__(Shape<kDim>::kThreads, 1)
    attention_prompt_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                            const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ PromptParams p) {
  using C = Shape<kDim>;
  constexpr int kTiles = C::kTiles, kBlock = C::kBlock, kStagesK = C::kStagesK, kStagesV = C::kStagesV;
  constexpr int kBoxes = kDim / 64;            // 64-channel boxes of a row
  constexpr int kQBox = kRowsPerTile * 128, kKvBox = kBlock * 128;
  constexpr int kBf16 = std::is_same<T, __half>::value ? 0 : 1;

  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bar_q[2], bar_kfull[kStagesK], bar_kempty[kStagesK], bar_vfull[kStagesV],
      bar_vok[kStagesV], bar_vempty[kStagesV], bar_s[2], bar_p[2][2], bar_o[2][2], bar_done;
  __shared__ uint32_t s_tmem;
  __shared__ int s_found, s_bad;
  __shared__ Work s_work;
  uint8_t* const smem = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
  uint8_t* const smem_k = smem + kTiles * C::kQBytes;
  uint8_t* const smem_v = smem_k + kStagesK * C::kKvBytes;

  const int warp = warp_index(), lane = threadIdx.x & 31;
  if (warp == kWarpMma) tmem_alloc<512>(smem_u32(&s_tmem));
  if (threadIdx.x == 32 * kWarpGuard) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bar_q[i]), C::kQTmem ? 4 : 1);
      mbar_init(smem_u32(&bar_s[i]), 1);
      mbar_init(smem_u32(&bar_p[i][0]), 4);
      mbar_init(smem_u32(&bar_p[i][1]), 4);
      mbar_init(smem_u32(&bar_o[i][0]), 1);
      mbar_init(smem_u32(&bar_o[i][1]), 1);
    }
    for (int i = 0; i < kStagesK; ++i) {
      mbar_init(smem_u32(&bar_kfull[i]), 1);
      mbar_init(smem_u32(&bar_kempty[i]), 1);
    }
    for (int i = 0; i < kStagesV; ++i) {
      mbar_init(smem_u32(&bar_vfull[i]), 1);
      mbar_init(smem_u32(&bar_vok[i]), kGuardWarps);
      mbar_init(smem_u32(&bar_vempty[i]), 1);
    }
    mbar_init(smem_u32(&bar_done), 1);
    mbar_init_fence();
    s_bad = 0;
  }
  if (threadIdx.x == 32 * kWarpSoftmax) {
    tma_prefetch_desc(&tmap_q);
    tma_prefetch_desc(&tmap_k);
    tma_prefetch_desc(&tmap_v);
  }
  griddep_wait();  // the offsets, q, k and v may come from the previous kernel, which may still read o
  if (warp == 0) {  // the sequence and tile of this CTA: 32 sequences a round, the last tiles of a sequence first
    const int per = p.kv_heads * p.chunks;
    const int cta = static_cast<int>(blockIdx.x) / (kSplit ? p.split : 1);
    int tile = cta / per;
    const int rest = cta % per;
    bool found = false;
    for (int b0 = 0; b0 < p.batch && !found; b0 += 32) {
      const int b = b0 + lane;
      int first = 0, n = 0, k_first = 0, k_next = 0;
      if (b < p.batch) {
        k_first = __ldg(p.cu_k + b);
        k_next = __ldg(p.cu_k + b + 1);
        first = min(max(__ldg(p.cu_q + b), 0), p.total_q);
        n = min(max(__ldg(p.cu_q + b + 1), first), p.total_q) - first;
      }
      const int tiles = (n + kTiles * p.tokens - 1) / (kTiles * p.tokens);
      int upto = tiles;
      for (int s = 1; s < 32; s *= 2) {
        const int o = __shfl_up_sync(0xffffffffu, upto, s);
        if (lane >= s) upto += o;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, tile < upto);
      if (hit == 0) {
        tile -= __shfl_sync(0xffffffffu, upto, 31);
        continue;
      }
      found = true;
      if (lane == __ffs(hit) - 1) {
        Work w;
        w.q0 = first;
        w.n = n;
        w.k0 = min(max(k_first, 0), p.total_k);
        w.keys = min(max(k_next, w.k0), p.total_k) - w.k0;
        w.token = (upto - 1 - tile) * kTiles * p.tokens;
        w.kvh = rest / p.chunks;
        w.head = w.kvh * p.group + (rest % p.chunks) * p.chunk_heads;
        w.heads = min(p.chunk_heads, (w.kvh + 1) * p.group - w.head);
        s_work = w;
      }
    }
    if (lane == 0) s_found = found ? 1 : 0;
  }
  if (warp == kWarpGuard) {
    OffsetsCheck of_q(p.cu_q, p.batch, p.total_q), of_k(p.cu_k, p.batch, p.total_k);
    of_q.finish();
    of_k.finish();
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  griddep_launch_dependents();
  const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);  // (values that the compiler knows to be the same in every lane)
  if (__shfl_sync(0xffffffffu, s_found, 0)) {
    Work w = s_work;
    // per tile: blocks to run, and the first of them that some row does not see whole
    int blocks[kTiles], partial[kTiles], most = 0, guard_from = 1 << 30;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      const int first = w.token + t * p.tokens, last = min(first + p.tokens, w.n) - 1;
      blocks[t] = first < w.n ? (seen_by(w, p.causal, last) + kBlock - 1) / kBlock : 0;
      blocks[t] = __shfl_sync(0xffffffffu, blocks[t], 0);
      most = max(most, blocks[t]);
    }
    if constexpr (kSplit) {  // this CTA's run of the blocks: from here on the keys begin with it
      const int run = (most + p.split - 1) / p.split, from = static_cast<int>(blockIdx.x) % p.split * run;
      w.k0 += from * kBlock;
      w.keys -= from * kBlock;
      most = max(0, min(run, most - from));
#pragma unroll
      for (int t = 0; t < kTiles; ++t) blocks[t] = max(0, min(blocks[t] - from, most));
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      partial[t] = seen_by(w, p.causal, w.token + t * p.tokens) / kBlock;
      if (blocks[t] > 0) guard_from = min(guard_from, partial[t]);
    }

    if (warp == kWarpLoad) {
      // ------------------------------------------------------------------ TMA
      if constexpr (kTiles == 2) setmaxnreg_dec<64>();
      bool ok = *const_cast<volatile int*>(&g_debug_hold_loads) == 0;
      if (ok && most > 0) {
        if (elect_one()) {
#pragma unroll
          for (int t = 0; t < kTiles; ++t) {
            if (C::kQTmem || blocks[t] == 0) continue;
            const uint32_t bar = smem_u32(&bar_q[t]);
            mbar_arrive_expect_tx(bar, static_cast<uint32_t>(p.chunk_heads * p.tokens * kDim * 2));
            for (int c = 0; c < kBoxes; ++c)
              tma_load_3d(smem_u32(smem + t * C::kQBytes + c * kQBox), &tmap_q, c * 64, w.head, w.q0 + w.token + t * p.tokens, bar);
          }
        }
        __syncwarp();
        auto fetch = [&](const CUtensorMap* map, uint8_t* stage, uint64_t* empty, uint64_t* full, int j, int stages) {
          if (!mbar_wait_warp(smem_u32(empty), (static_cast<uint32_t>(j / stages) & 1u) ^ 1u)) return false;
          if (elect_one()) {
            mbar_arrive_expect_tx(smem_u32(full), C::kKvBytes);
            for (int c = 0; c < kBoxes; ++c) tma_load_3d(smem_u32(stage + c * kKvBox), map, c * 64, w.kvh, w.k0 + j * kBlock, smem_u32(full));
          }
          __syncwarp();
          return true;
        };
        int ks = 0, vs = 0;  // blocks of K and of V asked for
        for (int j = 0; j < most; ++j) {
          const int k = j % kStagesK, v = j % kStagesV;
          if (!fetch(&tmap_k, smem_k + k * C::kKvBytes, &bar_kempty[k], &bar_kfull[k], j, kStagesK)) break;
          ks = j + 1;
          if (C::kQTmem && j == C::kStageAt && !mbar_wait_warp(smem_u32(&bar_q[0]), 0)) break;  // Q has left the stages
          if (!fetch(&tmap_v, smem_v + v * C::kKvBytes, &bar_vempty[v], &bar_vfull[v], j, kStagesV)) break;
          vs = j + 1;
        }
        // before leaving, let every load land
        for (int t = 0; t < kTiles; ++t)
          if (!C::kQTmem && blocks[t] > 0) mbar_wait_warp(smem_u32(&bar_q[t]), 0);
        for (int j = max(0, ks - kStagesK); j < ks; ++j) mbar_wait_warp(smem_u32(&bar_kfull[j % kStagesK]), static_cast<uint32_t>(j / kStagesK) & 1u);
        for (int j = max(0, vs - kStagesV); j < vs; ++j) mbar_wait_warp(smem_u32(&bar_vfull[j % kStagesV]), static_cast<uint32_t>(j / kStagesV) & 1u);
      }
      __syncwarp();
    } else if (warp == kWarpMma) {
      // ------------------------------------------------------------------ MMA
      if constexpr (kTiles == 2) setmaxnreg_dec<64>();
      constexpr uint32_t idesc_s = idesc_f16_f32(kBf16, kRowsPerTile, kBlock, 0);
      constexpr uint32_t idesc_o = idesc_f16_f32(kBf16, kRowsPerTile, kDim, 1);
      const uint32_t k_hi = static_cast<uint32_t>(smem_desc_sw128(0) >> 32), v_hi = static_cast<uint32_t>(smem_desc_sw128_mn(0, kKvBox) >> 32);
      const uint32_t q_lo = static_cast<uint32_t>(smem_desc_sw128(smem_u32(smem))), k_lo = static_cast<uint32_t>(smem_desc_sw128(smem_u32(smem_k))),
                     v_lo = static_cast<uint32_t>(smem_desc_sw128_mn(smem_u32(smem_v), kKvBox));  // addresses in units of 16 bytes
      bool ok = true;
      auto wait = [&](uint64_t* bar, int n) {  // completion n of a barrier
        ok = ok && mbar_wait_warp(smem_u32(bar), static_cast<uint32_t>(n) & 1u);
        return ok;
      };
      // S of tile t (buffer b) from K's stage s
      auto scores = [&](int t, int b, int s) {
        tc_fence_after();
        if (elect_one()) {
          const uint32_t d = tmem + static_cast<uint32_t>(b * kBlock);
          const uint32_t k = k_lo + static_cast<uint32_t>(s * (C::kKvBytes / 16)), q = q_lo + static_cast<uint32_t>(t * (C::kQBytes / 16));
          const uint32_t qt = tmem + static_cast<uint32_t>(C::kQCol);
#pragma unroll
          for (int i = 0; i < kDim / 16; ++i) {
            const uint32_t kk = k + (i / 4) * (kKvBox / 16) + (i % 4) * 2;
            if constexpr (C::kQTmem) {
              mma_f16_ts(d, qt + i * 8, kk, k_hi, idesc_s, i != 0);
            } else {
              mma_f16_ss(d, q + (i / 4) * (kQBox / 16) + (i % 4) * 2, k_hi, kk, k_hi, idesc_s, i != 0);
            }
          }
          mma_commit(smem_u32(&bar_s[b]));
        }
        __syncwarp();
      };
      // O of tile t += P (buffer b, for the n-th time) V (stage s), in halves as P comes
      auto values = [&](int t, int b, int n, int s, int j) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (!wait(&bar_p[b][half], n)) return;
          tc_fence_after();
          if (elect_one()) {
            const uint32_t d = tmem + static_cast<uint32_t>(C::kOCol + t * kDim), a = tmem + static_cast<uint32_t>(b * kBlock);
            const uint32_t v = v_lo + static_cast<uint32_t>(s * (C::kKvBytes / 16));
#pragma unroll
            for (int i = half * kBlock / 32; i < (half + 1) * kBlock / 32; ++i) mma_f16_ts(d, a + i * 8, v + i * 128, v_hi, idesc_o, !(j == 0 && i == 0));
            if (half == 1) mma_commit(smem_u32(&bar_o[t][j & 1]));
          }
          __syncwarp();
        }
      };
      auto release = [&](uint64_t* bar) {  // free once every product issued so far is done
        if (elect_one()) mma_commit(smem_u32(bar));
        __syncwarp();
      };
      if constexpr (kTiles == 2) {
        if (most > 0 && wait(&bar_kfull[0], 0)) {
          for (int t = 0; t < 2 && ok; ++t)
            if (blocks[t] > 0 && wait(&bar_q[t], 0)) scores(t, t, 0);
          if (ok) release(&bar_kempty[0]);
        }
        for (int j = 0; j < most && ok; ++j) {
          const int s = j % kStagesV, s1 = (j + 1) % kStagesK;
          if (!wait(&bar_vok[s], j / kStagesV)) break;
          if (j + 1 < most && !wait(&bar_kfull[s1], (j + 1) / kStagesK)) break;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (ok && j < blocks[t]) values(t, t, j, s, j);
            if (t == 1 && ok) release(&bar_vempty[s]);
            if (ok && j + 1 < blocks[t]) scores(t, t, s1);  // over P, which the product before it has read
          }
          if (ok && j + 1 < most) release(&bar_kempty[s1]);
        }
      } else {
        if (most > 0 && wait(&bar_kfull[0], 0) && wait(&bar_q[0], 0)) {
          scores(0, 0, 0);
          release(&bar_kempty[0]);
        }
        for (int j = 0; j < most && ok; ++j) {
          const int s = j % kStagesV, s1 = (j + 1) % kStagesK;
          if (j + 1 < most) {  // the next S, over the P that the product before last has read
            if (!wait(&bar_kfull[s1], (j + 1) / kStagesK)) break;
            scores(0, (j + 1) & 1, s1);
            release(&bar_kempty[s1]);
          }
          if (!wait(&bar_vok[s], j / kStagesV)) break;
          values(0, j & 1, j >> 1, s, j);
          if (ok) release(&bar_vempty[s]);
        }
      }
      if (elect_one()) {
        mma_commit(smem_u32(&bar_done));  // every product issued above has completed once this flips
        mbar_wait(smem_u32(&bar_done), 0);
      }
      __syncwarp();
    } else if (warp < kWarpSoftmax) {
      // ------------------------------------------------------------------ the guard of V
      if constexpr (kTiles == 2) setmaxnreg_dec<64>();
      for (int j = 0; j < most; ++j) {
        const int s = j % kStagesV;
        if (!mbar_wait_warp(smem_u32(&bar_vfull[s]), static_cast<uint32_t>(j / kStagesV) & 1u)) break;
        const int inside = min(kBlock, w.keys - j * kBlock);  // rows of the sequence; the rest is its neighbour's
        const bool look = p.causal && j >= guard_from;
        if (look || inside < kBlock) {
          bool bad = false;
#pragma unroll 4
          for (int i = (warp - kWarpGuard) * 32 + lane; i < kBoxes * kBlock * 8; i += 32 * kGuardWarps) {
            const int row = (i >> 3) % kBlock;
            uint4* at = reinterpret_cast<uint4*>(smem_v + s * C::kKvBytes + i * 16);
            if (row >= inside) {
              *at = make_uint4(0, 0, 0, 0);
            } else if (look) {
              const uint4 x = *at;
              if (any_not_finite<T>(x.x) | any_not_finite<T>(x.y) | any_not_finite<T>(x.z) | any_not_finite<T>(x.w)) {
                *at = make_uint4(x.x ^ not_finite<T>(x.x), x.y ^ not_finite<T>(x.y), x.z ^ not_finite<T>(x.z), x.w ^ not_finite<T>(x.w));
                bad = true;
              }
            }
          }
          if (bad) *const_cast<volatile int*>(&s_bad) = 1;
          fence_proxy_async_smem();
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar_vok[s]));
      }
      __syncwarp();
    } else {
      // ------------------------------------------------------------------ softmax and output: a thread a row
      if constexpr (kTiles == 2) setmaxnreg_inc<216>();  // 128 x 64 + 256 x 216 of the launch's 384 x 168
      const int t = kTiles == 2 ? (warp - kWarpSoftmax) >> 2 : 0;
      const int row = (warp & 3) * 32 + lane;
      const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
      const int token = w.token + t * p.tokens + row / p.chunk_heads, head = row % p.chunk_heads;
      const bool live = row < p.tokens * p.chunk_heads && token < w.n && head < w.heads;
      const int seen = live ? seen_by(w, p.causal, token) : w.keys;
      const int n = blocks[t], from = partial[t];
      const uint32_t o_at = tmem + lanes + static_cast<uint32_t>(C::kOCol + t * kDim);
      if (C::kQTmem && n > 0) {
        // Q to TMEM, two channels a column.  A warp's 32 rows pass through stages of V that are free yet: read by its own thread a
        // row touches another 128-byte line with every lane, which took 0.8 us more.  Pieces of 16 bytes, exchanged by the row's last
        // three bits.  (O written that way gained 0.4 to 0.8 us with full tiles, and cost 0.4 with few rows and, by its registers, 3% of
        // long calls with 128 channels.)
        uint8_t* const rows_at = smem_v + C::kStageAt * C::kKvBytes + (warp & 3) * 32 * kDim * 2;
        constexpr int kRowLanes = kDim / 8, kRowsAtOnce = 32 / kRowLanes;  // lanes of a row, rows of an access
        auto piece_at = [&](int r, int c) { return reinterpret_cast<uint4*>(rows_at + r * kDim * 2 + ((c ^ (r & 7)) * 16)); };
        const int64_t offset = live ? (w.q0 + token) * p.q_stride + (w.head + head) * kDim : -1;
#pragma unroll 16
        for (int r0 = 0; r0 < 32; r0 += kRowsAtOnce) {
          const int r = r0 + lane / kRowLanes, c = lane % kRowLanes;
          const int64_t from_row = __shfl_sync(0xffffffffu, offset, r);
          *piece_at(r, c) = from_row >= 0 ? __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + from_row + c * 8)) : make_uint4(0, 0, 0, 0);
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < kDim / 32; ++i) {
          uint32_t y[16];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint4 v = *piece_at(lane, i * 4 + e);
            y[4 * e] = v.x;
            y[4 * e + 1] = v.y;
            y[4 * e + 2] = v.z;
            y[4 * e + 3] = v.w;
          }
          tmem_st16(tmem + lanes + static_cast<uint32_t>(C::kQCol + i * 16), y);
        }
        tmem_st_wait();
        tc_fence_before();
        fence_proxy_async_smem();  // V comes to these stages next
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar_q[0]));
      }
      float m = -INFINITY, sum = 0.0f;
      bool ok = true;
      // Product j of this tile is in O.  Up to two products may be outstanding where this is asked (S of a block shows that of two
      // blocks before), so they complete on two barriers in turn: none can pass the phase that is waited for.
      auto o_has = [&](int j) { return mbar_wait_warp(smem_u32(&bar_o[t][j & 1]), static_cast<uint32_t>(j >> 1) & 1u); };
      for (int j = 0; j < n; ++j) {
        const int b = kTiles == 2 ? t : j & 1, visit = kTiles == 2 ? j : j >> 1;
        if (!mbar_wait_warp(smem_u32(&bar_s[b]), static_cast<uint32_t>(visit) & 1u)) { ok = false; break; }
        tc_fence_after();
        const uint32_t s_at = tmem + lanes + static_cast<uint32_t>(b * kBlock);
        uint32_t x[kBlock / 32][32];
#pragma unroll
        for (int i = 0; i < kBlock / 32; ++i) tmem_ld32(s_at + i * 32, x[i]);
        tmem_ld_wait();
        if (j >= from) {  // some row of the tile does not see all of this block
          const int left = seen - j * kBlock;
#pragma unroll
          for (int i = 0; i < kBlock; ++i)
            if (i >= left) x[i / 32][i % 32] = __float_as_uint(-INFINITY);
        }
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < kBlock; ++i) top = fmaxf(top, __uint_as_float(x[i / 32][i % 32]));
        top *= p.c;
        const bool grown = top > m + kGrowth || (m == -INFINITY && top > -INFINITY);
        if (__any_sync(0xffffffffu, grown)) {
          const float keep = grown ? ex2(m - top) : 1.0f;
          if (grown) m = top;
          sum *= keep;
          if (j > 0) {
            // the product of block j - 1 has to be in O
            if (!o_has(j - 1)) { ok = false; break; }
            tc_fence_after();
#pragma unroll 1
            for (int i = 0; i < kDim / 32; ++i) {
              uint32_t y[32];
              tmem_ld32(o_at + i * 32, y);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) y[e] = __float_as_uint(__uint_as_float(y[e]) * keep);
              tmem_st32(o_at + i * 32, y);
            }
            tmem_st_wait();
          }
        }
        const float ref = m == -INFINITY ? 0.0f : m - kLift<T>;  // (a row that has seen nothing yet)
        const float2 scale2 = make_float2(p.c, p.c), ref2 = make_float2(-ref, -ref);
        float2 part[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
        for (int i = 0; i < kBlock / 32; ++i) {
          uint32_t y[16];
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 d = fma2(make_float2(__uint_as_float(x[i][e]), __uint_as_float(x[i][e + 1])), scale2, ref2);
            const float2 v = make_float2(ex2(d.x), ex2(d.y));
            part[e / 2 & 1] = add2(part[e / 2 & 1], v);
            y[e / 2] = pack2<T>(v.x, v.y);
          }
          tmem_st16(s_at + i * 16, y);
          if (i % (kBlock / 64) == kBlock / 64 - 1) {  // half of the block
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar_p[b][i / (kBlock / 64)]));
          }
        }
        part[0] = add2(part[0], part[1]);
        sum += part[0].x + part[0].y;
      }
      if (ok && n > 0) {
        ok = o_has(n - 1);
        tc_fence_after();
      }
      const bool bad = *const_cast<volatile int*>(&s_bad) != 0;
      const int seen_here = min(seen, most * kBlock);
      auto add_bad = [&](float (&y)[32], int i) {  // the NaN and infinities that the guard took out and this row sees
        for (int key = guard_from * kBlock; key < seen_here; ++key) {
          const T* src = static_cast<const T*>(p.v) + (w.k0 + key) * p.v_stride + w.kvh * kDim + i * 32;
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float x = static_cast<float>(src[e]);
            if (!(fabsf(x) < INFINITY)) y[e] += x;
          }
        }
      };
      if constexpr (kSplit) {
        // every product of the CTA is done once all its rows are here: O goes over the operands, for the cluster to read
        softmax_sync<128 * kTiles>();
        float* const dst = reinterpret_cast<float*>(smem) + (t * kRowsPerTile + row) * C::kORow;
        reinterpret_cast<float2*>(smem + C::kOBytes)[t * kRowsPerTile + row] = make_float2(m, n <= 0 ? 0.0f : ok ? sum : -1.0f);
        if (ok && n > 0) {
#pragma unroll 1
          for (int i = 0; i < kDim / 32; ++i) {
            uint32_t r[32];
            __syncwarp();  // (rows add back as many values as they see; a load of TMEM wants the warp together)
            tmem_ld32(o_at + i * 32, r);
            tmem_ld_wait();
            float y[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) y[e] = __uint_as_float(r[e]);
            if (bad && live) add_bad(y, i);
#pragma unroll
            for (int e = 0; e < 32; e += 4) *reinterpret_cast<float4*>(dst + i * 32 + e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
          }
        }
      } else if (ok) {
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const bool wide = (reinterpret_cast<uint64_t>(p.o) & 31) == 0;
        T* const dst = static_cast<T*>(p.o) + (static_cast<size_t>(w.q0 + token) * p.heads + w.head + head) * kDim;
#pragma unroll 2
        for (int i = 0; i < kDim / 32; ++i) {
          float y[32];
          uint32_t r[32];
          if (n > 0) {
            __syncwarp();
            tmem_ld32(o_at + i * 32, r);
            tmem_ld_wait();
          }
#pragma unroll
          for (int e = 0; e < 32; ++e) y[e] = n > 0 ? __uint_as_float(r[e]) * inv : 0.0f;
          if (bad && live) add_bad(y, i);
          if (live) {
#pragma unroll
            for (int e = 0; e < 32; e += 16) {
              uint32_t q[8];
#pragma unroll
              for (int c = 0; c < 8; ++c) q[c] = pack2<T>(y[e + 2 * c], y[e + 2 * c + 1]);
              store_row(dst + i * 32 + e, q, wide);
            }
          }
        }
      }
      tc_fence_before();
    }
    if constexpr (kSplit) {
      // ------------------------------------------------------------------ the cluster's join
      __syncwarp();
      cluster_sync();
      const int rank = static_cast<int>(blockIdx.x) % p.split;
      if (p.split == 2) join<T, kDim, 2, 4>(p, w, smem, rank);
      else if (p.split <= 4) join<T, kDim, 4, 2>(p, w, smem, rank);
      else join<T, kDim, 8, 1>(p, w, smem, rank);
      __syncwarp();
      cluster_sync();  // nobody leaves while its rows are being read
    }
  }
  __syncthreads();
  tc_fence_after();
  if (warp == kWarpMma) tmem_dealloc<512>(tmem);
}

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
  static std::once_flag once;
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

// Packed tokens of `heads` heads as 64 channels x box_heads x box_tokens, under the 128-byte swizzle.
cudaError_t make_tmap_heads(CUtensorMap* m, const void* base, int bf16, int dim, int heads, int tokens, int64_t stride, int box_heads,
                            int box_tokens) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dim), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(tokens)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(dim) * 2, static_cast<cuuint64_t>(stride) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_tokens)};
  const cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = enc(m, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box,
                   estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// Raise a kernel's dynamic shared-memory limit, once per kernel and device.  (A set of them could throw, through the C entry.)
template <typename T, int kDim, bool kSplit>
cudaError_t prepare_kernel() {
  static std::atomic<uint64_t> raised{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
  if (raised.load(std::memory_order_relaxed) & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(attention_prompt_kernel<T, kDim, kSplit>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<kDim>::kSmem);
  if (e == cudaSuccess) raised.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// Clusters of `size` CTAs that the current device holds at once (asked once a size and device); 0 if it cannot tell.
template <typename T, int kDim>
int resident_clusters(int size) {
  using C = Shape<kDim>;
  constexpr int kDevices = 32;
  static std::atomic<int> known[kDevices][9];  // count + 1
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= kDevices) return 0;
  const int seen = known[dev][size].load(std::memory_order_relaxed);
  if (seen > 0) return seen - 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(size));
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = static_cast<unsigned>(size);
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  auto kern = attention_prompt_kernel<T, kDim, true>;
  if (prepare_kernel<T, kDim, true>() != cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, kern, &cfg) != cudaSuccess) {
    cudaGetLastError();  // (plain launches do without)
    n = 0;
  }
  known[dev][size].store(n + 1, std::memory_order_relaxed);
  return n;
}

template <typename T, int kDim>
cudaError_t launch(const PromptArgs& a) {
  using C = Shape<kDim>;
  PromptParams p;
  p.cu_q = a.cu_q;
  p.cu_k = a.cu_k;
  p.o = a.o;
  p.q = a.q;
  p.v = a.v;
  p.q_stride = a.q_stride;
  p.v_stride = a.v_stride;
  p.batch = a.batch;
  p.total_q = a.total_q;
  p.total_k = a.total_k;
  p.heads = a.heads;
  p.kv_heads = a.kv_heads;
  p.group = a.heads / a.kv_heads;
  // more than 128 query heads on a key/value head: equal chunks of them, a token a tile
  p.chunks = (p.group + kRowsPerTile - 1) / kRowsPerTile;
  p.chunk_heads = (p.group + p.chunks - 1) / p.chunks;
  p.tokens = kRowsPerTile / p.chunk_heads;
  p.causal = a.causal;
  p.c = a.scale * kLog2e;
  // without keys nothing is loaded; the maps still need a valid base
  const int bf16 = std::is_same<T, __half>::value ? 0 : 1, keys = a.total_k > 0 ? a.total_k : 1;
  CUtensorMap tq = {}, tk = {}, tv = {};
  cudaError_t e = make_tmap_heads(&tq, a.q, bf16, kDim, a.heads, a.total_q, a.q_stride, p.chunk_heads, p.tokens);
  if (e == cudaSuccess) e = make_tmap_heads(&tk, a.total_k > 0 ? a.k : a.q, bf16, kDim, a.kv_heads, keys, a.k_stride, 1, C::kBlock);
  if (e == cudaSuccess) e = make_tmap_heads(&tv, a.total_k > 0 ? a.v : a.q, bf16, kDim, a.kv_heads, keys, a.v_stride, 1, C::kBlock);
  if (e != cudaSuccess) return e;
  // at most this many groups of tiles, however the tokens are spread over the sequences
  const int64_t per = static_cast<int64_t>(C::kTiles) * p.tokens;
  const int64_t groups = (a.total_q + static_cast<int64_t>(a.batch) * (per - 1)) / per;
  const int64_t ctas = groups * a.kv_heads * p.chunks;
  if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
  // Where CTAs would leave SMs idle and sequences of middling length have kSplitKeys keys, a cluster a group of tiles: as large as
  // the SMs hold at once, with at least kLeastKeys keys a CTA. Clusters against CTAs, us, 8 heads of 128 channels on one: 64 tokens
  // on 2000 keys 17.1 against 27.6, 1500 on 1500 20.1 against 23.0, but 816 on 816 16.8 against 15.8: the join takes 3 to 4.
  const int64_t middling = a.total_k / a.batch;
  int64_t split = middling < kSplitKeys ? 1 : a.num_sms / ctas;
  if (split > middling / kLeastKeys) split = middling / kLeastKeys;
  if (split > 8) split = 8;
  while (split > 1 && resident_clusters<T, kDim>(static_cast<int>(split)) < ctas) --split;
  p.split = split < 2 ? 1 : static_cast<int>(split);
  auto kern = p.split > 1 ? attention_prompt_kernel<T, kDim, true> : attention_prompt_kernel<T, kDim, false>;
  e = p.split > 1 ? prepare_kernel<T, kDim, true>() : prepare_kernel<T, kDim, false>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(ctas * p.split));
  cfg.blockDim = dim3(C::kThreads);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.split);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.split > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, kern, tq, tk, tv, p);
  if (e != cudaSuccess) return e;
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_prompt(const PromptArgs& a) {
  if (a.dt == 0)
    return a.head_dim == 64 ? launch<__half, 64>(a) : a.head_dim == 128 ? launch<__half, 128>(a) : launch<__half, 256>(a);
  return a.head_dim == 64 ? launch<__nv_bfloat16, 64>(a)
                          : a.head_dim == 128 ? launch<__nv_bfloat16, 128>(a) : launch<__nv_bfloat16, 256>(a);
}

cudaError_t read_and_clear_error_word_prompt(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess || *out == 0) return e;  // (cleared only where it is set: the check goes through every unit's word)
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

cudaError_t set_debug_hooks_prompt(unsigned long long wait_limit_ns, int hold_loads) {
  cudaError_t e = cudaDeviceSynchronize();
  if (e != cudaSuccess) return e;
  e = cudaMemcpyToSymbol(g_wait_limit_ns, &wait_limit_ns, sizeof(wait_limit_ns));
  if (e != cudaSuccess) return e;
  return cudaMemcpyToSymbol(g_debug_hold_loads, &hold_loads, sizeof(hold_loads));
}

}  // namespace qvla
