// Attention of a few query tokens over the 4-bit key/value cache:
//   s_j = scale Dk_j (q' . ck_j),   o = sum_j p_j Dv_j cv_j / sum_j p_j,   p_j = exp(s_j - max s)
// with codes ck, cv, scales Dk, Dv and, for a rotated cache, q' = q H / sqrt(D) and the output o H / sqrt(D).
//
// For single tokens the codes' bytes (D + 8 for a token and head) are the bound, for chunks the launch and the matrix
// instructions.  A warp takes 16 or 32 cached tokens at a time through a ring of its own in shared memory (16-byte cp.async, several
// steps ahead; loads into registers came no further ahead than one step) into the registers of mma.m16n8k16 fragments:
// the contraction over channels and the rows of O may be permuted at will, so a lane's share of a key is D / 8 contiguous
// bytes and of a value D / 16.  16-byte pieces are placed so that no read meets a bank conflict.
//   S^T = K Q^T      A = key codes (16 keys x 16 channels), B = queries (8 rows): grouped heads' single tokens fill 8 columns
//   O^T += V^T P^T   A = value codes (16 channels x 16 keys), B = P^T, from S^T's accumulators by an 8 x 8 transpose
// A value's code becomes float16 by one logic operation and one exact addition on two at a time.  A key's takes the logic
// operation alone: code + 8 in the low bits of a float16 is the subnormal (code + 8) 2^-24 (2^-20 from the nibble above, whose
// queries carry a factor 1/16), and 8 sum_c q'_c is taken from the row's scores.  (For values that offset would grow with
// the number of tokens and cost the sum its last bits.)
//   Dk_j multiplies the score, Dv_j the probability: p_j = exp2(s_j - r) is summed in float32, and w_j = p_j Dv_j is rounded to
// float16 for the second product.  The row's reference r follows the largest w, not the largest p, so a weight has float16's
// 11 bits whatever the scales' size; it moves when a w would pass 2^15 (or a p 2^96, where all scales are tiny).
//   A query row is multiplied by a power of two that brings its largest entry to [0.5, 1) before it is rounded to
// float16.  A query that is not rotated keeps its bits so, but for entries that become float16 subnormals: below 2^-14 of that
// power of two in even channels and 2^-10 in odd ones (which carry the factor 1/16), and then it is off by at most 2^-25 and 2^-21
// of it, which is as far as a score's float32 sums resolve with the codes' offset in them.  A rotated float16 query is taken in two
// parts, or its rounding would show beside a float16 output's (error 1.6 times that of float32 queries; beside a bfloat16
// output's it does not).
//
// The cached tokens of a sequence are split into chunks over CTAs (of kWarps warps, each with every kWarps-th step).  The device
// decides the chunks from the lengths it finds, so that a captured graph follows its lengths.  Two ways:
//   - a cluster of up to 8 CTAs a sequence, head and row tile, each with an equal part, whose results are joined through
//     distributed shared memory: one launch, for contexts short enough that the longest part does not outlast the rest;
//   - chunks of about equal length over all sequences, joined by a second kernel: long and short contexts of one call share
//     the SMs evenly.
//
// Measured: eight contexts of 32768 to 65536 tokens, 32 heads of 128 channels on 8, 100 us (5.0 TB/s of codes; issue 62%, DRAM
// 63%: a step's chain of products and exponentials on four warps a scheduler, and its 600 instructions); 23 contexts of 1 to 6001,
// 15.8 us, and 4 x 50 tokens over 866 with 8 heads of 256 on one, 18.0 us (a CTA's own chain: finding its chunk, pages, first codes,
// a few steps, joins); one token over 817, 8.6 us.
#include <cuda_runtime.h>

#include <atomic>
#include <cfloat>
#include <type_traits>

#include "griddep.cuh"
#include "kv4.cuh"

namespace qvla {
namespace {

constexpr int kWarps = 4;
constexpr float kLog2e = 1.4426950408889634f;
// What a reference lets through.  It is set 2^7 below the largest weight, so that weights use float16's range up to 2^15 and 2^-32 of the
// largest one is resolved; with 2^-25, hundreds of thousands of tokens far below a leading one would not add up.
constexpr float kMostWeight = 0x1p15f, kMostP = 0x1p96f, kLift = 7.0f;  // (kLift: log2)
constexpr float kLeastScale = -81.0f;                     // log2 of the scale below which p bounds the reference
constexpr int kTile = 16;        // cached tokens of a matrix instruction

struct Kv4Params {
  Kv4AttentionArgs a;
  int group;         // query heads on a key/value head
  int rows;          // query rows of a CTA (8 or 16): (token, head of the group), tokens outer
  int per;           // CTAs of a chunk: kv_heads x row tiles for max_q queries
  int row_tiles;
  int target;        // CTAs to aim for, those that the SMs hold at once; 0: one chunk a sequence
  int most_target;   // the same where there is work enough to even out over several waves
  int ctas;          // at most this many: most_target and a CTA for the remainder of every sequence
  int cluster;       // CTAs of a cluster that share a sequence's keys; 0: chunks by length
  float* part;       // [ctas][rows][head_dim + 2]: sums over the values, then the reference and sum p
};
constexpr int kLeastChunk = kTile * kWarps;
// CTAs that an SM holds (their registers allow it), and how often to fill the SMs: single tokens' contexts differ in length.
constexpr int ctas_per_sm(int dim, int rows) { return rows == 8 ? (dim == 256 ? 3 : 4) : (dim == 64 ? 3 : 2); }
constexpr int kWaves8 = 2, kWaves16 = 1;
constexpr int kLongChunk = 1024;  // tokens of a CTA above which more waves pay (a CTA's own start and end take about 5 us)
constexpr int cluster_len(int dim) { return dim == 256 ? 2048 : 4096; }  // longest context that clusters share

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Of a word of 8 codes: (code + 8) 2^-24 at nibbles 0 and 4, (code + 8) 2^-20 at 1 and 5.
struct OffsetBits {
  uint32_t low = hidden_constant<0x00080008u>(), high = hidden_constant<0x00800080u>();
  __device__ __forceinline__ uint32_t offsets_04(uint32_t w) const { return and_xor(w, 0x000f000fu, low); }
  __device__ __forceinline__ uint32_t offsets_15(uint32_t w) const { return and_xor(w, 0x00f000f0u, high); }
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

template <int kWords>
__device__ __forceinline__ void read_words(uint32_t (&r)[kWords], uint32_t at) {
  if constexpr (kWords == 1) {
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(r[0]) : "r"(at));
  } else if constexpr (kWords == 2) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(at));
  } else {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
  }
}
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// Two floats of a CTA of the cluster (address from mapa_shared).
__device__ __forceinline__ float2 cluster_load2(uint32_t at) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kBut>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kBut) : "memory");
}

// One sequence's first query row, queries and cached tokens.
struct Sequence {
  int q0, n, len;
};
template <bool kL2 = false>
__device__ __forceinline__ Sequence load_sequence(const Kv4AttentionArgs& a, int b) {
  Sequence s;
  s.q0 = min(max(read_index<kL2>(a.cu_q + b), 0), a.total_q);
  s.n = min(max(read_index<kL2>(a.cu_q + b + 1), s.q0), a.total_q) - s.q0;
  s.len = read_index<kL2>(a.kv_len + b);
  return s;
}
// False where it exceeds the launch's bounds and is to be skipped.
__device__ __forceinline__ bool usable(const Kv4AttentionArgs& a, const Sequence& s) { return s.n <= a.max_q && s.len >= 0 && s.len <= a.max_len; }
// Cached tokens that query token i sees.
__device__ __forceinline__ int seen_by(const Sequence& s, int causal, int i) { return causal ? max(0, s.len - s.n + i + 1) : s.len; }

// The split: every sequence gets one chunk for each started `length` tokens, of equal size.  The kernel that attends and the one that
// joins both work it out, and a part placed elsewhere by one of them would be lost.  So every operation here has its rounding
// stated (__fmul_rn, __fadd_rn; __fdividef is one approximate division of PTX), and the compiler may not contract products
// and sums in one kernel and not in the other.
__device__ __forceinline__ int usable_length(const Kv4AttentionArgs& a, int len) { return min(max(len, 0), a.max_len); }
// (a quotient in float, never above the exact one)
__device__ __forceinline__ int chunks_of(int len, float per_length) { return 1 + static_cast<int>(__fmul_rn(static_cast<float>(len - 1), per_length)); }
__device__ __forceinline__ int chunk_size(int len, int chunks) {
  const unsigned even = (static_cast<unsigned>(len) + chunks - 1u) / static_cast<unsigned>(chunks);
  return static_cast<int>((even + kLeastChunk - 1) / kLeastChunk * kLeastChunk);
}
// 1 / length, the same in every CTA of both kernels; `len`: of sequence `lane` (0 where there is none), loaded already.
template <bool kL2 = false>
__device__ __forceinline__ float split_of(const Kv4Params& p, int len) {
  if (p.target == 0) return 0.0f;
  constexpr float kLess = 1.0f - 0x1p-20f;  // more than the roundings of a quotient can add
  const int lane = static_cast<int>(threadIdx.x & 31);
  uint32_t low = len & 0xffff, high = len >> 16;  // (65535 sequences of up to 2^30 tokens)
  for (int b = 32 + lane; b < p.a.batch; b += 32) {
    const int n = usable_length(p.a, read_index<kL2>(p.a.kv_len + b));
    low += n & 0xffff;
    high += n >> 16;
  }
  low = __reduce_add_sync(0xffffffffu, low);
  high = __reduce_add_sync(0xffffffffu, high);
  const float all = __fmul_rn(__fadd_rn(__fmul_rn(static_cast<float>(high), 65536.0f), static_cast<float>(low)), static_cast<float>(p.per));
  const float target = static_cast<float>(all > __fmul_rn(static_cast<float>(p.target), kLongChunk) ? p.most_target : p.target);
  auto inverse = [](float length) {  // of the length in whole kLeastChunk
    return __fdividef(kLess, __fmul_rn(fmaxf(1.0f, ceilf(__fmul_rn(length, 1.0f / kLeastChunk))), kLeastChunk));
  };
  float length = __fdividef(all, __fmul_rn(target, kLess)), per_length = inverse(length);
  // the remainders of the sequences come on top: lengthen the chunks until all fit the target, so that no CTA is left for a wave
  // of its own (a few tries, where the lengths are at hand)
  for (int i = 0; i < 4 && p.a.batch <= 32; ++i) {
    const float ctas = static_cast<float>(__reduce_add_sync(0xffffffffu, lane < p.a.batch ? chunks_of(len, per_length) : 0) * p.per);
    if (ctas <= target) break;
    length = __fadd_rn(__fdividef(ctas, __fmul_rn(target, per_length)), 1.0f);
    per_length = inverse(length);
  }
  return per_length;
}

template <int kDim, int kTiles, bool kSplitQ>
struct Cfg {
  static constexpr int kRows = 8 * kTiles;
  static constexpr int kTeam = kDim / 8;                   // lanes that hold a head, 8 channels each
  static constexpr int kQBytes = kRows * kDim * (kSplitQ ? 4 : 2);  // the staged queries, in the order of the fragments
  // A step of 32 tokens halves the work around the matrix instructions, for as many registers as single tokens leave free.
  static constexpr int kParts = kTiles == 1 && kDim < 256 ? 2 : 1;
  static constexpr int kStep = kTile * kParts;              // cached tokens a warp takes at once
  static constexpr int kStages = kDim == 256 || kParts == 2 ? 3 : 4;  // steps of a warp's ring
  static constexpr int kPartBytes = kTile * (kDim + 8);    // key codes, value codes, key scales, value scales
  static constexpr int kStepBytes = kParts * kPartBytes;
  static constexpr int kRing = kWarps * kStages * kStepBytes;
  // The warps' sums, over the ring at the end: an eighth of a row's channels (a lane's) every kEighth floats, rows kJoinRow
  // apart, which spreads the fragments' stores over the banks.
  static constexpr int kEighth = kDim / 8 + 2, kJoinRow = 8 * kEighth + 4;
  static constexpr int kJoin = kWarps * kRows * kJoinRow * 4;
  static constexpr int kPart = kRows * (kDim + 2) * 4;      // this CTA's result, for its cluster
  static constexpr int kSmem = (kRing > kJoin + kPart ? kRing : kJoin + kPart) + kQBytes;
};

template <typename T, int kDim, int kTiles, bool kSplitQ>
__global__ void __launch_bounds__(32 * kWarps, ctas_per_sm(kDim, 8 * kTiles)) attention_kv4_kernel(const __grid_constant__ Kv4Params p) {
  using C = Cfg<kDim, kTiles, kSplitQ>;
  constexpr int kRows = C::kRows, kTeam = C::kTeam, kTeams = 32 * kWarps / kTeam, kStages = C::kStages, kParts = C::kParts,
                kStep = C::kStep;
  constexpr int kRow = kDim / 2;  // bytes of a token's codes
  constexpr bool kQInRegs = kTiles * kDim <= 256;
  const Kv4AttentionArgs& a = p.a;
  extern __shared__ __align__(128) uint8_t s_raw[];
  // Queries as B fragments: of row tile n, word w (8 channels of each lane's quarter) and half c of it, a lane's two registers.
  uint2* const q_at = reinterpret_cast<uint2*>(s_raw);
  constexpr int kRest = kRows * kDim / 4;  // where what float16 leaves of the queries lies
  auto q_index = [](int n, int w, int c) { return ((n * (kDim / 32) + w) * 2 + c) * 32; };
  uint8_t* const s_ring = s_raw + C::kQBytes;                                 // [kWarps][kStages][kStepBytes]
  float* const s_o = reinterpret_cast<float*>(s_ring);                        // [kWarps][kRows][kJoinRow] at the end
  float* const s_part = reinterpret_cast<float*>(s_ring + C::kJoin);          // [kRows][kDim + 2]
  static_assert(C::kQBytes % 128 == 0, "the ring's pieces are placed by 128-byte lines");
  __shared__ float s_f[kRows], s_sum[kRows], s_m[kWarps][kRows], s_l[kWarps][kRows];
  __shared__ int s_end[kWarps][kStages][kParts];  // first token that nobody may use

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  griddep_wait();  // the queries, lengths and the cache may come from the previous kernel, which may still read o
  griddep_launch_dependents();
  OffsetsCheck offsets(a.cu_q, a.batch, a.total_q);
  // this CTA's sequence b, chunk ch of it, key/value head and row tile
  const int unit = p.cluster ? static_cast<int>(blockIdx.x) / p.cluster : static_cast<int>(blockIdx.x);
  const int rest = unit % p.per, tile = rest % p.row_tiles, kvh = rest / p.row_tiles;
  int ch = unit / p.per, b = -1, chunk = 0;
  Sequence seq = {0, 0, 0};  // of sequence b0 + lane, then of b
  if (p.cluster) {
    b = ch;
    ch = static_cast<int>(blockIdx.x) % p.cluster;  // (the CTA's rank)
    seq = load_sequence(a, b);
    chunk = max(kLeastChunk, chunk_size(usable_length(a, seq.len), p.cluster));
  } else {
    if (lane < a.batch) seq = load_sequence(a, lane);
    const float per_length = split_of(p, usable_length(a, seq.len));
    for (int b0 = 0; b0 < a.batch && b < 0; b0 += 32) {
      if (b0 > 0 && b0 + lane < a.batch) seq = load_sequence(a, b0 + lane);
      const int len = usable_length(a, seq.len), n = b0 + lane < a.batch ? chunks_of(len, per_length) : 0;
      int upto = n;
#pragma unroll
      for (int h = 1; h < 32; h *= 2) {
        const int o = __shfl_up_sync(0xffffffffu, upto, h);
        if (lane >= h) upto += o;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, ch < upto);
      const int from = hit ? __ffs(hit) - 1 : 31;
      ch -= __shfl_sync(0xffffffffu, hit ? upto - n : upto, from);
      if (hit == 0) continue;
      b = b0 + from;
      chunk = __shfl_sync(0xffffffffu, chunk_size(len, max(n, 1)), from);
      seq = {__shfl_sync(0xffffffffu, seq.q0, from), __shfl_sync(0xffffffffu, seq.n, from), __shfl_sync(0xffffffffu, seq.len, from)};
    }
  }
  if (warp == 0) offsets.finish();
  if (b < 0) return;
  if (!usable(a, seq)) {
    if (threadIdx.x == 0) report_index();
    return;
  }
  const int row0 = tile * kRows, rows = min(kRows, seq.n * p.group - row0);
  if (rows <= 0) return;
  const int most = seen_by(seq, a.causal, (row0 + rows - 1) / p.group);  // tokens that the last row sees
  const int k0 = ch * chunk, k1 = min(most, k0 + chunk);
  if (ch > 0 && k0 >= most && !p.cluster) return;  // (the CTAs of a cluster stay together)

  // ---- the queries and the first cached tokens are asked for together
  constexpr int kQRounds = (kRows + kTeams - 1) / kTeams;
  uint4 q_raw[kQRounds];
  const int tl = threadIdx.x % kTeam, q_low = tl * (a.pool.rotate ? 4 : 8), q_high = a.pool.rotate ? kDim / 2 + q_low : q_low + 4;
#pragma unroll
  for (int i = 0; i < kQRounds; ++i) {
    const int r = i * kTeams + static_cast<int>(threadIdx.x) / kTeam;
    const int token = seq.q0 + (row0 + r) / p.group, head = kvh * p.group + (row0 + r) % p.group;
    const T* const src = static_cast<const T*>(a.q) + token * a.q_stride + head * kDim;
    const uint2 low = r < rows ? __ldg(reinterpret_cast<const uint2*>(src + q_low)) : make_uint2(0, 0);
    const uint2 high = r < rows ? __ldg(reinterpret_cast<const uint2*>(src + q_high)) : make_uint2(0, 0);
    q_raw[i] = make_uint4(low.x, low.y, high.x, high.y);
  }
  const uint32_t block = (kDim + 8u) << a.pool.log_page, stride = block * a.pool.kv_heads;  // of a head's page, of a page
  const uint8_t* const base = a.pool.base + static_cast<uint64_t>(kvh) * block;
  const int plane = kRow << a.pool.log_page, slots = (1 << a.pool.log_page) - 1;
  const int steps = k1 > k0 + kStep * warp ? (k1 - k0 - kStep * warp + kStep * kWarps - 1) / (kStep * kWarps) : 0;
  // Places in the ring.  Keys: as they are, with 256 channels a row's 16-byte pieces exchanged in pairs in odd rows.  Values: a
  // 128-byte line's pieces c at c ^ 2 x, x counting pairs of rows (with 64 channels groups of four).
  const uint32_t ring = smem_u32(s_ring) + warp * kStages * C::kStepBytes;
  auto key_piece = [](int row, int c) { return kDim == 256 ? c ^ (row & 1) : c; };
  auto value_place = [](int row, int c) {  // of piece c of a row's kRow / 16
    const int at = row * (kRow / 16) + c, x = kDim == 64 ? (row >> 2) & 1 : (row >> 1) & 3;
    return 16 * ((at & ~7) | ((at & 7) ^ (2 * x)));
  };
  const int row_first = lane / (kRow / 16), piece = lane % (kRow / 16);
  const uint32_t k_put = row_first * kRow + 16 * key_piece(row_first, piece), v_put = 8 * kDim + value_place(row_first, piece);
  const uint32_t s_put = 16 * kDim + (lane & 7) * 16;
  const uint32_t s_src = 2 * plane + (((lane >> 2) & 1) << a.pool.log_page) * 4 + (lane & 3) * 16;
  constexpr int kFetch = 32 / kParts;  // steps whose pages are fetched at once, one a lane
  int pages = 0;
  uint32_t missing = 0;  // those of them that are not there
  auto load = [&](int i, int slot) {
    if (i < steps) {
      if (i % kFetch == 0) {
        const int at = k0 + kStep * (warp + kWarps * (i + lane / kParts)) + kTile * (lane % kParts);
        pages = at < k1 ? __ldg(a.table + static_cast<size_t>(b) * a.max_pages + (at >> a.pool.log_page)) : 0;
        const bool none = static_cast<uint32_t>(pages) >= static_cast<uint32_t>(a.pool.num_pages);
        missing = __ballot_sync(0xffffffffu, none);
        if (none) {
          report_index();
          pages = 0;
        }
      }
      const int at = k0 + kStep * (warp + kWarps * i);
      uint32_t to = ring + slot * C::kStepBytes;
#pragma unroll
      for (int h = 0; h < kParts; ++h, to += C::kPartBytes) {
        const int from = i % kFetch * kParts + h;
        const int page = __shfl_sync(0xffffffffu, pages, from);
        const int in = (at + kTile * h) & slots;
        const uint8_t* const src = base + static_cast<uint64_t>(static_cast<uint32_t>(page)) * stride;
        const uint8_t* const codes = src + in * kRow + lane * 16;
#pragma unroll
        for (int c = 0; c < kDim / 64; ++c) {
          // (256 channels: the next four rows, whose pieces are placed two pairs of rows on)
          copy16(to + (k_put + c * 512), codes + c * 512);
          copy16(to + ((kDim == 256 && (c & 1) ? v_put ^ 64 : v_put) + c * 512), codes + plane + c * 512);
        }
        if (lane < 8) copy16(to + s_put, src + s_src + in * 4);
        if (lane == 0) s_end[warp][slot][h] = missing >> from & 1 ? 0 : k1;
      }
    }
    copy_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) load(i, i);

  // ---- queries: rotated, scaled by a power of two, float16, in the order of the codes' pairs (all rounds at once: one after the
  // other their shuffles' latencies took 2 us with 16 rows of 256 channels)
  float y[kQRounds][8], top[kQRounds], sums[kQRounds];  // sums: of the rounded queries
#pragma unroll
  for (int i = 0; i < kQRounds; ++i) unpack8<T>(q_raw[i], y[i]);
  if (a.pool.rotate) rotate_from_halves<kTeam>(y);
#pragma unroll
  for (int i = 0; i < kQRounds; ++i) {
    top[i] = 0.0f;
#pragma unroll
    for (int c = 0; c < 8; ++c) top[i] = fmaxf(top[i], fabsf(y[i][c]));
  }
#pragma unroll
  for (int h = 1; h < kTeam; h *= 2)
#pragma unroll
    for (int i = 0; i < kQRounds; ++i) top[i] = fmaxf(top[i], __shfl_xor_sync(0xffffffffu, top[i], h));
#pragma unroll
  for (int i = 0; i < kQRounds; ++i) {
    const int r = i * kTeams + static_cast<int>(threadIdx.x) / kTeam;
    const int e = min(126, max(-126, static_cast<int>(__float_as_uint(top[i]) >> 23) - 126));
    const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
    top[i] = __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
    sums[i] = 0.0f;
    if (r < kRows) {
      __half h[8], rest[8];
      float total = 0.0f;
#pragma unroll
      for (int c = 0; c < 8; ++c) {  // nibbles 1, 3, 5, 7 are read 16 times too large
        const float part = (c & 1) ? 0.0625f : 1.0f;
        h[c] = __float2half_rn(y[i][c] * down * part);
        rest[c] = __float2half_rn(y[i][c] * down * part - __half2float(h[c]));
        total += (__half2float(h[c]) + (kSplitQ ? __half2float(rest[c]) : 0.0f)) * (c & 1 ? 16.0f : 1.0f);
      }
      sums[i] = total;
      __half2 v[4] = {__halves2half2(h[0], h[4]), __halves2half2(h[1], h[5]), __halves2half2(h[2], h[6]), __halves2half2(h[3], h[7])};
      const int w = tl % (kDim / 32), at = (r & 7) * 4 + tl / (kDim / 32);
      q_at[q_index(r >> 3, w, 0) + at] = *reinterpret_cast<const uint2*>(v);
      q_at[q_index(r >> 3, w, 1) + at] = *reinterpret_cast<const uint2*>(v + 2);
      if constexpr (kSplitQ) {
        __half2 u[4] = {__halves2half2(rest[0], rest[4]), __halves2half2(rest[1], rest[5]), __halves2half2(rest[2], rest[6]), __halves2half2(rest[3], rest[7])};
        q_at[kRest + q_index(r >> 3, w, 0) + at] = *reinterpret_cast<const uint2*>(u);
        q_at[kRest + q_index(r >> 3, w, 1) + at] = *reinterpret_cast<const uint2*>(u + 2);
      }
    }
  }
#pragma unroll
  for (int h = 1; h < kTeam; h *= 2)
#pragma unroll
    for (int i = 0; i < kQRounds; ++i) sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], h);
#pragma unroll
  for (int i = 0; i < kQRounds; ++i) {
    const int r = i * kTeams + static_cast<int>(threadIdx.x) / kTeam;
    if (r < kRows && tl == 0) {
      s_f[r] = a.scale * kLog2e * top[i];
      s_sum[r] = sums[i];
    }
  }
  __syncthreads();
  uint32_t q[kQInRegs ? kTiles : 1][kQInRegs ? kDim / 8 : 1];
  if constexpr (kQInRegs) {
#pragma unroll
    for (int n = 0; n < kTiles; ++n)
#pragma unroll
      for (int w = 0; w < kDim / 32; ++w) {
        const uint2 lo = q_at[q_index(n, w, 0) + lane], hi = q_at[q_index(n, w, 1) + lane];
        q[n][4 * w] = lo.x;
        q[n][4 * w + 1] = lo.y;
        q[n][4 * w + 2] = hi.x;
        q[n][4 * w + 3] = hi.y;
      }
  }
  // this lane's rows of S^T and O^T: 8 n + 2 t and the next
  float f[kTiles][2], zero[kTiles][2], m[kTiles][2], l[kTiles][2], o[kDim / 16][kTiles][4];
  int seen[kTiles][2], least = most;
#pragma unroll
  for (int n = 0; n < kTiles; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 8 * n + 2 * t + e;
      f[n][e] = s_f[r] * 0x1p24f;
      zero[n][e] = -8.0f * 0x1p-24f * s_sum[r];  // what the offset adds to a score, taken from its accumulator's start
      seen[n][e] = seen_by(seq, a.causal, min(row0 + r, row0 + rows - 1) / p.group);
      m[n][e] = -FLT_MAX;
      l[n][e] = 0.0f;
    }
  if (a.causal) least = seen_by(seq, 1, row0 / p.group);  // of the first row
#pragma unroll
  for (int i = 0; i < kDim / 16; ++i)
#pragma unroll
    for (int n = 0; n < kTiles; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.0f;

  // this lane's reads of a step: tokens g and g + 8 of the keys, 2 t, 2 t + 1, 2 t + 8 and 2 t + 9 of the values
  constexpr int kKeyWords = kDim / 32, kValueWords = kDim / 64;
  const uint32_t k_get = g * kRow + (kDim == 256 ? 0 : t * (kDim / 8));
  uint32_t v_get[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) v_get[e] = 8 * kDim + value_place(2 * t + e, g * (kDim / 16) / 16) + (g * (kDim / 16) & 15);
  const OffsetBits kbits;
  const CodeBits vbits;
  auto step = [&](int i, int slot) {
    const int at = k0 + kStep * (warp + kWarps * i);
    const uint32_t from = ring + slot * C::kStepBytes;
    float x[kParts][kTiles][4], dk[kParts][2], dv[kParts][2];
    int end[kParts], first_end = k1;
#pragma unroll
    for (int h = 0; h < kParts; ++h) {
      uint32_t k[2][kKeyWords];
      const uint32_t part = from + h * C::kPartBytes;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if constexpr (kDim == 256) {
          uint32_t lo[4], hi[4];
          read_words(lo, part + k_get + e * 8 * kRow + 16 * ((2 * t) ^ (g & 1)));
          read_words(hi, part + k_get + e * 8 * kRow + 16 * ((2 * t + 1) ^ (g & 1)));
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            k[e][w] = lo[w];
            k[e][w + kKeyWords - 4] = hi[w];
          }
        } else {
          read_words(k[e], part + k_get + e * 8 * kRow);
        }
        uint32_t d[1];
        read_words(d, part + 16 * kDim + g * 4 + e * 32);
        dk[h][e] = __uint_as_float(d[0]);
        read_words(d, part + 16 * kDim + 64 + g * 4 + e * 32);
        dv[h][e] = __uint_as_float(d[0]);
      }
      end[h] = *const_cast<volatile int*>(&s_end[warp][slot][h]);
      first_end = min(first_end, end[h]);
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[h][n][e] = zero[n][e & 1];
      float x2[4] = {};  // one tile: two independent sums of a score
#pragma unroll
      for (int w = 0; w < kKeyWords; ++w) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const uint32_t a0 = kbits.offsets_04(k[0][w]), a1 = kbits.offsets_04(k[1][w]), a2 = kbits.offsets_15(k[0][w]), a3 = kbits.offsets_15(k[1][w]);
#pragma unroll
          for (int n = 0; n < kTiles; ++n) {
            if constexpr (kQInRegs) {
              mma16816(kTiles == 1 && c ? x2 : x[h][n], a0, a1, a2, a3, q[n][4 * w + 2 * c], q[n][4 * w + 2 * c + 1]);
            } else {
              const uint2 v = q_at[q_index(n, w, c) + lane];
              mma16816(x[h][n], a0, a1, a2, a3, v.x, v.y);
            }
            if constexpr (kSplitQ) {
              const uint2 v = q_at[kRest + q_index(n, w, c) + lane];
              mma16816(kTiles == 1 && !c ? x2 : x[h][n], a0, a1, a2, a3, v.x, v.y);
            }
          }
          k[0][w] >>= 8;
          k[1][w] >>= 8;
        }
      }
      if constexpr (kTiles == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[h][0][e] += x2[e];
      }
    }
    float pr[kParts][kTiles][4], wt[kParts][kTiles][4];  // probabilities, weights
    const bool hidden = at + kStep > min(least, first_end);  // some row does not see all of these tokens
    auto sees = [&](int h, int n, int e) { return at + kTile * h + g + (e < 2 ? 0 : 8) < min(seen[n][e & 1], end[h]); };
    auto against = [&]() {
#pragma unroll
      for (int h = 0; h < kParts; ++h)
#pragma unroll
        for (int n = 0; n < kTiles; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            pr[h][n][e] = ex2(fmaf(x[h][n][e], dk[h][e >> 1] * f[n][e & 1], -m[n][e & 1]));
            wt[h][n][e] = pr[h][n][e] * dv[h][e >> 1];
          }
      if (hidden) {
#pragma unroll
        for (int h = 0; h < kParts; ++h)
#pragma unroll
          for (int n = 0; n < kTiles; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (!sees(h, n, e)) pr[h][n][e] = wt[h][n][e] = 0.0f;
      }
    };
    against();
    float most_p = 0.0f, most_w = 0.0f;
#pragma unroll
    for (int h = 0; h < kParts; ++h)
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          most_p = fmaxf(most_p, fmaxf(pr[h][n][e], pr[h][n][e + 1]));
          most_w = fmaxf(most_w, fmaxf(wt[h][n][e], wt[h][n][e + 1]));
        }
    // (p = inf times a scale of 0 is the NaN that fmax passes over: p shows it)
    if (__any_sync(0xffffffffu, most_w > kMostWeight || most_p > kMostP)) {  // move the references
#pragma unroll
      for (int n = 0; n < kTiles; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float top = m[n][e];
#pragma unroll
          for (int h = 0; h < kParts; ++h)
#pragma unroll
            for (int c = e; c < 4; c += 2)
              if (!hidden || sees(h, n, c))
                top = fmaxf(top, x[h][n][c] * (dk[h][c >> 1] * f[n][e]) + (fmaxf(lg2(dv[h][c >> 1]), kLeastScale) - kLift));
#pragma unroll
          for (int h = 4; h < 32; h *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, h));
          const float keep = ex2(m[n][e] - top);
          l[n][e] *= keep;
          m[n][e] = top;
#pragma unroll
          for (int c = 0; c < kDim / 16; ++c) {
            o[c][n][e] *= keep;
            o[c][n][e + 2] *= keep;
          }
        }
      against();
    }
#pragma unroll
    for (int h = 0; h < kParts; ++h) {
      uint32_t b0[kTiles], b1[kTiles];
#pragma unroll
      for (int n = 0; n < kTiles; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) l[n][e & 1] += pr[h][n][e];
        const __half2 lo = __floats2half2_rn(wt[h][n][0], wt[h][n][1]), hi = __floats2half2_rn(wt[h][n][2], wt[h][n][3]);
        b0[n] = transpose8(*reinterpret_cast<const uint32_t*>(&lo));
        b1[n] = transpose8(*reinterpret_cast<const uint32_t*>(&hi));
      }
      uint32_t v[4][kValueWords];
#pragma unroll
      for (int e = 0; e < 4; ++e) read_words(v[e], from + h * C::kPartBytes + v_get[e & 1] + (e >> 1) * 8 * kRow);
#pragma unroll
      for (int w = 0; w < kValueWords; ++w)
#pragma unroll
        for (int u = 0; u < 2; ++u) {  // channels 4 u .. 4 u + 3 of the word, two tokens in each register
          uint32_t v0 = __byte_perm(v[0][w], v[1][w], u ? 0x7632 : 0x5410), v1 = __byte_perm(v[2][w], v[3][w], u ? 0x7632 : 0x5410);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t a0 = vbits.codes_04(v0), a1 = vbits.codes_15(v0), a2 = vbits.codes_04(v1), a3 = vbits.codes_15(v1);
#pragma unroll
            for (int n = 0; n < kTiles; ++n) mma16816(o[4 * w + 2 * u + c][n], a0, a1, a2, a3, b0[n], b1[n]);
            v0 >>= 8;
            v1 >>= 8;
          }
        }
    }
  };
  int slot = 0, fill = kStages - 1;
  for (int i = 0; i < steps; ++i) {
    copy_wait<kStages - 2>();
    __syncwarp();  // step i has landed for every lane, and every lane has read step i - 1
    load(i + kStages - 1, fill);
    step(i, slot);
    fill = slot;
    if (++slot == kStages) slot = 0;
  }
  copy_wait<0>();
  __syncthreads();  // the warps' sums take the rings' place

  // ---- join the warps
#pragma unroll
  for (int n = 0; n < kTiles; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int h = 4; h < 32; h *= 2) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], h);
      const int r = 8 * n + 2 * t + e;
      if (g == 0) {
        s_m[warp][r] = m[n][e];
        s_l[warp][r] = l[n][e];
      }
      float* const dst = s_o + (warp * kRows + r) * C::kJoinRow + g * C::kEighth;
#pragma unroll
      for (int c = 0; c < kDim / 16; ++c) *reinterpret_cast<float2*>(dst + 2 * c) = make_float2(o[c][n][e], o[c][n][e + 2]);
    }
  __syncthreads();
  const bool whole = most <= chunk && !p.cluster;
#pragma unroll
  for (int r0 = 0; r0 < kRows; r0 += kTeams) {
    const int r = r0 + static_cast<int>(threadIdx.x) / kTeam;
    const int rr = min(r, kRows - 1);
    float top = s_m[0][rr], sum = 0.0f, z[1][8] = {}, (&y)[8] = z[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) top = fmaxf(top, s_m[w][rr]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float k = ex2(s_m[w][rr] - top);
      sum += s_l[w][rr] * k;
      const float* const src = s_o + (w * kRows + rr) * C::kJoinRow + tl * 8 / (kDim / 8) * C::kEighth + tl * 8 % (kDim / 8);
#pragma unroll
      for (int c = 0; c < 8; c += 2) {
        const float2 v = *reinterpret_cast<const float2*>(src + c);
        y[c] += v.x * k;
        y[c + 1] += v.y * k;
      }
    }
    if (whole) {
      const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int c = 0; c < 8; ++c) y[c] *= inv;
      if (a.pool.rotate) rotate_to_halves<kTeam>(z);
      if (r < rows) {
        const int token = seq.q0 + (row0 + r) / p.group, head = kvh * p.group + (row0 + r) % p.group;
        store_head<kTeam>(static_cast<T*>(a.o) + (static_cast<size_t>(token) * a.heads + head) * kDim, y, a.pool.rotate);
      }
    } else if (r < rows) {
      float* const dst = p.cluster ? s_part + r * (kDim + 2) : p.part + (static_cast<size_t>(blockIdx.x) * kRows + r) * (kDim + 2);
#pragma unroll
      for (int c = 0; c < 8; c += 2) *reinterpret_cast<float2*>(dst + tl * 8 + c) = make_float2(y[c], y[c + 1]);
      if (tl == 0) *reinterpret_cast<float2*>(dst + kDim) = make_float2(top, sum);
    }
  }
  if (!p.cluster) return;

  // ---- join the cluster: its CTAs take the rows in turn
  __syncwarp();
  cluster_sync();
  const uint32_t mine = smem_u32(s_part);
  for (int r0 = 0; r0 < rows; r0 += kTeams * p.cluster) {
    const int r = r0 + ch * kTeams + static_cast<int>(threadIdx.x) / kTeam;
    float m = -FLT_MAX, sum = 0.0f, z[1][8] = {}, (&y)[8] = z[0];
    if (r < rows) {
      for (int c = 0; c < p.cluster; ++c) {
        const uint32_t at = mapa_shared(mine + static_cast<uint32_t>(r) * (kDim + 2) * 4, static_cast<uint32_t>(c));
        const float2 ml = cluster_load2(at + kDim * 4);
        float2 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = cluster_load2(at + tl * 32 + e * 8);
        const float top = fmaxf(m, ml.x), keep = ex2(m - top), k = ex2(ml.x - top);
        m = top;
        sum = sum * keep + ml.y * k;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[2 * e] = y[2 * e] * keep + v[e].x * k;
          y[2 * e + 1] = y[2 * e + 1] * keep + v[e].y * k;
        }
      }
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int c = 0; c < 8; ++c) y[c] *= inv;
    if (a.pool.rotate) rotate_to_halves<kTeam>(z);
    if (r < rows) {
      const int token = seq.q0 + (row0 + r) / p.group, head = kvh * p.group + (row0 + r) % p.group;
      store_head<kTeam>(static_cast<T*>(a.o) + (static_cast<size_t>(token) * a.heads + head) * kDim, y, a.pool.rotate);
    }
  }
  __syncwarp();
  cluster_sync();  // nobody leaves while its result is being read
}

// The chunks of a query row (one head of one token) joined, teams of D / 8 lanes taking chunks in turn: by a CTA, where there are
// many, or by a warp.
template <typename T, int kDim, bool kMany>
__global__ void __launch_bounds__(32 * kWarps) attention_kv4_join_kernel(const __grid_constant__ Kv4Params p) {
  constexpr int kTeam = kDim / 8, kWarpTeams = 32 / kTeam, kTeams = kMany ? kWarps * kWarpTeams : kWarpTeams;
  __shared__ float s_m[kMany ? kWarps : 1], s_l[kMany ? kWarps : 1];
  __shared__ __align__(16) float s_y[kMany ? kWarps : 1][kMany ? kDim : 1];
  const Kv4AttentionArgs& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, tl = lane % kTeam;
  const int row = kMany ? blockIdx.x : blockIdx.x * kWarps + warp;
  const int token = row / a.heads, head = row % a.heads;
  const int team = (kMany ? warp * kWarpTeams : 0) + lane / kTeam;
  // Where the row's parts lie follows from offsets and lengths.  They can be read ahead of the wait: this kernel starts once all CTAs
  // of the other one are past their own wait, so what wrote them has ended.
  int b = 0, first = 0, chunks = 0, before = 0, kvh = 0, r = 0, tile = 0;
  if (row < a.total_q * a.heads) {
    const int len = lane < a.batch ? usable_length(a, read_index<true>(a.kv_len + lane)) : 0;
    const bool found = find_sequence<true>(a.cu_q, a.batch, token, b, first);
    const Sequence seq = load_sequence<true>(a, b);
    if (found && usable(a, seq) && token >= seq.q0 && token - seq.q0 < seq.n) {  // (offsets may be cut)
      const float per_length = split_of<true>(p, len);
      const int chunk = chunk_size(seq.len, chunks_of(seq.len, per_length));
      kvh = head / p.group;
      r = (token - seq.q0) * p.group + head % p.group;
      tile = r / p.rows;
      const int most = seen_by(seq, a.causal, (min((tile + 1) * p.rows, seq.n * p.group) - 1) / p.group);
      chunks = (most + chunk - 1) / max(chunk, 1);
      for (int b0 = 0; b0 < b; b0 += 32) {  // chunks of the sequences ahead
        const int at = b0 + lane;
        before += __reduce_add_sync(
            0xffffffffu, at < b ? chunks_of(b0 == 0 ? len : usable_length(a, read_index<true>(a.kv_len + at)), per_length) : 0);
      }
    }
  }
  griddep_wait();
  griddep_launch_dependents();
  if (chunks < 2) return;  // its CTA has written the result, or nobody has to
  const size_t unit = static_cast<size_t>(before) * p.per + kvh * p.row_tiles + tile;
  const float* const src = p.part + (unit * p.rows + r % p.rows) * (kDim + 2);
  const size_t next = static_cast<size_t>(p.per) * p.rows * (kDim + 2);
  float m = -FLT_MAX, l = 0.0f, z[1][8] = {}, (&y)[8] = z[0];
  auto add = [&](float m2, float l2, const float (&y2)[8]) {
    const float top = fmaxf(m, m2), keep = ex2(m - top), k = ex2(m2 - top);
    m = top;
    l = l * keep + l2 * k;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = y[e] * keep + y2[e] * k;
  };
#pragma unroll 4
  for (int c = team; c < chunks; c += kTeams) {
    const float* const at = src + c * next;
    const float2 ml = *reinterpret_cast<const float2*>(at + kDim);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const float2 w = *reinterpret_cast<const float2*>(at + tl * 8 + e);
      v[e] = w.x;
      v[e + 1] = w.y;
    }
    add(ml.x, ml.y, v);
  }
#pragma unroll
  for (int h = kTeam; h < 32; h *= 2) {  // the warp's teams (a sum or maximum of two is the same on both sides)
    float v[8];
    const float m2 = __shfl_xor_sync(0xffffffffu, m, h), l2 = __shfl_xor_sync(0xffffffffu, l, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __shfl_xor_sync(0xffffffffu, y[e], h);
    add(m2, l2, v);
  }
  if constexpr (kMany) {
    if (lane < kTeam) {
      if (tl == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
      }
#pragma unroll
      for (int e = 0; e < 8; e += 4) *reinterpret_cast<float4*>(&s_y[warp][tl * 8 + e]) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
    }
    __syncthreads();
    if (warp > 0) return;
    m = -FLT_MAX;
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = s_y[w][tl * 8 + e];
      add(s_m[w], s_l[w], v);
    }
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int c = 0; c < 8; ++c) y[c] *= inv;
  if (a.pool.rotate) rotate_to_halves<kTeam>(z);
  if (lane < kTeam) store_head<kTeam>(static_cast<T*>(a.o) + (static_cast<size_t>(token) * a.heads + head) * kDim, y, a.pool.rotate);
}

int rows_of(const Kv4AttentionArgs& a) { return static_cast<int64_t>(a.max_q) * (a.heads / a.pool.kv_heads) <= 8 ? 8 : 16; }

// The split, as far as the workspace has room for the CTAs' results.
cudaError_t plan_split(const Kv4AttentionArgs& a, size_t ws_bytes, Kv4Params* p) {
  p->group = a.heads / a.pool.kv_heads;
  p->rows = rows_of(a);
  const int64_t tiles = (static_cast<int64_t>(a.max_q) * p->group + p->rows - 1) / p->rows;
  const int64_t units = static_cast<int64_t>(a.batch) * a.pool.kv_heads * tiles;
  if (units > 0x3fffffff) return cudaErrorInvalidConfiguration;
  p->row_tiles = static_cast<int>(tiles);
  p->per = static_cast<int>(a.pool.kv_heads * tiles);
  // A cluster a unit where clusters of eight leave SMs to spare and a part stays short: then the second launch is what a call
  // can save.  One token over 817, 8 heads of 256 channels on one: 8.6 us either way on the device, 11.5 against 14 as the host's calls
  // follow one another; over 4000, 8 heads of 128: 8.2 against 11.4 on the device; of 256 channels, 16 contexts: 16.4 against
  // 14.0.  (23 ragged contexts of up to 6001 tokens and 8 heads, in clusters all the same: 24 against 20.5 when that was tried.)
  const int64_t parts = (static_cast<int64_t>(a.max_len) + kLeastChunk - 1) / kLeastChunk;
  p->cluster = 0;
  p->target = p->most_target = 0;
  if (units * 8 <= a.num_sms && parts > 1 && a.max_len <= cluster_len(a.pool.head_dim)) {
    p->cluster = static_cast<int>(parts < 8 ? parts : 8);
    p->ctas = static_cast<int>(units * p->cluster);
    return cudaSuccess;
  }
  int64_t target = static_cast<int64_t>(a.num_sms) * ctas_per_sm(a.pool.head_dim, p->rows), most_target = target * (p->rows == 8 ? kWaves8 : kWaves16);
  const int64_t part = static_cast<int64_t>(p->rows) * (a.pool.head_dim + 2) * 4;
  const int64_t least = units * parts;  // CTAs with the least chunks
  const int64_t room = static_cast<int64_t>(ws_bytes / part) - units;
  if (units * a.max_len <= target * kLongChunk) most_target = target;
  if (target > room) target = room;
  if (most_target > room) most_target = room;
  if (target < units || least <= units) target = most_target = 0;  // (no more than a chunk a sequence)
  p->target = static_cast<int>(target);
  p->most_target = static_cast<int>(most_target);
  p->ctas = static_cast<int>(target == 0 ? units : most_target + units < least ? most_target + units : least);
  return cudaSuccess;
}

template <typename T, int kDim, int kTiles, bool kSplitQ>
cudaError_t launch(const Kv4AttentionArgs& a) {
  Kv4Params p;
  p.a = a;
  if (cudaError_t e = plan_split(a, a.ws ? a.ws_bytes : 0, &p)) return e;
  p.part = static_cast<float*>(a.ws);
  const int64_t joins = static_cast<int64_t>(a.total_q) * a.heads;
  if (joins > 0x7fffffff) return cudaErrorInvalidConfiguration;
  using C = Cfg<kDim, kTiles, kSplitQ>;
  auto kern = attention_kv4_kernel<T, kDim, kTiles, kSplitQ>;
  if (C::kSmem > 48 * 1024) {  // once a device
    static std::atomic<uint64_t> raised{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? uint64_t{1} << dev : 0;
    if (bit == 0 || !(raised.load(std::memory_order_relaxed) & bit)) {
      e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem);
      if (e != cudaSuccess) return e;
      raised.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(p.ctas));
  cfg.blockDim = dim3(32 * kWarps);
  cfg.dynamicSmemBytes = C::kSmem;
  cfg.stream = a.stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = static_cast<unsigned>(p.cluster);
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.cluster ? 2 : 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p);
  if (e != cudaSuccess) return e;
  if (p.target > 0) {
    // about so many chunks a sequence: a CTA a row where a warp would take many rounds
    const int64_t units = static_cast<int64_t>(a.batch) * p.per;
    const bool many = p.target >= 8 * units;
    cfg.gridDim = dim3(static_cast<unsigned>(many ? joins : (joins + kWarps - 1) / kWarps));
    cfg.dynamicSmemBytes = 0;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, many ? attention_kv4_join_kernel<T, kDim, true> : attention_kv4_join_kernel<T, kDim, false>, p);
    if (e != cudaSuccess) return e;
  }
  return cudaGetLastError();
}

template <typename T, int kDim>
cudaError_t launch(const Kv4AttentionArgs& a) {
  if (std::is_same<T, __half>::value && a.pool.rotate)
    return rows_of(a) == 8 ? launch<T, kDim, 1, std::is_same<T, __half>::value>(a) : launch<T, kDim, 2, std::is_same<T, __half>::value>(a);
  return rows_of(a) == 8 ? launch<T, kDim, 1, false>(a) : launch<T, kDim, 2, false>(a);
}

}  // namespace

size_t attention_kv4_workspace(const Kv4AttentionArgs& a) {
  Kv4Params p;
  if (plan_split(a, ~static_cast<size_t>(0) >> 1, &p) != cudaSuccess || p.target == 0) return 0;
  const size_t n = static_cast<size_t>(p.ctas) * p.rows * (a.pool.head_dim + 2) * 4;
  return (n + 255) & ~static_cast<size_t>(255);
}

cudaError_t launch_attention_kv4(const Kv4AttentionArgs& a) {
  if (a.dt == 0)
    return a.pool.head_dim == 64 ? launch<__half, 64>(a) : a.pool.head_dim == 128 ? launch<__half, 128>(a) : launch<__half, 256>(a);
  return a.pool.head_dim == 64 ? launch<__nv_bfloat16, 64>(a)
                               : a.pool.head_dim == 128 ? launch<__nv_bfloat16, 128>(a) : launch<__nv_bfloat16, 256>(a);
}

cudaError_t read_and_clear_error_word_attention_kv4(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess || *out == 0) return e;  // (cleared only where it is set: the check goes through every unit's word)
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

}  // namespace qvla
