// Block-scaled tcgen05.mma of 4-bit floating-point codes: instructions, descriptors and tensor maps that the products share.
#pragma once

#include <algorithm>
#include <atomic>

#include "fp4.cuh"
#include "gemm_kernel.cuh"

namespace qvla {
namespace {

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

// gelu in its tanh form: g / (1 + exp(-2 u)), u = sqrt(2 / pi) (g + 0.044715 g^3); the exponential and the reciprocal by the
// hardware's approximations (2^-22 and 2^-23 of their values), without the steps that would keep subnormal results.
__device__ __forceinline__ float gelu_fast(float g) {
  const float t = g * fmaf(-0.1029432397f, g * g, -2.3022081986f);  // -2 u log2(e)
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return g * r;
}

// ---- on the host -----------------------------------------------------------------------------------------------------------

// Scale tiles [row groups][tiles of a row][512 bytes], read in boxes of kTiles tiles of `groups` row groups.
cudaError_t make_tmap_scales(CUtensorMap* m, const void* base, int row_groups, int tiles, int box_tiles, int box_groups) {
  PFN_cuTensorMapEncodeTiled_v12000 enc = tensor_map_encoder();
  if (!enc) return cudaErrorNotSupported;
  const cuuint64_t dims[3] = {128, static_cast<cuuint64_t>(tiles), static_cast<cuuint64_t>(row_groups)};
  const cuuint64_t strides[2] = {512, static_cast<cuuint64_t>(tiles) * 512};
  const cuuint32_t box[3] = {128, static_cast<cuuint32_t>(box_tiles), static_cast<cuuint32_t>(box_groups)};
  const cuuint32_t estr[3] = {1, 1, 1};
  CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

const CUtensorMap& weight_map(const Fp4GemmArgs& a, int i) {
  return *reinterpret_cast<const CUtensorMap*>(static_cast<const uint8_t*>(a.maps) + i * kFp4MapBytes);
}

// Raises the kernel's limit of dynamic shared memory once per device; `done` holds the devices where it is.
cudaError_t raise_smem(const void* kern, int bytes, std::atomic<unsigned long long>* done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = 1ull << (dev & 63);
  if (done->load() & bit) return cudaSuccess;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess) done->fetch_or(bit);
  return e;
}

}  // namespace
}  // namespace qvla
