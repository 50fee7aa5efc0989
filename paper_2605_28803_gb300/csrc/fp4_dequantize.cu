// Codes of 4-bit floating point back to values: code * block scale (exact) * the row's scale, one float32 rounding, one to the
// output's type.  A warp takes 1024 channels, a thread words of 8 that lie 32 apart, so that a warp's loads and stores are whole
// lines (32 consecutive channels a thread took 8.8 us at 816 x 16384).  Bound by the writes.
#include "fp4_rows.cuh"

namespace qvla {
namespace {

template <typename T, int kFmt>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* codes, const uint8_t* scales, const float* row_scale, int M, int K,
                                                         T* out) {
  const int chunks = (K + 1023) / 1024;  // of a row, one to a warp
  const int w = static_cast<int>(blockIdx.x) * 8 + static_cast<int>(threadIdx.x >> 5), m = w / chunks;
  const int first = (w - m * chunks) * 128 + static_cast<int>(threadIdx.x & 31);  // this thread's words of 8 codes: 32 apart
  griddep_wait();
  griddep_launch_dependents();
  if (m >= M) return;
  const float row = kFmt == fp4::kMx ? 1.0f : row_scale[m];
  uint32_t c[4], b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int word = first + 32 * i;
    if (word * 8 >= K) break;
    c[i] = reinterpret_cast<const uint32_t*>(codes)[static_cast<size_t>(m) * (K >> 3) + word];
    b[i] = kFmt == fp4::kMx ? scales[fp4::scale_offset(m, word >> 2, K >> 7)] : scales[fp4::scale_offset(m, word >> 1, K >> 6)];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int word = first + 32 * i;
    if (word * 8 >= K) break;
    // (an E4M3 byte with the sign set is no scale; its other bits are taken)
    const float s = kFmt == fp4::kMx ? fp4::e8m0_value(b[i]) : fp4::e4m3_value(b[i] & 0x7Fu);
    float2 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k].x = fp4::e2m1_value(c[i] >> (8 * k)) * s * row;
      v[k].y = fp4::e2m1_value(c[i] >> (8 * k + 4)) * s * row;
    }
    fp4::write_unit(out + static_cast<size_t>(m) * K + word * 8, v);
  }
}

template <typename T>
cudaError_t launch(const uint8_t* codes, const uint8_t* scales, const float* row_scale, int fmt, int M, int K, void* out, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((static_cast<size_t>(M) * ((K + 1023) / 1024) + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaError_t e = cudaLaunchKernelEx(&cfg, fmt == fp4::kMx ? dequantize_kernel<T, fp4::kMx> : dequantize_kernel<T, fp4::kNv>, codes, scales,
                                     row_scale, M, K, static_cast<T*>(out));
  return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_fp4_dequantize(const uint8_t* codes, const uint8_t* scales, const float* row_scale, int fmt, int M, int K,
                                  void* out, int odt, cudaStream_t stream) {
  if (odt == 0) return launch<__half>(codes, scales, row_scale, fmt, M, K, out, stream);
  if (odt == 1) return launch<__nv_bfloat16>(codes, scales, row_scale, fmt, M, K, out, stream);
  return launch<float>(codes, scales, row_scale, fmt, M, K, out, stream);
}

}  // namespace qvla
