// Codes of 4-bit floating point back to values: code * block scale (exact) * the row's scale, one float32 rounding, one to the
// output's type.  A thread takes 32 channels; for calibration and checks, bound by the writes.
#include "fp4_rows.cuh"

namespace qvla {
namespace {

template <typename T, int kFmt>
__global__ void __launch_bounds__(256) dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                         const float* __restrict__ row_scale, int M, int K, T* __restrict__ out) {
  const int per = K >> 5;
  const size_t at = static_cast<size_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  griddep_wait();
  griddep_launch_dependents();
  if (at >= static_cast<size_t>(M) * per) return;
  const int m = static_cast<int>(at / per), j = static_cast<int>(at - static_cast<size_t>(m) * per);
  const uint4 c = *reinterpret_cast<const uint4*>(codes + at * 16);
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  float s[2], row = 1.0f;
  if constexpr (kFmt == fp4::kMx) {
    s[0] = s[1] = fp4::e8m0_value(scales[fp4::scale_offset(m, j, K >> 7)]);
  } else {
    const uint32_t b = *reinterpret_cast<const uint16_t*>(scales + fp4::scale_offset(m, 2 * j, K >> 6));
    // (a byte with the sign set is no scale; its other bits are taken)
    s[0] = fp4::e4m3_value(b & 0x7Fu);
    s[1] = fp4::e4m3_value((b >> 8) & 0x7Fu);
    row = row_scale[m];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float2 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k].x = fp4::e2m1_value(w[i] >> (8 * k)) * s[i >> 1] * row;
      v[k].y = fp4::e2m1_value(w[i] >> (8 * k + 4)) * s[i >> 1] * row;
    }
    fp4::write_unit(out + at * 32 + i * 8, v);
  }
}

template <typename T>
cudaError_t launch(const uint8_t* codes, const uint8_t* scales, const float* row_scale, int fmt, int M, int K, void* out, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((static_cast<size_t>(M) * (K >> 5) + 255) / 256));
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
