// The norms around a block, with branch and output in f16 and the residual in f16 or float32 (fp4_rows.cuh).
#include "fp4_rows.cuh"

namespace qvla {

cudaError_t launch_norm_f16(const RowsArgs& a) {
  using T = __half;
  return a.xdt == 2 ? fp4::launch_norm<float, T>(a) : fp4::launch_norm<T, T>(a);
}

cudaError_t read_and_clear_error_word_norm_f16(unsigned int* out, cudaStream_t stream) {
  cudaError_t e = cudaStreamSynchronize(stream);
  if (e != cudaSuccess) return e;
  e = cudaMemcpyFromSymbol(out, g_error_word, sizeof(unsigned int));
  if (e != cudaSuccess || *out == 0) return e;
  const unsigned int zero = 0;
  return cudaMemcpyToSymbol(g_error_word, &zero, sizeof(unsigned int));
}

}  // namespace qvla
