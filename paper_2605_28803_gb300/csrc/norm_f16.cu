// The norms around a block, with branch and output in f16 and the residual in f16 or float32 (fp4_rows.cuh).
#include "fp4_rows.cuh"

namespace qvla {

cudaError_t launch_norm_f16(const RowsArgs& a) {
  using T = __half;
  if (a.codes != nullptr) return a.xdt == 2 ? fp4::launch_quant<float, T, true>(a) : fp4::launch_quant<T, T, true>(a);
  return a.xdt == 2 ? fp4::launch_rows<float, T, true, false, fp4::kPieces, 0>(a) : fp4::launch_rows<T, T, true, false, fp4::kPieces, 0>(a);
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
