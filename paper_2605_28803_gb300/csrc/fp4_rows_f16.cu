// Rows of f16 to 4-bit floating point (fp4_rows.cuh).
#include "fp4_rows.cuh"

namespace qvla {

cudaError_t launch_fp4_quantize_f16(const RowsArgs& a) { return fp4::launch_quantize_fmt<__half>(a); }

}  // namespace qvla
