// Rows of bf16 to 4-bit floating point (fp4_rows.cuh).
#include "fp4_rows.cuh"

namespace qvla {

cudaError_t launch_fp4_quantize_bf16(const RowsArgs& a) { return fp4::launch_quantize_fmt<__nv_bfloat16>(a); }

}  // namespace qvla
