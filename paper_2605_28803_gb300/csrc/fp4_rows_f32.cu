// Rows of f32 to 4-bit floating point (fp4_rows.cuh).
#include "fp4_rows.cuh"

namespace qvla {

cudaError_t launch_fp4_quantize_f32(const RowsArgs& a) { return fp4::launch_quantize_fmt<float>(a); }

}  // namespace qvla
