// i8_gemm_long_f32.cu -- the int8 products with float results and long sums.
#include "i8_gemm.cuh"

namespace ilw {
template cudaError_t launch_i8<float, true>(const I8Params &, int32_t, int, size_t, cudaStream_t);
}  // namespace ilw
