// i8_gemm_f32.cu -- the int8 products with float results (a translation unit each, so that they compile in parallel).
#include "i8_gemm.cuh"

namespace ilw {
template cudaError_t launch_i8<float, false>(const I8Params &, int32_t, int, size_t, cudaStream_t);
}  // namespace ilw
