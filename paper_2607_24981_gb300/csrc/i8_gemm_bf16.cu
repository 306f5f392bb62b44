// i8_gemm_bf16.cu -- the int8 products with __nv_bfloat16 results (a translation unit each, so that they compile in parallel).
#include "i8_gemm.cuh"

namespace ilw {
template cudaError_t launch_i8<__nv_bfloat16, false>(const I8Params &, int32_t, int, size_t, cudaStream_t);
}  // namespace ilw
