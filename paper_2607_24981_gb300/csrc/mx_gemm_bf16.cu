// mx_gemm_bf16.cu -- the MXFP4 products with __nv_bfloat16 results (a translation unit each, so that they compile in parallel).
#include "mx_gemm.cuh"

namespace ilw {
template cudaError_t launch_mx<__nv_bfloat16>(const MxParams &, int32_t, int, size_t, cudaStream_t);
}  // namespace ilw
