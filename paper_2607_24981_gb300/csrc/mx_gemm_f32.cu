// mx_gemm_f32.cu -- the MXFP4 products with float results (a translation unit each, so that they compile in parallel).
#include "mx_gemm.cuh"

namespace ilw {
template cudaError_t launch_mx<float>(const MxParams &, int32_t, int, size_t, cudaStream_t);
}  // namespace ilw
