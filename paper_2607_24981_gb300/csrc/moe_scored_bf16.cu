// moe_scored_bf16.cu -- routing by scores for bf16 logits.
#include "moe_scored.cuh"

namespace ilw {
template cudaError_t launch_route_scored<__nv_bfloat16>(const MoeScoredParams &, cudaStream_t);
}  // namespace ilw
