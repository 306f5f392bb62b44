// moe_scored_f32.cu -- routing by scores for fp32 logits.
#include "moe_scored.cuh"

namespace ilw {
template cudaError_t launch_route_scored<float>(const MoeScoredParams &, cudaStream_t);
}  // namespace ilw
