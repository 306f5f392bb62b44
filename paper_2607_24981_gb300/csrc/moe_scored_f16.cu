// moe_scored_f16.cu -- routing by scores for fp16 logits.
#include "moe_scored.cuh"

namespace ilw {
template cudaError_t launch_route_scored<__half>(const MoeScoredParams &, cudaStream_t);
}  // namespace ilw
