// moe_scored.cu -- host side of routing by scores (moe_scored.cuh, instantiated by type in files of their own, which compile in parallel).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ilwdetr.h"
#include "mx_kernels.h"

namespace ilw {
template <typename T> cudaError_t launch_route_scored(const MoeScoredParams &p, cudaStream_t s);
extern template cudaError_t launch_route_scored<float>(const MoeScoredParams &, cudaStream_t);
extern template cudaError_t launch_route_scored<__half>(const MoeScoredParams &, cudaStream_t);
extern template cudaError_t launch_route_scored<__nv_bfloat16>(const MoeScoredParams &, cudaStream_t);

cudaError_t launch_moe_route_scored(const MoeScoredParams &r, cudaStream_t s) {
    MoeScoredParams p = r;
    RouteScores &q = p.scores;
    q.group_size = p.E / q.groups;
    q.per_group = divisor(q.group_size);
    if (p.form == ILW_FP32) return launch_route_scored<float>(p, s);
    if (p.form == ILW_FP16) return launch_route_scored<__half>(p, s);
    return launch_route_scored<__nv_bfloat16>(p, s);
}

}  // namespace ilw
