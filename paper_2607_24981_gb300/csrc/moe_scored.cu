// moe_scored.cu -- routing by scores, with a bias for balance and by groups of experts: selection (moe_scores.cuh), a warp a token, with
// the order of moe.cu.
#include <algorithm>
#include <cstdint>

#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "moe_order.cuh"
#include "moe_scores.cuh"
#include "mx_kernels.h"

namespace ilw {
namespace {

// max|bias| of what fp32 scores are added to, by a warp
__device__ __forceinline__ float largest_bias(const MoeScoredParams &p, int lane) {
    float m = 0.0f;
    if (p.scores.bias)
        for (int e = lane; e < p.E; e += 32) m = fmaxf(m, fabsf(__ldg(p.scores.bias + e)));
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    return m;
}

// Selection by scores of a chunk's tokens by a cluster, a warp a token, and the chunk's counts.
constexpr int kScoredThreads = 512;
template <typename T, int S>
__global__ void __cluster_dims__(kSelectCtas, 1, 1) __launch_bounds__(kScoredThreads) route_scored_kernel(const __grid_constant__ MoeScoredParams p, int wide) {
    __shared__ int32_t count[kRouteMaxExperts];
    constexpr int kTokens = select_tokens(S);
    const int lane = threadIdx.x & 31;
    for (int e = threadIdx.x; e < p.E; e += kScoredThreads) count[e] = 0;
    __syncthreads();
    grid_wait();
    const float bias_max = largest_bias(p, lane);
    for (int i = threadIdx.x >> 5; i < kTokens; i += kScoredThreads / 32) {
        const int64_t t = (int64_t)blockIdx.x * kTokens + i;
        if (t >= p.T) break;
        int32_t e;
        float w;
        select_scored<T, S / 2>(p, t, wide, bias_max, lane, e, w);
        if (lane < p.k) {
            p.expert[t * p.k + lane] = e;
            p.weight[t * p.k + lane] = w;
            if (e >= 0) atomicAdd(&count[e], 1);  // (whole numbers: any order gives the same)
        }
    }
    __syncthreads();
    add_counts<kScoredThreads>(p, count);
}

// Few tokens by scores: all of it by one CTA, a warp a token.
template <typename T, int S>
__global__ void __launch_bounds__(4 * kOneTokens) route_one_scored_kernel(const __grid_constant__ MoeScoredParams p, int wide) {
    extern __shared__ __align__(16) uint32_t dyn[];
    __shared__ int32_t base[kRouteMaxExperts], count[kRouteMaxExperts], all;
    constexpr int words = kOneTokens / 32, row = words + 1, kEntries = kRouteMaxTop / 4;
    int32_t *out_e = (int32_t *)dyn;  // [T][k], then bits [E][row] and the running counts
    uint32_t *bits = dyn + p.T * p.k;
    const int lane = threadIdx.x & 31;
    for (int i = threadIdx.x; i < p.E * row; i += blockDim.x) bits[i] = 0;
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
    __syncthreads();
    grid_wait();
    const float bias_max = largest_bias(p, lane);
    for (int t = threadIdx.x >> 5; t < p.T; t += blockDim.x / 32) {
        int32_t e;
        float w;
        select_scored<T, S / 2>(p, t, wide, bias_max, lane, e, w);
        if (lane < p.k) {
            out_e[t * p.k + lane] = p.expert[t * p.k + lane] = e;
            p.weight[t * p.k + lane] = w;
            if (e >= 0) atomicAdd(&count[e], 1);
        }
    }
    __syncthreads();
    int32_t ex[kEntries];
#pragma unroll
    for (int j = 0; j < kEntries; ++j) {
        const int i = j * blockDim.x + threadIdx.x;
        ex[j] = i < p.T * p.k ? out_e[i] : -1;
    }
    if (threadIdx.x < 32) {
        const int32_t x = scan_experts(p.E, count, base, threadIdx.x);
        if (threadIdx.x == 0) all = x;
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= p.E; e += blockDim.x) p.offsets[e] = e < p.E ? base[e] : all;
    place_chunk<words>(p, 0, p.T * p.k, ex, bits, (int32_t *)bits + p.E * row, base);
    for (int i = all + threadIdx.x; i < p.T * p.k; i += blockDim.x) p.source[i] = -1;
}

size_t one_scored_smem(int32_t T, int32_t E, int32_t k) { return ((size_t)2 * E * (kOneTokens / 32 + 1) + (size_t)T * k) * 4; }
template <typename T, int S>
cudaError_t route_scored(const MoeScoredParams &p, cudaStream_t s) {
    constexpr int kLane = std::min(16, S / 2 * (int)sizeof(T));  // bytes of a lane's loads
    const int wide = (uintptr_t)p.logits % kLane == 0 && p.ld * (int64_t)sizeof(T) % kLane == 0 && p.E * sizeof(T) % kLane == 0;
    if (moe_route_in_one(p.T, p.E)) {
        static SmemLimit limit;
        const cudaError_t e = raise_smem_limit(limit, (const void *)route_one_scored_kernel<T, S>, (int)one_scored_smem(kOneTokens, kRouteMaxExperts, kRouteMaxTop));
        if (e != cudaSuccess) return e;
        return launch_after(route_one_scored_kernel<T, S>, 1, 4 * kOneTokens, one_scored_smem(p.T, p.E, p.k), s, p, wide);
    }
    constexpr int kChunk = chunk_tokens(S);
    const int32_t chunks = (int32_t)((p.T + (int64_t)kChunk - 1) / kChunk);
    const cudaError_t e = launch_after(route_scored_kernel<T, S>, chunks * kSelectCtas, kScoredThreads, 0, s, p, wide);
    if (e != cudaSuccess) return e;
    return launch_moe_place(p, kChunk, s);
}
template <typename T>
cudaError_t route_scored_form(const MoeScoredParams &p, cudaStream_t s) {
    switch (group_size(p.E)) {
        case 4: return route_scored<T, 4>(p, s);
        case 8: return route_scored<T, 8>(p, s);
        case 16: return route_scored<T, 16>(p, s);
        default: return route_scored<T, 32>(p, s);
    }
}

}  // namespace

cudaError_t launch_moe_route_scored(const MoeScoredParams &r, cudaStream_t s) {
    MoeScoredParams p = r;
    RouteScores &q = p.scores;
    q.group_size = p.E / q.groups;
    q.per_group = divisor(q.group_size);
    const int per = group_size(p.E) / 2, lanes = q.group_size / per;  // experts a lane
    q.lanes_per_group = q.group_size % per == 0 && (lanes & (lanes - 1)) == 0 ? lanes : 0;
    if (p.form == ILW_FP32) return route_scored_form<float>(p, s);
    if (p.form == ILW_FP16) return route_scored_form<__half>(p, s);
    return route_scored_form<__nv_bfloat16>(p, s);
}

}  // namespace ilw
