// moe_scored.cuh -- the kernels of routing by scores, with a bias for balance and by groups of experts: selection as in moe_scores.cuh, order as in moe.cu.
#pragma once
#include <algorithm>
#include <cstdint>

#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "moe_order.cuh"
#include "moe_scores.cuh"
#include "mx_kernels.h"

namespace ilw {
namespace {

// The biases to shared memory by a warp (0 past the last); their largest magnitude.
__device__ __forceinline__ float load_bias(const MoeScoredParams &p, float *to, int words, int lane) {
    float m = 0.0f;
    for (int e = lane; e < words; e += 32) {
        const float b = e < p.E ? __ldg(p.scores.bias + e) : 0.0f;
        to[e] = b;
        m = fmaxf(m, fabsf(b));
    }
    return max_of_lanes<32>(m);
}

// Selection of a chunk's tokens by a cluster, L lanes each, and the chunk's counts, as route_select_kernel.
template <typename T, int S, int L>
__global__ void __cluster_dims__(kSelectCtas, 1, 1) __launch_bounds__(select_tokens(S) * L) route_scored_kernel(const __grid_constant__ MoeScoredParams p, int wide) {
    extern __shared__ __align__(16) uint32_t dyn[];
    __shared__ float s_bias_max;
    constexpr int kSelectTokens = select_tokens(S), kSelectThreads = kSelectTokens * L;
    constexpr int kStride = kGroups * S + 4, kWarpTokens = 32 / L;
    const int lane = threadIdx.x & 31, warp0 = (threadIdx.x >> 5) * kWarpTokens, mine = threadIdx.x / L;
    const int ks = p.k | 1, rs = rank_words(p.scores);
    float *rows = (float *)dyn, *bias = rows + kSelectTokens * kStride, *ranks = bias + (p.scores.bias ? kGroups * S : 0);
    int32_t *out_e = (int32_t *)(ranks + kSelectTokens * rs);
    float *out_w = (float *)out_e + kSelectTokens * ks;
    int32_t *count = (int32_t *)out_w + kSelectTokens * ks;
    for (int e = threadIdx.x; e < p.E; e += kSelectThreads) count[e] = 0;
    grid_wait();
    const int64_t t0 = (int64_t)blockIdx.x * kSelectTokens;
    const int n = (int)max((int64_t)0, min((int64_t)kSelectTokens, p.T - t0));
    if (p.scores.bias && threadIdx.x < 32) {
        const float m = load_bias(p, bias, kGroups * S, lane);
        if (lane == 0) s_bias_max = m;
    }
    load_rows<T, S>(p, t0 + warp0, max(0, min(kWarpTokens, n - warp0)), rows + warp0 * kStride, wide, lane);
    __syncthreads();
    if (warp0 < n) {
        clear_row<L, S>(rows + mine * kStride, mine < n);
        route_tokens<T, L, S>(p, t0 + warp0, mine < n, p.scores.bias ? bias : nullptr, p.scores.bias ? s_bias_max : 0.0f, rows + mine * kStride, ranks + mine * rs,
                                         out_e + mine * ks, ks, out_w + mine * ks);
    }
    __syncthreads();
    const uint32_t over_k = reciprocal(p.k);
    for (int i = threadIdx.x; i < n * p.k; i += kSelectThreads) {
        const int t = over(i, over_k), at = t * ks + i - t * p.k;
        const int32_t e = out_e[at];
        p.expert[t0 * p.k + i] = e;
        p.weight[t0 * p.k + i] = out_w[at];
        if (e >= 0) atomicAdd(&count[e], 1);  // (whole numbers: any order gives the same)
    }
    add_counts<kSelectThreads>(p, count);
}

// Lanes a token where one CTA takes all (16 tokens of 256 experts in groups and with a bias: 11.6 us with eight, 13.0 with 16, 12.8 with four).
constexpr int kManyLanes = 8, kManyTokens = 64, kFewLanes = 4;

// Few tokens (a multiple of 32 / L, the last ones filled up): all of it by one CTA, L threads a token, as route_one_kernel.
template <typename T, int S, int L>
__global__ void __launch_bounds__(L == kManyLanes ? kManyLanes * kManyTokens : kFewLanes * kOneTokens, 1) route_one_scored_kernel(const __grid_constant__ MoeScoredParams p, int wide, int tokens) {
    extern __shared__ __align__(16) uint32_t dyn[];
    __shared__ int32_t base[kRouteMaxExperts], count[kRouteMaxExperts], all;
    __shared__ float s_bias_max;
    constexpr int words = kOneTokens / 32, row = words + 1, kEntries = kRouteMaxTop / 4, kStride = kGroups * S + 4, kWarpTokens = 32 / L;
    const int lane = threadIdx.x & 31, mine = threadIdx.x / L, first = (threadIdx.x >> 5) * kWarpTokens;
    const int rs = rank_words(p.scores);
    float *rows = (float *)dyn, *bias = rows + tokens * kStride, *ranks = bias + (p.scores.bias ? kGroups * S : 0);
    int32_t *out_e = (int32_t *)(ranks + tokens * rs);
    float *out_w = (float *)out_e + tokens * p.k;
    uint32_t *bits = (uint32_t *)out_w + tokens * p.k;
    for (int i = threadIdx.x; i < p.E * row; i += blockDim.x) bits[i] = 0;
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
    grid_wait();
    if (p.scores.bias && threadIdx.x >= blockDim.x - 32) {
        const float m = load_bias(p, bias, kGroups * S, lane);
        if (lane == 0) s_bias_max = m;
    }
    if (first < tokens) load_rows<T, S>(p, first, max(0, min(kWarpTokens, p.T - first)), rows + first * kStride, wide, lane);
    __syncthreads();
    if (first < tokens) {
        clear_row<L, S>(rows + mine * kStride, mine < p.T);
        route_tokens<T, L, S>(p, first, mine < p.T, p.scores.bias ? bias : nullptr, p.scores.bias ? s_bias_max : 0.0f, rows + mine * kStride, ranks + mine * rs, out_e + mine * p.k,
                              p.k, out_w + mine * p.k);
    }
    __syncthreads();
    int32_t ex[kEntries];
#pragma unroll
    for (int j = 0; j < kEntries; ++j) {
        const int i = j * blockDim.x + threadIdx.x;
        ex[j] = -1;
        if (i < p.T * p.k) {
            ex[j] = p.expert[i] = out_e[i];
            p.weight[i] = out_w[i];
            if (ex[j] >= 0) atomicAdd(&count[ex[j]], 1);
        }
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int32_t x = scan_experts(p.E, count, base, threadIdx.x);
        if (threadIdx.x == 0) all = x;
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= p.E; e += blockDim.x) p.offsets[e] = e < p.E ? base[e] : all;
    place_chunk<words>(p, 0, p.T * p.k, ex, bits, (int32_t *)bits + p.E * row, base);
    for (int i = all + threadIdx.x; i < p.T * p.k; i += blockDim.x) p.source[i] = -1;
}

size_t scored_smem(int tokens, int32_t E, int32_t k, const RouteScores &q) {
    return ((size_t)tokens * (row_words(E) + rank_words(q) + 2 * k) + (q.bias ? kGroups * group_size(E) : 0)) * 4;
}
int one_lanes(int32_t T) { return T <= kManyTokens ? kManyLanes : kFewLanes; }
size_t one_scored_smem(int32_t T, int32_t E, int32_t k, const RouteScores &q) {
    const int per = 32 / one_lanes(T), tokens = (std::max(T, 1) + per - 1) / per * per;
    return scored_smem(tokens, E, k, q) + (size_t)2 * E * (kOneTokens / 32 + 1) * 4;
}
template <typename T, int S, int L>
cudaError_t route_one_scored(const MoeScoredParams &p, int wide, size_t smem, cudaStream_t s) {
    static SmemLimit limit;
    const cudaError_t e = raise_smem_limit(limit, (const void *)route_one_scored_kernel<T, S, L>, kOneSmem);
    if (e != cudaSuccess) return e;
    constexpr int per = 32 / L;
    const int tokens = (std::max(p.T, 1) + per - 1) / per * per;
    return launch_after(route_one_scored_kernel<T, S, L>, 1, std::max(L * tokens, 256), smem, s, p, wide, tokens);
}
template <typename T, int S>
cudaError_t route_scored(const MoeScoredParams &r, cudaStream_t s) {
    MoeScoredParams p = r;
    const int wide = (uintptr_t)p.logits % 16 == 0 && p.ld * (int64_t)sizeof(T) % 16 == 0 && p.E * sizeof(T) % 16 == 0;
    const size_t one = one_scored_smem(p.T, p.E, p.k, p.scores);
    if (moe_route_in_one(p.T, p.E) && one <= (size_t)kOneSmem)
        return one_lanes(p.T) == kManyLanes ? route_one_scored<T, S, kManyLanes>(p, wide, one, s) : route_one_scored<T, S, kFewLanes>(p, wide, one, s);
    // few tokens whose ranks have no room in one CTA: a single chunk, whose counts the one placing CTA reads before it writes offsets
    if (moe_route_in_one(p.T, p.E)) p.counts = p.offsets;
    constexpr int kTokens = select_tokens(S), kChunk = chunk_tokens(S);
    // (a CTA's most: rows, ranks of 32 groups, biases, experts and weights, counts)
    constexpr int kMost = (kTokens * (kGroups * S + 4 + 65 + 2 * (kRouteMaxTop | 1)) + 2 * kGroups * S) * 4;
    static_assert(kMost <= 200 * 1024, "shared memory of a selecting CTA");
    const int32_t chunks = (int32_t)((p.T + (int64_t)kChunk - 1) / kChunk);
    const size_t smem = scored_smem(kTokens, p.E, p.k | 1, p.scores) + p.E * 4;
    auto select = [&](auto kernel, SmemLimit &limit, int lanes) {
        const cudaError_t e = raise_smem_limit(limit, (const void *)kernel, kMost);
        return e != cudaSuccess ? e : launch_after(kernel, chunks * kSelectCtas, kTokens * lanes, smem, s, p, wide);
    };
    // Four lanes a token for tokens that fill few CTAs, where a token's chain counts; two where warps do (128 experts, biases, groups: 4800 tokens
    // 26.8 us with four and 30.1 with two, 65536 51.6 and 47.3; 512 experts, biases: 4800 33.8 and 44.5, 19200 61.2 and 56.7).
    static SmemLimit two, four;
    const cudaError_t e =
        2 * chunks * kSelectCtas <= 3 * sm_count() ? select(route_scored_kernel<T, S, 4>, four, 4) : select(route_scored_kernel<T, S, 2>, two, 2);
    if (e != cudaSuccess) return e;
    return launch_moe_place(p, kChunk, s);
}
}  // namespace

template <typename T>
cudaError_t launch_route_scored(const MoeScoredParams &p, cudaStream_t s) {
    switch (group_size(p.E)) {
        case 4: return route_scored<T, 4>(p, s);
        case 8: return route_scored<T, 8>(p, s);
        case 16: return route_scored<T, 16>(p, s);
        default: return route_scored<T, 32>(p, s);
    }
}

}  // namespace ilw
