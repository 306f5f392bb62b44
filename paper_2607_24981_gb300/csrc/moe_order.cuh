// moe_order.cuh -- what routing kernels share (moe.cu, moe_scored.cuh): the sizes of chunks, tokens' rows in shared memory and the places of entries.
#pragma once
#include <algorithm>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "mx_kernels.h"

namespace ilw {
namespace {

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
// Two lanes a token (65536 rows of 128, 8 experts: 30 us with the order; 31 with four, 38 with one), 64 tokens a CTA; 32 where
// 64 rows are all of an SM's shared memory (8192 rows of 512: 24 us instead of 41).
constexpr int kSelectLanes = 2, kSelectCtas = 8;
__host__ __device__ constexpr int select_tokens(int S) { return S >= 32 ? 32 : 64; }
__host__ __device__ constexpr int chunk_tokens(int S) { return select_tokens(S) * kSelectCtas; }
constexpr int kPlaceThreads = 1024;
// What one CTA takes alone (one kernel and two, in us: 16 tokens of 64 experts 3.6 and 7.6, 256 of 64 7.1 and 8.1, 128 of 256 11.1 and
// 12.1, 224 of 128 10.6 and 10.4, 256 of 128 11.6 and 10.7)
constexpr int kOneTokens = 256, kOneLogits = 32 * 1024 - 4096, kOneSmem = 200 * 1024;
constexpr int kGroups = 16;

// Experts a group (4, 8, 16 or 32), and words between the rows of the tokens' logits in shared memory: 16 groups, filled up with
// -inf, and one more piece of 16 bytes, so that pieces of eight rows in a row meet in no bank.
__host__ __device__ inline int group_size(int E) { return E <= 64 ? 4 : E <= 128 ? 8 : E <= 256 ? 16 : 32; }
__host__ __device__ inline int row_words(int E) { return kGroups * group_size(E) + 4; }

// i / k for i < 2^13 and k <= 16: i * ceil(2^17 / k) / 2^17 (the rounding adds less than i / 2^17 < 1 / k)
__device__ __forceinline__ uint32_t reciprocal(int k) { return ((1u << 17) + k - 1) / k; }
__device__ __forceinline__ int over(int i, uint32_t r) { return (int)(((uint64_t)(uint32_t)i * r) >> 17); }
// A logit as it is compared: -inf for what is never taken.
__device__ __forceinline__ float logit(float x) { return x > __int_as_float(0xff800000) ? x : __int_as_float(0xff800000); }

// n rows of the logits from token t0 on to shared memory, by one warp; 16 bytes of them at a time where rows allow it
// (65536 rows of 128: 30 us, else 82; 257 rows 11 and 21).
template <typename T, int S>
__device__ __forceinline__ void load_rows(const MoeRouteParams &p, int32_t t0, int n, float *rows, bool wide, int lane) {
    constexpr int V = 16 / sizeof(T), kWords = kGroups * S, kStride = kWords + 4;
    const float none = __int_as_float(0xff800000);
    const T *x = (const T *)p.logits + (int64_t)t0 * p.ld;
    if (wide) {
        struct alignas(16) Pack {
            T v[V];
        };
        for (int c = lane * V; c < kWords; c += 32 * V) {
#pragma unroll 8
            for (int t = 0; t < n; ++t) {
                Pack y;
                if (c < p.E) y = *(const Pack *)(x + t * p.ld + c);
#pragma unroll
                for (int j = 0; j < V; j += 4)
                    *(float4 *)(rows + t * kStride + c + j) =
                        c < p.E ? make_float4(logit(to_f(y.v[j])), logit(to_f(y.v[j + 1])), logit(to_f(y.v[j + 2])), logit(to_f(y.v[j + 3])))
                                : make_float4(none, none, none, none);
            }
        }
    } else {
        for (int c = lane; c < kWords; c += 32) {
#pragma unroll 8
            for (int t = 0; t < n; ++t) rows[t * kStride + c] = c < p.E ? logit(to_f(x[t * p.ld + c])) : none;
        }
    }
}

// A row past the last token (the rest of its warp has one): nothing to select from.
template <int L, int S>
__device__ __forceinline__ void clear_row(float *row, bool is_token) {
    if (!is_token)
        for (int c = threadIdx.x % L; c < kGroups * S; c += L) row[c] = __int_as_float(0xff800000);
    __syncwarp();
}

// Places of a chunk's entries: base[e] + the earlier tokens of e in the chunk.  Entry i of the chunk (token i / k) is ex[i / threads] of
// thread i % threads.  bits [E][W + 1]: bitmaps of W words, and their words' running counts in pre.
template <int W, int N>
__device__ __forceinline__ void place_chunk(const MoeRouteParams &p, int32_t t0, int n, const int32_t (&ex)[N], uint32_t *bits,
                                            int32_t *pre, const int32_t *base) {
    constexpr int row = W + 1;  // (an odd number of words a row apart: no bank met by all)
    const uint32_t over_k = reciprocal(p.k);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = j * blockDim.x + threadIdx.x, t = over(i, over_k);
        if (i < n && ex[j] >= 0) atomicOr(&bits[ex[j] * row + (t >> 5)], 1u << (t & 31));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < (p.E * W + 31) / 32 * 32; i += blockDim.x) {  // W lanes a bitmap
        const int e = i / W, w = i % W;
        const int32_t c = e < p.E ? __popc(bits[e * row + w]) : 0;
        int32_t x = c;
#pragma unroll
        for (int d = 1; d < W; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, x, d, W);
            if (w >= d) x += y;
        }
        if (e < p.E) pre[e * row + w] = base[e] + x - c;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int i = j * blockDim.x + threadIdx.x, t = over(i, over_k);
        if (i >= n) break;
        int32_t s = -1;
        if (ex[j] >= 0) {
            const int at = ex[j] * row + (t >> 5);
            s = pre[at] + __popc(bits[at] & ((1u << (t & 31)) - 1));
            p.source[s] = t0 + t;
        }
        p.slot[(int64_t)t0 * p.k + i] = s;
    }
}

// Exclusive sums over the experts of total[e] (shared, E <= 512) into base[e] by one warp; returns the sum of all.
__device__ __forceinline__ int32_t scan_experts(int E, const int32_t *total, int32_t *base, int lane) {
    int32_t carry = 0;
    for (int e0 = 0; e0 < E; e0 += 32) {
        const int e = e0 + lane;
        const int32_t n = e < E ? total[e] : 0;
        int32_t x = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (e < E) base[e] = carry + x - n;
        carry += __shfl_sync(0xffffffffu, x, 31);
    }
    return carry;
}

// The counts of a cluster's CTAs, added up, to their chunk's.
template <int kThreads>
__device__ __forceinline__ void add_counts(const MoeRouteParams &p, const int32_t *count) {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    const uint32_t rank = blockIdx.x % kSelectCtas, at = (uint32_t)__cvta_generic_to_shared(count);
    for (int e = rank * kThreads + threadIdx.x; e < p.E; e += kSelectCtas * kThreads) {
        int32_t sum = 0;
#pragma unroll
        for (int r = 0; r < kSelectCtas; ++r) {
            uint32_t a;
            int32_t c;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at + 4 * e), "r"(r));
            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(c) : "r"(a) : "memory");
            sum += c;
        }
        p.counts[(int64_t)(blockIdx.x / kSelectCtas) * p.E + e] = sum;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

}  // namespace
}  // namespace ilw
