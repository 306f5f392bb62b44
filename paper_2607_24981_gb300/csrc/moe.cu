// moe.cu -- routing of tokens to experts and the weighted join of the experts' rows.
//
// Routing: a row's k largest logits (equal ones by index; -inf and NaN are never taken), their softmax, and the
// order in which the experts' products want the rows: by expert, and by token within an expert.
//
// Selection: two lanes a token (four in calls of few tokens), its row in shared memory, its experts in 16 groups of
// consecutive ones, of which they know the largest logit.  The k times the largest group is found and scanned again
// without what was taken: some 155 instructions a token, where a warp a token, with its warp-wide maxima, took 525.
// 65536 rows of 128 fp32 logits, 8 taken: 30 us with the order (the bytes take 6 us).  Bound by latency: the rows in shared
// memory leave room for five CTAs, 20 warps, an SM, whose schedulers issue in 42 of 100 cycles, and 1024 CTAs are one round
// of 760 and a third of one.
//
// Order: a counting sort over chunks of 512 tokens (256 where rows are long), one to a cluster of 8 CTAs.  The first kernel selects, and
// adds up in distributed shared memory how many tokens of the chunk each expert gets; the second finds its chunk's places from
// the counts of all chunks (each placing CTA reads them: T^2 E / 2^18 words in all, from the L2; 8 MB of 65536 tokens and 128
// experts, but 2 GB of a million tokens).  A token names an expert at most once, so within a chunk an entry's place is the number
// of earlier tokens in its expert's bitmap: the same whatever order the bits were set in.  Calls of few tokens do
// both in one CTA.
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
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

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

// exp(x - best) of 4 N values, added up in four parts and pairwise.
template <int N>
__device__ __forceinline__ float4 sum_exp(const float4 *x, float best) {
    if constexpr (N == 1) {
        return make_float4(expf(x->x - best), expf(x->y - best), expf(x->z - best), expf(x->w - best));
    } else {
        const float4 a = sum_exp<N / 2>(x, best), b = sum_exp<N / 2>(x + N / 2, best);
        return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w);
    }
}

// The k largest of a token's row by L lanes (lane q of them here; all 32 lanes of the warp call it): its experts and weights to
// out_e and out_w, in order.  `row` loses what is taken.
template <int L, int S>
__device__ __forceinline__ void select_token(const MoeRouteParams &p, float *row, int q, int32_t *out_e, float *out_w) {
    constexpr int G = kGroups / L;  // this lane's groups: q, q + L, ...
    const float none = __int_as_float(0xff800000);
    float top[G], best = none;
#pragma unroll
    for (int i = 0; i < G; ++i) {
        const float4 *x = (const float4 *)(row + (L * i + q) * S);
        float m = none;
#pragma unroll
        for (int c = 0; c < S / 4; ++c) m = fmaxf(fmaxf(fmaxf(m, x[c].x), fmaxf(x[c].y, x[c].z)), x[c].w);
        top[i] = m;
        best = fmaxf(best, m);
    }
#pragma unroll
    for (int d = 1; d < L; d <<= 1) best = fmaxf(best, __shfl_xor_sync(0xffffffffu, best, d));
    float sum = 0.0f;
    if (!p.renormalize && best > none) {  // over every expert of the row, by group and in four parts: short chains of roundings
        float4 part = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
        for (int i = 0; i < G; ++i) {
            const float4 *x = (const float4 *)(row + (L * i + q) * S);
            const float4 of = sum_exp<S / 4>(x, best);
            part.x += of.x, part.y += of.y, part.z += of.z, part.w += of.w;
        }
        sum = (part.x + part.y) + (part.z + part.w);
    }
#pragma unroll
    for (int d = 1; d < L; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    for (int j = 0; j < p.k; ++j) {
        // the largest group, the first of equal ones
        float m = top[0];
        int g = 0;
#pragma unroll
        for (int i = 1; i < G; ++i)
            if (top[i] > m) m = top[i], g = i;
        g = L * g + q;
#pragma unroll
        for (int d = 1; d < L; d <<= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, d);
            const int g2 = __shfl_xor_sync(0xffffffffu, g, d);
            if (m2 > m || (m2 == m && g2 < g)) m = m2, g = g2;
        }
        const bool taken = m > none;
        if (taken && g % L == q) {  // its lane takes the first expert with that logit
            const float4 *x = (const float4 *)(row + g * S);
            int at = S;
            float rest = none;
#pragma unroll
            for (int c = 0; c < S / 4; ++c) {
                const float4 v = x[c];
                const float u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const bool hit = u[w] == m && at == S;
                    at = hit ? 4 * c + w : at;
                    rest = fmaxf(rest, hit ? none : u[w]);
                }
            }
            row[g * S + min(at, S - 1)] = none;
#pragma unroll
            for (int i = 0; i < G; ++i)
                if (i == g / L) top[i] = rest;
            out_e[j] = g * S + at;
            out_w[j] = expf(m - best);
        }
        if (!taken && q == 0) out_e[j] = -1, out_w[j] = 0.0f;
        if (L > 1) __syncwarp();
    }
    if (p.renormalize)
        for (int j = p.k - 1; j >= 0; --j) sum += out_w[j];  // (the small ones first)
    if (L > 1) __syncwarp();
    for (int j = q; j < p.k; j += L)
        if (out_e[j] >= 0) out_w[j] /= sum;
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

// Selection of a chunk's tokens by a cluster, and the chunk's counts.  Each warp loads its own tokens' rows.
template <typename T, int S>
__global__ void __cluster_dims__(kSelectCtas, 1, 1) __launch_bounds__(select_tokens(S) * kSelectLanes) route_select_kernel(const MoeRouteParams p, int wide) {
    extern __shared__ __align__(16) uint32_t dyn[];
    constexpr int kSelectTokens = select_tokens(S), kSelectThreads = kSelectTokens * kSelectLanes;
    constexpr int kStride = kGroups * S + 4, kWarpTokens = 32 / kSelectLanes;
    const int lane = threadIdx.x & 31, warp0 = (threadIdx.x >> 5) * kWarpTokens, mine = threadIdx.x / kSelectLanes;
    const int ks = p.k | 1;      // (an odd number of words a token: no bank met by all)
    float *rows = (float *)dyn;  // [tokens][stride], then experts and weights [tokens][ks], then counts [E]
    int32_t *out_e = (int32_t *)dyn + kSelectTokens * kStride;
    float *out_w = (float *)out_e + kSelectTokens * ks;
    int32_t *count = (int32_t *)out_w + kSelectTokens * ks;
    for (int e = threadIdx.x; e < p.E; e += kSelectThreads) count[e] = 0;
    grid_wait();
    const int32_t t0 = blockIdx.x * kSelectTokens;
    const int n = max(0, min(kSelectTokens, p.T - t0));
    load_rows<T, S>(p, t0 + warp0, max(0, min(kWarpTokens, n - warp0)), rows + warp0 * kStride, wide, lane);
    __syncwarp();
    if (warp0 < n) {
        clear_row<kSelectLanes, S>(rows + mine * kStride, mine < n);
        select_token<kSelectLanes, S>(p, rows + mine * kStride, lane % kSelectLanes, out_e + mine * ks, out_w + mine * ks);
    }
    __syncthreads();
    const uint32_t over_k = reciprocal(p.k);
    for (int i = threadIdx.x; i < n * p.k; i += kSelectThreads) {
        const int t = over(i, over_k), at = t * ks + i - t * p.k;
        const int32_t e = out_e[at];
        p.expert[(int64_t)t0 * p.k + i] = e;
        p.weight[(int64_t)t0 * p.k + i] = out_w[at];
        if (e >= 0) atomicAdd(&count[e], 1);  // (whole numbers: any order gives the same)
    }
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    const uint32_t rank = blockIdx.x % kSelectCtas, at = (uint32_t)__cvta_generic_to_shared(count);
    for (int e = rank * kSelectThreads + threadIdx.x; e < p.E; e += kSelectCtas * kSelectThreads) {
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

template <int W>  // words of a chunk's bitmap
__global__ void __launch_bounds__(kPlaceThreads) route_place_kernel(const MoeRouteParams p, int32_t chunks) {
    extern __shared__ uint32_t bits[];  // [E][words + 1], then as many running counts
    __shared__ int32_t total[kRouteMaxExperts], before[kRouteMaxExperts], base[kRouteMaxExperts], all;
    constexpr int kChunk = 32 * W, row = W + 1, kEntries = kChunk * kRouteMaxTop / kPlaceThreads;
    for (int i = threadIdx.x; i < p.E * row; i += kPlaceThreads) bits[i] = 0;
    for (int e = threadIdx.x; e < p.E; e += kPlaceThreads) total[e] = before[e] = 0;
    __syncthreads();
    grid_wait();
    const int32_t t0 = blockIdx.x * kChunk;
    const int n = min(kChunk, p.T - t0) * p.k;
    int32_t ex[kEntries];
#pragma unroll
    for (int j = 0; j < kEntries; ++j) ex[j] = j * kPlaceThreads + (int)threadIdx.x < n ? p.expert[(int64_t)t0 * p.k + j * kPlaceThreads + threadIdx.x] : -1;
    // counts of each expert in all chunks and in those before this one: as many threads an expert as there are
    const int span = (p.E + 31) & ~31, groups = kPlaceThreads / span;
    const int e = threadIdx.x % span, g = threadIdx.x / span;
    if (e < p.E && g < groups) {
        int32_t a = 0, b = 0;
#pragma unroll 16
        for (int c = g; c < chunks; c += groups) {
            const int32_t x = p.counts[(int64_t)c * p.E + e];
            a += x;
            if (c < (int)blockIdx.x) b += x;
        }
        atomicAdd(&total[e], a);
        atomicAdd(&before[e], b);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int32_t x = scan_experts(p.E, total, base, threadIdx.x);
        if (threadIdx.x == 0) all = x;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.E; i += kPlaceThreads) {
        if (blockIdx.x == 0) p.offsets[i] = base[i];
        base[i] += before[i];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = all;
    place_chunk<W>(p, t0, n, ex, bits, (int32_t *)bits + p.E * row, base);
    // places past the last entry name no token
    for (int64_t i = all + blockIdx.x * (int64_t)kPlaceThreads + threadIdx.x; i < (int64_t)p.T * p.k; i += (int64_t)gridDim.x * kPlaceThreads)
        p.source[i] = -1;
}

// Few tokens (a multiple of eight, at most 256, with the last ones filled up): all of it by one CTA, four threads a token and
// more for the order.
template <typename T, int S>
__global__ void __launch_bounds__(4 * kOneTokens) route_one_kernel(const MoeRouteParams p, int wide, int tokens) {
    extern __shared__ __align__(16) uint32_t dyn[];
    __shared__ int32_t base[kRouteMaxExperts], count[kRouteMaxExperts], all;
    constexpr int words = kOneTokens / 32, row = words + 1, kEntries = kRouteMaxTop / 4, kStride = kGroups * S + 4;
    const int mine = threadIdx.x >> 2, first = (threadIdx.x & ~31) / 4;  // the warp's eight tokens
    float *rows = (float *)dyn;  // [tokens][stride], then experts and weights [tokens][k], then bits [E][row] and the running counts
    int32_t *out_e = (int32_t *)rows + tokens * kStride;
    float *out_w = (float *)out_e + tokens * p.k;
    uint32_t *bits = (uint32_t *)out_w + tokens * p.k;
    for (int i = threadIdx.x; i < p.E * row; i += blockDim.x) bits[i] = 0;
    for (int e = threadIdx.x; e < p.E; e += blockDim.x) count[e] = 0;
    grid_wait();
    if (first < tokens) {
        load_rows<T, S>(p, first, max(0, min(8, p.T - first)), rows + first * kStride, wide, threadIdx.x & 31);
        __syncwarp();
        clear_row<4, S>(rows + mine * kStride, mine < p.T);
        select_token<4, S>(p, rows + mine * kStride, threadIdx.x & 3, out_e + mine * p.k, out_w + mine * p.k);
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

size_t select_smem(int32_t E, int32_t k) {
    return ((size_t)select_tokens(group_size(E)) * (row_words(E) + 2 * (k | 1)) + E) * 4;
}
size_t one_smem(int32_t T, int32_t E, int32_t k) {
    const size_t tokens = (std::max(T, 1) + 7) / 8 * 8;
    return ((size_t)2 * E * (kOneTokens / 32 + 1) + tokens * (2 * k + row_words(E))) * 4;
}
bool route_in_one(int32_t T, int32_t E) { return T <= kOneTokens && (int64_t)T * E <= kOneLogits && one_smem(T, E, kRouteMaxTop) <= kOneSmem; }

template <typename T, int S>
cudaError_t route(const MoeRouteParams &p, cudaStream_t s) {
    const int wide = (uintptr_t)p.logits % 16 == 0 && p.ld * (int64_t)sizeof(T) % 16 == 0 && p.E * sizeof(T) % 16 == 0;
    if (route_in_one(p.T, p.E)) {
        static SmemLimit limit;
        const cudaError_t e = raise_smem_limit(limit, (const void *)route_one_kernel<T, S>, kOneSmem);
        if (e != cudaSuccess) return e;
        const int tokens = (std::max(p.T, 1) + 7) / 8 * 8;
        return launch_after(route_one_kernel<T, S>, 1, std::max(4 * tokens, 256), one_smem(p.T, p.E, p.k), s, p, wide, tokens);
    }
    static SmemLimit limit;
    cudaError_t e = raise_smem_limit(limit, (const void *)route_select_kernel<T, S>, (int)select_smem(kGroups * S, kRouteMaxTop));
    if (e != cudaSuccess) return e;
    constexpr int kChunk = chunk_tokens(S), W = kChunk / 32;
    const int32_t chunks = (int32_t)((p.T + (int64_t)kChunk - 1) / kChunk);
    e = launch_after(route_select_kernel<T, S>, chunks * kSelectCtas, select_tokens(S) * kSelectLanes, select_smem(p.E, p.k), s, p, wide);
    if (e != cudaSuccess) return e;
    static_assert(2 * kGroups * S * (W + 1) * 4 + 3 * kRouteMaxExperts * 4 + 16 <= 48 * 1024, "route_place_kernel: no limit raised");
    return launch_after(route_place_kernel<W>, chunks, kPlaceThreads, (size_t)2 * p.E * (W + 1) * 4, s, p, chunks);
}
template <typename T>
cudaError_t route_form(const MoeRouteParams &p, cudaStream_t s) {
    switch (group_size(p.E)) {
        case 4: return route<T, 4>(p, s);
        case 8: return route<T, 8>(p, s);
        case 16: return route<T, 16>(p, s);
        default: return route<T, 32>(p, s);
    }
}

// out[t, c] = (res[t, c] +) sum_j weight[t, j] Y[slot[t, j], c], j ascending, in fp32.  Bound by HBM: 16384 tokens of 8 rows of 4096
// bf16 take 204 us (5.9 TB/s) in pieces of 16 bytes; rows off 16-byte boundaries go value by value: 1033 us of 4097, bound by the latency
// of one load of 2 bytes in flight a thread.
// Four rows in flight a thread instead of what the CTAs of an SM have among them: 283 us.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) combine_kernel(const MoeCombineParams p) {
    grid_wait();
    struct alignas(VEC * sizeof(T)) Pack {
        T t[VEC];
    };
    // the grid covers a row; tokens go round in 32 bits without a sign, which T and a grid's height together do not pass
    const uint32_t i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (uint32_t)p.N / VEC) return;
    const int64_t c = (int64_t)i * VEC;
    for (uint32_t t = blockIdx.y; t < (uint32_t)p.T; t += gridDim.y) {
        float acc[VEC];
#pragma unroll
        for (int u = 0; u < VEC; ++u) acc[u] = 0.0f;
        for (int j = 0; j < p.k; ++j) {
            const int32_t s = p.slot[(int64_t)t * p.k + j];
            if (s < 0 || s >= p.rows) {
                if (s != -1 && p.status && i == 0) atomicExch(p.status, kStatusBadIndex);
                continue;
            }
            const float w = p.weight[(int64_t)t * p.k + j];
            const Pack y = *(const Pack *)((const T *)p.Y + s * p.ldy + c);
#pragma unroll
            for (int u = 0; u < VEC; ++u) acc[u] = fmaf(w, to_f(y.t[u]), acc[u]);
        }
        if (p.res) {
            const Pack r = *(const Pack *)((const T *)p.res + t * p.ldr + c);
#pragma unroll
            for (int u = 0; u < VEC; ++u) acc[u] += to_f(r.t[u]);
        }
        Pack o;
#pragma unroll
        for (int u = 0; u < VEC; ++u) o.t[u] = from_f<T>(acc[u]);
        *(Pack *)((T *)p.out + t * p.ldo + c) = o;
    }
}

template <typename T>
cudaError_t combine(const MoeCombineParams &p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    auto fits = [&](const void *q, int64_t ld) { return (uintptr_t)q % 16 == 0 && ld % V == 0; };
    const bool vec = p.N % V == 0 && fits(p.Y, p.ldy) && fits(p.out, p.ldo) && (!p.res || fits(p.res, p.ldr));
    const int64_t per = vec ? p.N / V : p.N;
    const int threads = per >= 256 ? 256 : (int)(per + 31) / 32 * 32;
    const dim3 grid((unsigned)((per + threads - 1) / threads), (unsigned)std::min(p.T, 65535));
    if (vec) return launch_after(combine_kernel<T, V>, grid, threads, 0, s, p);
    return launch_after(combine_kernel<T, 1>, grid, threads, 0, s, p);
}

}  // namespace

size_t moe_route_workspace(int32_t T, int32_t E) {
    const int64_t chunk = chunk_tokens(group_size(E));
    return route_in_one(T, E) ? 0 : (size_t)((T + chunk - 1) / chunk) * E * sizeof(int32_t);
}

cudaError_t launch_moe_route(const MoeRouteParams &p, cudaStream_t s) {
    if (p.form == ILW_FP32) return route_form<float>(p, s);
    if (p.form == ILW_FP16) return route_form<__half>(p, s);
    return route_form<__nv_bfloat16>(p, s);
}

cudaError_t launch_moe_combine(const MoeCombineParams &q, cudaStream_t s) {
    if (q.T == 0 || q.N == 0) return cudaSuccess;
    MoeCombineParams p = q;
    p.status = status_word_ptr();
    if (p.form == ILW_FP32) return combine<float>(p, s);
    if (p.form == ILW_FP16) return combine<__half>(p, s);
    return combine<__nv_bfloat16>(p, s);
}

}  // namespace ilw
