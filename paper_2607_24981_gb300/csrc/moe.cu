// moe.cu -- routing of tokens to experts and the weighted join of the experts' rows.
//
// Routing: a row's k largest logits (equal ones by index; -inf and NaN are never taken), their softmax, and the
// order in which the experts' products want the rows: by expert, and by token within an expert.  That order is a
// counting sort over chunks of tokens: the first kernel selects, and counts the tokens of its chunk that each expert
// gets; the second finds its chunk's places from the counts of all chunks.  A token names an expert at most
// once, so within a chunk an entry's place is the number of earlier tokens in its expert's bitmap: the same
// whatever order the bits were set in.  Calls of one chunk do both in one kernel.
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

constexpr int kRouteThreads = 1024, kRouteWarps = kRouteThreads / 32;
constexpr int kMaxChunk = 1024;  // tokens a chunk at most
constexpr int kOneChunk = 256;   // tokens that one CTA takes alone

// Tokens a chunk: all of a small call, else a multiple of 32 that gives each SM about one.
inline int32_t chunk_tokens(int32_t T) {
    if (T <= kOneChunk) return kOneChunk;
    const int32_t c = (T / 148 + 31) / 32 * 32;
    return c < 32 ? 32 : c > kMaxChunk ? kMaxChunk : c;
}

// Order-preserving bits of a logit; 0 for one that is never taken.
__device__ __forceinline__ uint32_t order_bits(float x) {
    if (!(x > __int_as_float(0xff800000))) return 0;
    x += 0.0f;  // -0 equals +0
    const uint32_t u = __float_as_uint(x);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_order_bits(uint32_t u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }

// The largest k of one token's logits by one warp, V of them a lane (expert 32 i + lane): each lane sorts its own (equal
// ones by index, as they come), then the largest head of the 32 lanes is taken k times.  Lane j returns the
// j-th selection's expert (-1: none) and weight.
template <typename T, int V>
__device__ __forceinline__ void select_token(const MoeRouteParams &p, const T *x, int lane, int32_t &expert, float &weight) {
    uint32_t u[V], id[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = 32 * i + lane;
        u[i] = e < p.E ? order_bits(to_f(x[e])) : 0;
        id[i] = e;
    }
#pragma unroll
    for (int n = 0; n < V; ++n)  // odd-even transposition: neighbours only, so equal values keep their order
#pragma unroll
        for (int i = n & 1; i + 1 < V; i += 2) {
            const bool swap = u[i + 1] > u[i];
            const uint32_t a = u[i], c = id[i];
            u[i] = swap ? u[i + 1] : a;
            id[i] = swap ? id[i + 1] : c;
            u[i + 1] = swap ? a : u[i + 1];
            id[i + 1] = swap ? c : id[i + 1];
        }
    const uint32_t top = __reduce_max_sync(0xffffffffu, u[0]);
    const float mx = from_order_bits(top);
    float sum = 0.0f;
    if (!p.renormalize && top) {  // over every expert of the row
#pragma unroll
        for (int i = 0; i < V; ++i) sum += u[i] ? __expf(from_order_bits(u[i]) - mx) : 0.0f;
#pragma unroll
        for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    expert = -1;
    uint32_t got = 0;
    for (int j = 0; j < p.k; ++j) {
        const uint32_t m = __reduce_max_sync(0xffffffffu, u[0]);
        if (!m) break;
        const uint32_t who = __ballot_sync(0xffffffffu, u[0] == m);
        uint32_t e = __shfl_sync(0xffffffffu, id[0], __ffs(who) - 1);
        if (who & (who - 1)) e = __reduce_min_sync(0xffffffffu, u[0] == m ? id[0] : 0xffffffffu);
        if (lane == j) got = m, expert = (int32_t)e;
        if (id[0] == e) {
#pragma unroll
            for (int i = 0; i + 1 < V; ++i) u[i] = u[i + 1], id[i] = id[i + 1];
            u[V - 1] = 0;
            if (V == 1) id[0] = 0xffffffffu;
        }
    }
    weight = expert < 0 ? 0.0f : __expf(from_order_bits(got) - mx);
    if (p.renormalize) {
        sum = weight;
#pragma unroll
        for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);  // (k <= 16: lanes 0 to 15 hold them all)
    }
    if (expert >= 0) weight /= sum;
}

// Places of a chunk's entries, experts[n] (token i / k of the chunk): base[e] + the earlier tokens of e in the chunk.
// bits [E][words + 1]: bitmaps, and their words' running counts in pre.
__device__ __forceinline__ void place_chunk(const MoeRouteParams &p, int32_t t0, int32_t t1, int words, uint32_t *bits, int32_t *pre,
                                            const int32_t *base) {
    const int n = (t1 - t0) * p.k, row = words + 1;  // (an odd number of words a row apart: no bank met by all)
    const int32_t *expert = p.expert + (int64_t)t0 * p.k;
    for (int i = threadIdx.x; i < n; i += kRouteThreads) {
        const int32_t e = expert[i], t = i / p.k;
        if (e >= 0) atomicOr(&bits[e * row + (t >> 5)], 1u << (t & 31));
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += kRouteThreads) {
        int32_t sum = base[e];
        for (int w = 0; w < words; ++w) {
            pre[e * row + w] = sum;
            sum += __popc(bits[e * row + w]);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kRouteThreads) {
        const int32_t e = expert[i], t = i / p.k;
        int32_t s = -1;
        if (e >= 0) {
            s = pre[e * row + (t >> 5)] + __popc(bits[e * row + (t >> 5)] & ((1u << (t & 31)) - 1));
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

// ONE: the call is one chunk, placed by the same CTA.
template <typename T, int V, bool ONE>
__global__ void __launch_bounds__(kRouteThreads) route_select_kernel(const MoeRouteParams p, int32_t chunk) {
    extern __shared__ uint32_t dyn[];  // ONE: bits and pre
    __shared__ int32_t count[kRouteMaxExperts], base[ONE ? kRouteMaxExperts : 1], all;
    for (int e = threadIdx.x; e < p.E; e += kRouteThreads) count[e] = 0;
    const int words = chunk / 32, row = words + 1;
    if (ONE)
        for (int i = threadIdx.x; i < p.E * row; i += kRouteThreads) dyn[i] = 0;
    grid_wait();
    __syncthreads();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t t0 = blockIdx.x * chunk, t1 = min(p.T, t0 + chunk);
    for (int32_t t = t0 + warp; t < t1; t += kRouteWarps) {
        int32_t e;
        float w;
        select_token<T, V>(p, (const T *)p.logits + (int64_t)t * p.ld, lane, e, w);
        if (lane < p.k) {
            p.expert[(int64_t)t * p.k + lane] = e;
            p.weight[(int64_t)t * p.k + lane] = w;
            if (e >= 0) atomicAdd(&count[e], 1);  // (whole numbers: any order gives the same)
        }
    }
    __syncthreads();
    if (!ONE) {
        for (int e = threadIdx.x; e < p.E; e += kRouteThreads) p.counts[(int64_t)blockIdx.x * p.E + e] = count[e];
        return;
    }
    if (warp == 0) {
        const int32_t n = scan_experts(p.E, count, base, lane);
        if (lane == 0) all = n;
    }
    __syncthreads();
    for (int e = threadIdx.x; e <= p.E; e += kRouteThreads) p.offsets[e] = e < p.E ? base[e] : all;
    place_chunk(p, t0, t1, words, dyn, (int32_t *)dyn + p.E * row, base);
    for (int i = all + threadIdx.x; i < p.T * p.k; i += kRouteThreads) p.source[i] = -1;
}

__global__ void __launch_bounds__(kRouteThreads) route_place_kernel(const MoeRouteParams p, int32_t chunk, int32_t chunks) {
    extern __shared__ uint32_t bits[];  // [E][words + 1], then as many running counts
    __shared__ int32_t total[kRouteMaxExperts], before[kRouteMaxExperts], base[kRouteMaxExperts], all;
    const int words = chunk / 32, row = words + 1;
    for (int i = threadIdx.x; i < p.E * row; i += kRouteThreads) bits[i] = 0;
    for (int e = threadIdx.x; e < p.E; e += kRouteThreads) total[e] = before[e] = 0;
    __syncthreads();
    grid_wait();
    // counts of each expert in all chunks and in those before this one: as many threads an expert as there are
    const int wide = (p.E + 31) & ~31, groups = kRouteThreads / wide;
    const int e = threadIdx.x % wide, g = threadIdx.x / wide;
    if (e < p.E && g < groups) {
        int32_t a = 0, b = 0;
#pragma unroll 8
        for (int c = g; c < chunks; c += groups) {
            const int32_t n = p.counts[(int64_t)c * p.E + e];
            a += n;
            if (c < (int)blockIdx.x) b += n;
        }
        atomicAdd(&total[e], a);
        atomicAdd(&before[e], b);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int32_t n = scan_experts(p.E, total, base, threadIdx.x);
        if (threadIdx.x == 0) all = n;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.E; i += kRouteThreads) {
        if (blockIdx.x == 0) p.offsets[i] = base[i];
        base[i] += before[i];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = all;
    place_chunk(p, blockIdx.x * chunk, min(p.T, (int32_t)(blockIdx.x + 1) * chunk), words, bits, (int32_t *)bits + p.E * row, base);
    // places past the last entry name no token
    for (int64_t i = all + blockIdx.x * (int64_t)kRouteThreads + threadIdx.x; i < (int64_t)p.T * p.k; i += (int64_t)gridDim.x * kRouteThreads)
        p.source[i] = -1;
}

constexpr int kPlaceSmem = 2 * kRouteMaxExperts * (kMaxChunk / 32 + 1) * 4;  // 132 KB at most
size_t place_smem(int32_t E, int32_t chunk) { return (size_t)2 * E * (chunk / 32 + 1) * 4; }

template <typename T, int V>
cudaError_t select(const MoeRouteParams &p, int32_t chunk, int32_t chunks, cudaStream_t s) {
    if (chunks > 1) return launch_after(route_select_kernel<T, V, false>, chunks, kRouteThreads, 0, s, p, chunk);
    static_assert(2 * kRouteMaxExperts * (kOneChunk / 32 + 1) * 4 <= 44 * 1024, "a one-chunk call needs no raised limit");
    return launch_after(route_select_kernel<T, V, true>, 1, kRouteThreads, place_smem(p.E, chunk), s, p, chunk);
}
template <typename T>
cudaError_t select_form(const MoeRouteParams &p, int32_t chunk, int32_t chunks, cudaStream_t s) {
    if (p.E <= 32) return select<T, 1>(p, chunk, chunks, s);
    if (p.E <= 64) return select<T, 2>(p, chunk, chunks, s);
    if (p.E <= 128) return select<T, 4>(p, chunk, chunks, s);
    if (p.E <= 256) return select<T, 8>(p, chunk, chunks, s);
    return select<T, 16>(p, chunk, chunks, s);
}

// out[t, c] = (res[t, c] +) sum_j weight[t, j] Y[slot[t, j], c], j ascending, in fp32.
template <typename T, int VEC>
__global__ void __launch_bounds__(256) combine_kernel(const MoeCombineParams p) {
    grid_wait();
    struct alignas(VEC * sizeof(T)) Pack {
        T t[VEC];
    };
    const int32_t per = (p.N + VEC - 1) / VEC;
    for (int32_t t = blockIdx.y; t < p.T; t += gridDim.y) {
        for (int32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < per; i += gridDim.x * blockDim.x) {
            const int64_t c = (int64_t)i * VEC;
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
}

template <typename T>
cudaError_t combine(const MoeCombineParams &p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    auto fits = [&](const void *q, int64_t ld) { return (uintptr_t)q % 16 == 0 && ld % V == 0; };
    const bool vec = p.N % V == 0 && fits(p.Y, p.ldy) && fits(p.out, p.ldo) && (!p.res || fits(p.res, p.ldr));
    const int32_t per = vec ? p.N / V : p.N;
    const int threads = per >= 256 ? 256 : (per + 31) / 32 * 32;
    const dim3 grid((unsigned)((per + threads - 1) / threads), (unsigned)std::min(p.T, 65535));
    if (vec) return launch_after(combine_kernel<T, V>, grid, threads, 0, s, p);
    return launch_after(combine_kernel<T, 1>, grid, threads, 0, s, p);
}

}  // namespace

static int32_t route_chunks(int32_t T) { return std::max(1, (int32_t)((T + (int64_t)chunk_tokens(T) - 1) / chunk_tokens(T))); }

size_t moe_route_workspace(int32_t T, int32_t E) {
    const int32_t chunks = route_chunks(T);
    return chunks > 1 ? (size_t)chunks * E * sizeof(int32_t) : 0;
}

cudaError_t launch_moe_route(const MoeRouteParams &p, cudaStream_t s) {
    const int32_t chunk = chunk_tokens(p.T), chunks = route_chunks(p.T);
    cudaError_t e;
    if (p.form == ILW_FP32) e = select_form<float>(p, chunk, chunks, s);
    else if (p.form == ILW_FP16) e = select_form<__half>(p, chunk, chunks, s);
    else e = select_form<__nv_bfloat16>(p, chunk, chunks, s);
    if (e != cudaSuccess || chunks == 1) return e;
    static SmemLimit limit;
    e = raise_smem_limit(limit, (const void *)route_place_kernel, kPlaceSmem);
    if (e != cudaSuccess) return e;
    return launch_after(route_place_kernel, chunks, kRouteThreads, place_smem(p.E, chunk), s, p, chunk, chunks);
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
