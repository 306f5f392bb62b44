// moe.cu -- routing of tokens to experts and the weighted join of the experts' rows.
//
// Routing: a row's k largest logits (equal ones by index; -inf and NaN are never taken), their softmax, and the
// order in which the experts' products want the rows: by expert, and by token within an expert.  That order is a
// counting sort in two kernels.  The first selects and counts the tokens of each chunk that each expert gets;
// the second finds its chunk's places from the counts of the chunks before it.  A token names an expert at most
// once, so within a chunk an entry's place is the number of earlier tokens in its expert's bitmap: the same
// whatever order the bits were set in.
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

constexpr int kRouteThreads = 256;
constexpr int kMaxChunk = 1024;  // tokens a chunk at most

// Tokens a chunk: a multiple of 32, about 128 chunks.
__host__ __device__ inline int32_t chunk_tokens(int32_t T) {
    int32_t c = (T / 128 + 31) / 32 * 32;
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

// One warp a token, V logits a lane (expert 32 i + lane).
template <typename T, int V>
__global__ void __launch_bounds__(kRouteThreads) route_select_kernel(const MoeRouteParams p, int32_t chunk) {
    extern __shared__ int32_t count[];  // [E]
    grid_wait();
    for (int e = threadIdx.x; e < p.E; e += kRouteThreads) count[e] = 0;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const int32_t t1 = min(p.T, (int32_t)(blockIdx.x + 1) * chunk);
    for (int32_t t = blockIdx.x * chunk + (threadIdx.x >> 5); t < t1; t += kRouteThreads / 32) {
        uint32_t u[V];
        uint32_t best = 0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int e = 32 * i + lane;
            u[i] = e < p.E ? order_bits(to_f(((const T *)p.logits)[(int64_t)t * p.ld + e])) : 0;
            best = max(best, u[i]);
        }
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        const float mx = from_order_bits(top);
        float sum = 0.0f;
        if (!p.renormalize && top) {  // over every expert of the row
#pragma unroll
            for (int i = 0; i < V; ++i) sum += u[i] ? expf(from_order_bits(u[i]) - mx) : 0.0f;
#pragma unroll
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        }
        float mine = 0.0f;  // lane j keeps the j-th selection
        int32_t mine_e = -1;
        for (int j = 0; j < p.k; ++j) {
            const uint32_t m = __reduce_max_sync(0xffffffffu, best);
            if (!m) break;
            int32_t at = 0x7fffffff;
#pragma unroll
            for (int i = V - 1; i >= 0; --i)
                if (u[i] == m) at = 32 * i + lane;
            const int32_t e = __reduce_min_sync(0xffffffffu, at);
            const float w = expf(from_order_bits(m) - mx);
            if (p.renormalize) sum += w;
            if (lane == j) mine = w, mine_e = e;
            if (lane == (e & 31)) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (32 * i + lane == e) u[i] = 0;
                best = 0;
#pragma unroll
                for (int i = 0; i < V; ++i) best = max(best, u[i]);
            }
        }
        if (lane < p.k) {
            p.expert[(int64_t)t * p.k + lane] = mine_e;
            p.weight[(int64_t)t * p.k + lane] = mine_e < 0 ? 0.0f : mine / sum;
            if (mine_e >= 0) atomicAdd(&count[mine_e], 1);  // (whole numbers: any order gives the same)
        }
    }
    __syncthreads();
    for (int e = threadIdx.x; e < p.E; e += kRouteThreads) p.counts[(int64_t)blockIdx.x * p.E + e] = count[e];
}

__global__ void __launch_bounds__(kRouteThreads) route_place_kernel(const MoeRouteParams p, int32_t chunk, int32_t chunks) {
    extern __shared__ uint32_t bits[];  // [E][words]: the chunk's tokens of each expert
    __shared__ int32_t base[kRouteMaxExperts], warp_sum[kRouteThreads / 32];
    grid_wait();
    const int words = chunk / 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t t0 = blockIdx.x * chunk, t1 = min(p.T, t0 + chunk);
    for (int i = threadIdx.x; i < p.E * words; i += kRouteThreads) bits[i] = 0;
    // base[e] = entries of experts before e, and those of e in earlier chunks
    int32_t carry = 0;
    for (int e0 = 0; e0 < p.E; e0 += kRouteThreads) {
        const int e = e0 + threadIdx.x;
        int32_t before = 0, total = 0;
        if (e < p.E) {
            for (int c = 0; c < chunks; ++c) {
                const int32_t n = p.counts[(int64_t)c * p.E + e];
                total += n;
                if (c < (int)blockIdx.x) before += n;
            }
        }
        int32_t x = total;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        if (lane == 31) warp_sum[warp] = x;
        __syncthreads();
        int32_t off = carry, all = carry;
        for (int w = 0; w < kRouteThreads / 32; ++w) {
            if (w < warp) off += warp_sum[w];
            all += warp_sum[w];
        }
        if (e < p.E) {
            base[e] = off + x - total + before;
            if (blockIdx.x == 0) p.offsets[e] = off + x - total;
        }
        carry = all;
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) p.offsets[p.E] = carry;
    const int32_t n = (t1 - t0) * p.k;
    for (int i = threadIdx.x; i < n; i += kRouteThreads) {
        const int32_t e = p.expert[(int64_t)t0 * p.k + i], t = i / p.k;
        if (e >= 0) atomicOr(&bits[e * words + (t >> 5)], 1u << (t & 31));
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kRouteThreads) {
        const int32_t e = p.expert[(int64_t)t0 * p.k + i], t = i / p.k;
        int32_t s = -1;
        if (e >= 0) {
            s = base[e];
            for (int w = 0; w < (t >> 5); ++w) s += __popc(bits[e * words + w]);
            s += __popc(bits[e * words + (t >> 5)] & ((1u << (t & 31)) - 1));
            p.source[s] = t0 + t;
        }
        p.slot[(int64_t)t0 * p.k + i] = s;
    }
    // places past the last entry name no token
    for (int64_t i = carry + blockIdx.x * (int64_t)kRouteThreads + threadIdx.x; i < (int64_t)p.T * p.k; i += (int64_t)gridDim.x * kRouteThreads)
        p.source[i] = -1;
}

template <typename T, int V>
cudaError_t select(const MoeRouteParams &p, int32_t chunk, int32_t chunks, cudaStream_t s) {
    return launch_after(route_select_kernel<T, V>, chunks, kRouteThreads, p.E * sizeof(int32_t), s, p, chunk);
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

size_t moe_route_workspace(int32_t T, int32_t E) {
    const int32_t chunk = chunk_tokens(T);
    return (size_t)std::max<int64_t>(1, (T + (int64_t)chunk - 1) / chunk) * E * sizeof(int32_t);
}

cudaError_t launch_moe_route(const MoeRouteParams &p, cudaStream_t s) {
    const int32_t chunk = chunk_tokens(p.T), chunks = std::max(1, (int32_t)((p.T + (int64_t)chunk - 1) / chunk));
    cudaError_t e;
    if (p.form == ILW_FP32) e = select_form<float>(p, chunk, chunks, s);
    else if (p.form == ILW_FP16) e = select_form<__half>(p, chunk, chunks, s);
    else e = select_form<__nv_bfloat16>(p, chunk, chunks, s);
    if (e != cudaSuccess) return e;
    const size_t smem = (size_t)p.E * (chunk / 32) * 4;  // at most 64 KB
    static SmemLimit limit;
    e = raise_smem_limit(limit, (const void *)route_place_kernel, 4 * kRouteMaxExperts * kMaxChunk / 32);
    if (e != cudaSuccess) return e;
    return launch_after(route_place_kernel, chunks, kRouteThreads, smem, s, p, chunk, chunks);
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
