// i8_few.cu -- products of int8 rows with float scales for few tokens: y = act(sa sw sum_k a w + bias), for one weight or for one
// weight per expert with ragged rows.
//
// A few tokens use every weight a few times, so what counts is the weights' stream.  A warp takes four rows of W and up to eight tokens
// and walks along K in steps of 512, every lane 16 bytes of each row; sums are whole numbers (dp4a, int32), so any split of K gives the
// same.  The warps of a CTA share its rows of W, or their K where there are too few rows of W to fill the SMs.
#include <algorithm>
#include <climits>
#include <cstdint>

#include "float_act.cuh"
#include "i8_kernels.h"
#include "ilw_kernels.h"
#include "ilwdetr.h"

namespace ilw {
namespace {

constexpr int kRows = 4, kTokens = 8, kWarps = 8;

struct FewParams {
    I8GemmProblem g;
    int32_t ksplit;    // warps that share K (1, 2, 4 or 8)
    int32_t nblocks;   // CTAs for all rows of W
    int64_t units;     // pieces of up to kTokens tokens at most
};

// 16 bytes of a row at k; bytes past K are zero and not read.
__device__ __forceinline__ int4 load16(const int8_t *row, int64_t k, int32_t K, bool on) {
    if (on && k + 16 <= K) return __ldg((const int4 *)(row + k));
    int4 v = make_int4(0, 0, 0, 0);
    if (on)
        for (int i = 0; k + i < K; ++i) ((int32_t *)&v)[i >> 2] |= (int32_t)(uint8_t)row[k + i] << (8 * (i & 3));
    return v;
}
__device__ __forceinline__ int32_t dot16(const int4 &a, const int4 &b, int32_t c) {
    return __dp4a(a.w, b.w, __dp4a(a.z, b.z, __dp4a(a.y, b.y, __dp4a(a.x, b.x, c))));
}

// This warp's part of K of rows n0 .. n0 + 3 of W and `T` tokens from row0 on (`rows` of them exist): the sums of (token t, row r) at
// index 4 t + r in lane index << (5 - log2(4 T)).
template <int T>
__device__ __forceinline__ int32_t sums(const FewParams &p, const int8_t *w, int32_t n0, int64_t row0, int rows, int part, int lane) {
    const I8GemmProblem &g = p.g;
    int32_t acc[kRows * T];
#pragma unroll
    for (int i = 0; i < kRows * T; ++i) acc[i] = 0;
    const int8_t *wr = w + (int64_t)n0 * g.w_ldc, *ar = g.a_codes + row0 * g.a_ldc;
#pragma unroll 2
    for (int64_t k = part * 512 + lane * 16; k < g.K; k += p.ksplit * 512) {
        int4 wv[kRows], av[T];
#pragma unroll
        for (int r = 0; r < kRows; ++r) wv[r] = load16(wr + r * g.w_ldc, k, g.K, n0 + r < g.N);
#pragma unroll
        for (int t = 0; t < T; ++t) av[t] = load16(ar + t * g.a_ldc, k, g.K, t < rows);
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int r = 0; r < kRows; ++r) acc[t * kRows + r] = dot16(wv[r], av[t], acc[t * kRows + r]);
    }
    __syncwarp();
    // lanes that differ in a bit exchange halves of their sums, then add what is left
    int d = 16;
#pragma unroll
    for (int n = kRows * T / 2; n >= 1; n /= 2, d /= 2) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const bool up = lane & d;
            const int32_t give = up ? acc[i] : acc[i + n], keep = up ? acc[i + n] : acc[i];
            acc[i] = keep + __shfl_xor_sync(0xffffffffu, give, d);
        }
    }
    for (; d >= 1; d /= 2) acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], d);
    return acc[0];
}

template <int ACT, typename T>
__global__ void __launch_bounds__(32 * kWarps) i8_few_kernel(const __grid_constant__ FewParams p) {
    __shared__ int32_t parts[kWarps][32];
    __shared__ int64_t s_row0;
    __shared__ int32_t s_rows, s_expert, s_head, s_tail;
    const I8GemmProblem &g = p.g;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t unit = blockIdx.x / p.nblocks;
    const int32_t block = (int32_t)(blockIdx.x - unit * p.nblocks);
    grid_wait();
    // this CTA's tokens: piece `unit` of the experts' rows, whose ranges are held in order, apart and inside [0, M]
    if (warp == 0) {
        const int32_t M = (int32_t)g.M;
        int32_t sum = 0, before = 0, head = M;
        int64_t row0 = 0;
        int32_t rows = 0, expert = 0;
        for (int e0 = 0; e0 < g.experts; e0 += 32) {
            const int e = e0 + lane;
            int32_t l = 0, h = e < g.experts ? M : 0;
            if (g.offsets && e < g.experts) {
                l = max(0, min(g.offsets[e], M));
                h = max(0, min(g.offsets[e + 1], M));
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t y = __shfl_up_sync(0xffffffffu, h, d);
                if (lane >= d) h = max(h, y);
            }
            h = max(h, before);
            const int32_t prev = __shfl_up_sync(0xffffffffu, h, 1);
            l = min(max(l, lane ? prev : before), h);
            if (e0 == 0) head = __shfl_sync(0xffffffffu, l, 0);
            before = __shfl_sync(0xffffffffu, h, 31);
            const int32_t n = e < g.experts ? (h - l + kTokens - 1) / kTokens : 0;
            int32_t x = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            const int64_t at = unit - sum - (x - n);  // the unit's number among this expert's
            const uint32_t hit = __ballot_sync(0xffffffffu, at >= 0 && at < n);
            if (hit) {
                const int src = __ffs(hit) - 1;
                row0 = __shfl_sync(0xffffffffu, l + at * kTokens, src);
                rows = __shfl_sync(0xffffffffu, (int32_t)min((int64_t)kTokens, h - (l + at * kTokens)), src);
                expert = e0 + src;
            }
            sum += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) s_row0 = row0, s_rows = rows, s_expert = expert, s_head = head, s_tail = before;
    }
    __syncthreads();
    const int64_t row0 = s_row0;
    const int rows = s_rows;
    constexpr bool kGate = ACT == ILW_ACT_SILU_GATE;
    const int32_t width = kGate ? g.N / 2 : g.N;
    if (rows > 0) {
        const int group = warp / p.ksplit, part = warp % p.ksplit;
        const int32_t n0 = (block * (kWarps / p.ksplit) + group) * kRows;
        const int8_t *w = g.w_codes + s_expert * g.w_codes_stride;
        int32_t v = 0;
        int shift = 0;  // index of a lane's sum: lane >> shift
        if (n0 < g.N) {
            if (rows == 1) v = sums<1>(p, w, n0, row0, rows, part, lane), shift = 3;
            else if (rows == 2) v = sums<2>(p, w, n0, row0, rows, part, lane), shift = 2;
            else if (rows <= 4) v = sums<4>(p, w, n0, row0, rows, part, lane), shift = 1;
            else v = sums<8>(p, w, n0, row0, rows, part, lane);
        }
        if (p.ksplit > 1) {
            parts[warp][lane] = v;
            __syncthreads();
            if (part == 0)
                for (int i = 1; i < p.ksplit; ++i) v += parts[warp + i][lane];
        }
        if (part == 0 && n0 < g.N) {
            const int i = lane >> shift, t = i / kRows, n = n0 + i % kRows;
            const bool in = t < rows && n < g.N && (lane & ((1 << shift) - 1)) == 0;
            float z = 0.0f;
            if (in) {
                const int64_t at = (int64_t)s_expert * g.N + n;
                z = (float)v * g.a_scales[row0 + t] * g.w_scales[at];
                if (g.bias) z += g.bias[at];
            }
            if constexpr (ACT == ILW_ACT_GELU) {
                float none = 0.0f;
                gelu2(z, none);
            }
            if constexpr (kGate) z = silu_gate<T>(z, __shfl_down_sync(0xffffffffu, z, 1 << shift));
            if (in && !(kGate && n & 1)) ((T *)g.Y)[(row0 + t) * g.ldy + (kGate ? n >> 1 : n)] = to_out<T>(z);
        }
    }
    // rows of no expert are zero
    if (g.offsets) {
        const int64_t head = s_head, tail = s_tail, total = (head + g.M - tail) * width;
        for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
            const int64_t r = i / width;
            ((T *)g.Y)[(r < head ? r : r - head + tail) * g.ldy + (i - r * width)] = to_out<T>(0.0f);
        }
    }
}

template <int ACT> cudaError_t launch(const FewParams &p, int64_t grid, cudaStream_t s) {
    if (p.g.form == ILW_FP32) return launch_after(i8_few_kernel<ACT, float>, (unsigned)grid, 32 * kWarps, 0, s, p);
    if (p.g.form == ILW_FP16) return launch_after(i8_few_kernel<ACT, __half>, (unsigned)grid, 32 * kWarps, 0, s, p);
    return launch_after(i8_few_kernel<ACT, __nv_bfloat16>, (unsigned)grid, 32 * kWarps, 0, s, p);
}

}  // namespace

cudaError_t launch_i8_few(const I8GemmProblem &g, cudaStream_t s) {
    if (g.M == 0 || g.N == 0) return cudaSuccess;
    FewParams p;
    p.g = g;
    p.units = g.offsets ? std::min<int64_t>(g.M, g.M / kTokens + g.experts) : (g.M + kTokens - 1) / kTokens;
    // as many warps to the same rows of W as have a step of K each, while there are fewer than 32 warps an SM
    const int64_t groups = ((int64_t)g.N + kRows - 1) / kRows;
    p.ksplit = 1;
    while (p.ksplit < kWarps && groups * p.units * p.ksplit < 32 * sm_count() && p.ksplit * 512 < g.K) p.ksplit *= 2;
    const int64_t per = kWarps / p.ksplit;
    p.nblocks = (int32_t)((groups + per - 1) / per);
    const int64_t grid = p.units * p.nblocks;
    if (grid > INT32_MAX) return cudaErrorInvalidValue;
    if (g.act == ILW_ACT_GELU) return launch<ILW_ACT_GELU>(p, grid, s);
    if (g.act == ILW_ACT_SILU_GATE) return launch<ILW_ACT_SILU_GATE>(p, grid, s);
    return launch<ILW_ACT_NONE>(p, grid, s);
}

}  // namespace ilw
