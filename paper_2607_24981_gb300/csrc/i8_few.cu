// i8_few.cu -- products of int8 rows with float scales for few tokens: y = act(sa sw sum_k a w + bias), for one weight or for one
// weight per expert with ragged rows.
//
// A few tokens use every weight a few times, so what counts is the weights' stream.  A warp takes four rows of W and up to eight tokens
// and walks along K in steps of 512, every lane 16 bytes of each row; sums are whole numbers (dp4a, int32), so any split of K gives the
// same.  The warps of a CTA take rows of W each, or share their K where there are too few rows of W to fill the SMs.  CTAs stay and go from
// one piece of work to the next, so that the experts' rows are looked up once.
#include <algorithm>
#include <climits>
#include <cstdint>

#include "divisor.cuh"
#include "float_act.cuh"
#include "i8_kernels.h"
#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "tile_gemm.cuh"

namespace ilw {
namespace {

// Two CTAs an SM (with three, 80 registers a thread, one token of 16384 x 16384 takes 67 us instead of 44) and two steps in flight a warp (one: 52
// us; four: as two, and one token of 4096 x 4096 3.8 us instead of 3.7).
constexpr int kRows = 4, kTokens = 8, kWarps = 8, kCtas = 2, kSteps = 2;

struct FewParams : I8GemmProblem {
    int32_t ksplit;   // warps that share K (1, 2, 4 or 8)
    // (as list_tiles and find_tile want them: tiles of four rows of W and up to kTokens tokens)
    int32_t E, nt, wtiles;
    uint32_t wdiv_m, wdiv_s;
};

__device__ __forceinline__ int32_t dot16(const int4 &a, const int4 &b, int32_t c) {
    return __dp4a(a.w, b.w, __dp4a(a.z, b.z, __dp4a(a.y, b.y, __dp4a(a.x, b.x, c))));
}

// This warp's part of K of rows n0 .. n0 + 3 of W and `T` tokens from row0 on (`rows` of them exist): the sums of (token t, row r) at
// index 4 t + r in lane index << (5 - log2(4 T)).  Rows and tokens past the last are that one again, and no one's.
template <int T>
__device__ __forceinline__ int32_t sums(const FewParams &g, const int8_t *w, int32_t n0, int64_t row0, int rows, int part, int lane) {
    int32_t acc[kRows * T];
#pragma unroll
    for (int i = 0; i < kRows * T; ++i) acc[i] = 0;
    const int8_t *wr[kRows], *a0 = g.a_codes + row0 * g.a_ldc;
#pragma unroll
    for (int r = 0; r < kRows; ++r) wr[r] = w + (int64_t)min(n0 + r, g.N - 1) * g.w_ldc;
    auto token = [&](int t) { return a0 + min(t, rows - 1) * g.a_ldc; };
    // steps of 512 of K, two at a time: their loads of W first; the tokens, which every warp reads, come from the L1
    const int32_t whole = g.K / 512, stride = g.ksplit * 512;
    int32_t n = (whole - part + g.ksplit - 1) / g.ksplit, k = part * 512 + lane * 16;
    for (; n >= kSteps; n -= kSteps) {
        int4 wv[kSteps][kRows];
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
#pragma unroll
            for (int r = 0; r < kRows; ++r) wv[j][r] = __ldcs((const int4 *)(wr[r] + k + j * stride));
#pragma unroll
        for (int j = 0; j < kSteps; ++j, k += stride)
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const int4 av = __ldg((const int4 *)(token(t) + k));
#pragma unroll
                for (int r = 0; r < kRows; ++r) acc[t * kRows + r] = dot16(wv[j][r], av, acc[t * kRows + r]);
            }
    }
    // the steps that are left, and of the last one what there is of it
    const bool rest = part == whole % g.ksplit && whole * 512 + lane * 16 + 16 <= g.K;
#pragma unroll 1
    for (; n >= 0; --n, k += stride) {
        if (n == 0 && !rest) break;
        if (n == 0) k = whole * 512 + lane * 16;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int4 av = __ldg((const int4 *)(token(t) + k));
#pragma unroll
            for (int r = 0; r < kRows; ++r) acc[t * kRows + r] = dot16(__ldg((const int4 *)(wr[r] + k)), av, acc[t * kRows + r]);
        }
    }
    // the last piece, of fewer than 16: four codes a lane, the last ones byte by byte (nothing past K is read)
    k = (g.K & ~15) + 4 * lane;
    if (lane < 4 && k < g.K && part == (k >> 9) % g.ksplit) {
        const int32_t left = g.K - k;
        auto four = [&](const int8_t *at) {
            if (left >= 4) return *(const int32_t *)at;
            int32_t v = (uint8_t)at[0];
            if (left > 1) v |= (int32_t)(uint8_t)at[1] << 8;
            if (left > 2) v |= (int32_t)(uint8_t)at[2] << 16;
            return v;
        };
        int32_t wv[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) wv[r] = four(wr[r] + k);
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int32_t av = four(token(t) + k);
#pragma unroll
            for (int r = 0; r < kRows; ++r) acc[t * kRows + r] = __dp4a(wv[r], av, acc[t * kRows + r]);
        }
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
__global__ void __launch_bounds__(32 * kWarps, kCtas) i8_few_kernel(const __grid_constant__ FewParams p) {
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ int32_t parts[2][kWarps][32];
    __shared__ int32_t s_experts, s_head, s_tail;
    TileExpert *tab = (TileExpert *)dyn;
    int32_t *tab_id = (int32_t *)(tab + p.E + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    grid_wait();
    if (warp == 0) {
        int32_t sum, count, head, tail;
        list_tiles<1>(p, tab, tab_id, lane, sum, count, head, tail);
        if (lane == 0) s_experts = count, s_head = head, s_tail = tail;
    }
    __syncthreads();
    const int experts = s_experts, teams = kWarps / p.ksplit, team = warp / p.ksplit, part = warp % p.ksplit;
    const int32_t tiles = tab[experts].start * p.wtiles;
    constexpr bool kGate = ACT == ILW_ACT_SILU_GATE;
    const int32_t width = kGate ? p.N / 2 : p.N;
    uint32_t turn = 0;
    for (int64_t t0 = (int64_t)blockIdx.x * teams; t0 < tiles; t0 += (int64_t)gridDim.x * teams, ++turn) {
        const int64_t tile = t0 + team;
        Tile x = {};
        int32_t v = 0;
        int shift = 0;  // index of a lane's sum: lane >> shift
        if (tile < tiles) {
            x = find_tile<TILE_ONE, 4>(p, tab, tab_id, experts, (int32_t)tile, 0);
            const int8_t *w = p.w_codes + x.e * p.w_codes_stride;
            if (x.rows == 1) v = sums<1>(p, w, x.n0, x.row0, x.rows, part, lane), shift = 3;
            else if (x.rows == 2) v = sums<2>(p, w, x.n0, x.row0, x.rows, part, lane), shift = 2;
            else if (x.rows <= 4) v = sums<4>(p, w, x.n0, x.row0, x.rows, part, lane), shift = 1;
            else v = sums<8>(p, w, x.n0, x.row0, x.rows, part, lane);
        }
        if (p.ksplit > 1) {
            parts[turn & 1][warp][lane] = v;
            __syncthreads();
            if (part == 0)
                for (int i = 1; i < p.ksplit; ++i) v += parts[turn & 1][warp + i][lane];
        }
        if (part == 0 && tile < tiles) {
            const int i = lane >> shift, t = i / kRows, n = x.n0 + i % kRows;
            const bool in = t < x.rows && n < p.N && (lane & ((1 << shift) - 1)) == 0;
            float z = 0.0f;
            if (in) {
                const int64_t at = (int64_t)x.e * p.N + n;
                z = scaled_sum((float)v, p.a_scales[x.row0 + t], p.w_scales[at], p.bias ? p.bias[at] : 0.0f);
            }
            if constexpr (ACT == ILW_ACT_GELU) {
                float none = 0.0f;
                gelu2(z, none);
            }
            if constexpr (kGate) z = silu_gate<T>(z, __shfl_down_sync(0xffffffffu, z, 1 << shift));
            if (in && !(kGate && n & 1)) ((T *)p.Y)[(int64_t)(x.row0 + t) * p.ldy + (kGate ? n >> 1 : n)] = to_out<T>(z);
        }
    }
    // rows of no expert are zero
    if (p.offsets) {
        const int64_t head = s_head, tail = s_tail, total = (head + p.M - tail) * width;
        for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
            const int64_t r = i / width;
            ((T *)p.Y)[(r < head ? r : r - head + tail) * p.ldy + (i - r * width)] = to_out<T>(0.0f);
        }
    }
}

template <int ACT, typename T> cudaError_t launch_form(const FewParams &p, int64_t grid, cudaStream_t s) {
    return launch_after(i8_few_kernel<ACT, T>, (unsigned)grid, 32 * kWarps, (p.E + 1) * sizeof(TileExpert) + p.E * 4, s, p);
}
template <int ACT> cudaError_t launch(const FewParams &p, int64_t grid, cudaStream_t s) {
    if (p.form == ILW_FP32) return launch_form<ACT, float>(p, grid, s);
    if (p.form == ILW_FP16) return launch_form<ACT, __half>(p, grid, s);
    return launch_form<ACT, __nv_bfloat16>(p, grid, s);
}

}  // namespace

cudaError_t launch_i8_few(const I8GemmProblem &g, cudaStream_t s) {
    if (g.M == 0 || g.N == 0) return cudaSuccess;
    FewParams p;
    static_cast<I8GemmProblem &>(p) = g;
    p.E = g.experts;
    p.nt = kTokens;
    p.wtiles = (g.N + kRows - 1) / kRows;
    const Divisor by = divisor(p.wtiles);
    p.wdiv_m = by.m, p.wdiv_s = by.s;
    const int64_t units = g.offsets ? std::min<int64_t>(g.M, g.M / kTokens + g.experts) : (g.M + kTokens - 1) / kTokens;
    const int64_t tiles = units * p.wtiles, room = (int64_t)kCtas * sm_count();
    if (tiles > INT32_MAX) return cudaErrorInvalidValue;
    // as many warps to the same rows of W as have a step of K each, while all find room at once
    p.ksplit = 1;
    while (p.ksplit < kWarps && 2 * p.ksplit * tiles <= kWarps * room && p.ksplit * 512 < g.K) p.ksplit *= 2;
    const int64_t grid = std::min(room, (tiles * p.ksplit + kWarps - 1) / kWarps);
    if (g.act == ILW_ACT_GELU) return launch<ILW_ACT_GELU>(p, grid, s);
    if (g.act == ILW_ACT_SILU_GATE) return launch<ILW_ACT_SILU_GATE>(p, grid, s);
    return launch<ILW_ACT_NONE>(p, grid, s);
}

}  // namespace ilw
