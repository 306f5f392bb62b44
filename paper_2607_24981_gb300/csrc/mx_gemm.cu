// mx_gemm.cu -- products of microscaled 4-bit (MXFP4) matrices on the 5th-generation tensor cores
// (tcgen05.mma kind::mxf4, sm_103a): Y = act(A W^T + bias), for one weight or for one weight per expert
// with ragged groups of rows.
//
//   z[m, n] = sum over blocks b of 2^(sa[m,b] + sw[n,b] - 254) sum_{k in b} a[m,k] w[n,k]  + bias[n]
//
// The tensor core multiplies the 4-bit codes and the block scales exactly and accumulates in fp32 in
// tensor memory; activation and rounding to the output type happen once, in the epilogue.
//
// Layout.  The rows of W take the 128 lanes of a tile and the rows of A (tokens) its columns: a tile is 128
// outputs x up to 224 tokens, with the number of tokens set at run time in steps of 16.  So one kernel
// serves a single token (the 128 rows of W stream past one 16-wide MMA), a ragged group of an expert
// (the columns past its end are neither computed beyond the next 16 nor stored) and a long batch.
// Scales arrive as they are stored, row-major, 16 bytes (512 values of K) a row by TMA; four warps turn them
// into the tensor core's layout (lane i of each quarter, column c: row 32 c + i; four scales of 128 values of K to
// a word) on their way through registers into tensor memory, so rows may start anywhere.
//
// One CTA per SM, 16 warps: TMA producer, MMA issuer, 4 scale warps, 8 epilogue warps (two spare).  Two
// accumulators let a tile's epilogue overlap the next tile's MMAs.  Tiles are dealt out in turn; with experts
// each CTA works out the list of tiles from the offsets itself, so no count has to reach the host.
// With few tiles the K range of each is split over the CTAs of a cluster, whose partial sums meet in
// distributed shared memory and are added in a fixed order.
//
// Every mbarrier wait is bounded; on expiry the kernel latches the device status word, stops issuing
// work, waits for its loads and MMAs in flight and frees its tensor memory.
#include <algorithm>
#include <climits>
#include <cstdint>
#include <cstring>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_ptx.cuh"
#include "ilwdetr.h"
#include "ilw_kernels.h"
#include "mx_kernels.h"

namespace ilw {
void gemm_debug_wait(int32_t *skip, long long *cycles);
namespace {

constexpr int kRowsW = 128;     // rows of W a tile
constexpr int kMaxTok = 224;    // tokens a tile
constexpr int kMaxStages = 16, kMaxScaleStages = 8;
constexpr int kThreads = 512;
constexpr int kScaleWarp0 = 4, kEpiWarp0 = 8, kEpiWarps = 8;
constexpr int kScaleCol = 2 * kMaxTok;  // tensor-memory columns: two accumulators, then two scale buffers of 24
constexpr int kScaleCols = 24;
constexpr int kSmemLimit = 227 * 1024;

struct MxParams {
    CUtensorMap wc, ws, ac, as;  // codes and scales of W [E, N, .] and A [M, .]
    const int32_t *offsets;
    const float *bias;
    void *Y;
    int64_t ldy, M;
    int32_t N, K, E;
    int32_t nkb, nsb;       // K in blocks of 256 (a data stage) and 512 (a scale stage)
    int32_t wtiles;         // tiles of 128 rows of W
    int32_t nt;             // most tokens a tile, a multiple of 16
    int32_t abox;           // rows of A a TMA box
    int32_t stages, sstages, stage_bytes, sstage_bytes;
    int32_t splits;         // CTAs of a cluster that share a tile's K (split form)
    int32_t dbg_skip;
    long long wait_cycles;
    int *status;
};

struct Tile {
    int32_t e, row0, rows, n0;
};

__device__ __forceinline__ bool wait_bar(uint32_t b, uint32_t parity, volatile int *abort, const MxParams &p, int code) {
    if (bar_try(b, parity)) return true;
    const long long t0 = clock64();
    for (uint32_t i = 0;; ++i) {
        if (bar_try(b, parity)) return true;
        if ((i & 63) == 63) {
            if (*abort) return false;
            if (clock64() - t0 > p.wait_cycles) {
                if (p.status) atomicExch(p.status, code);
                *abort = 1;
                return false;
            }
        }
    }
}

// The same for a whole warp, one answer for all lanes (the tcgen05 instructions after it are warp-wide).
__device__ __forceinline__ bool wait_warp(uint32_t b, uint32_t parity, volatile int *abort, const MxParams &p, int code) {
    return __all_sync(0xffffffffu, wait_bar(b, parity, abort, p, code));
}

__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                       uint32_t acc, uint32_t issue) {
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.b32 p, %6, 0;\n setp.ne.b32 q, %7, 0;\n"
        " @q tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc), "r"(issue)
        : "memory");
}
__device__ __forceinline__ void commit_if(uint32_t bar, uint32_t issue) {
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
        " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}\n" ::"r"(bar), "r"(issue)
        : "memory");
}
__device__ __forceinline__ void tst4(uint32_t t, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(t), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
__device__ __forceinline__ void lds128(uint32_t a, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(a));
}

// Instruction descriptor of kind::mxf4: E2M1 operands (format 1), UE8M0 scales, M = 128, N = n, both
// operands K-major; `id` (0 or 2) is the byte of a scale word at which this MMA's two scales begin.
__device__ __forceinline__ uint32_t idesc_mx(uint32_t n, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((128u >> 4) << 24) | (id << 29);
}

template <typename T> __device__ __forceinline__ T to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ __half to_out<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// An expert's rows in equal tiles of at most nt (a multiple of 16 each but the last).
__device__ __forceinline__ int32_t tile_width(int32_t rows, int32_t tiles) { return ((rows + tiles - 1) / tiles + 15) & ~15; }

// Tile t: the weight tile runs fastest, so CTAs that run together share a token tile's rows.
__device__ __forceinline__ Tile find_tile(const MxParams &p, const int32_t *start, const int32_t *lo, const int32_t *hi, int32_t t) {
    const int32_t tt = t / p.wtiles;
    int a = 0, b = p.E;  // the expert e with start[e] <= tt < start[e + 1]
    while (b - a > 1) {
        const int m = (a + b) >> 1;
        if (start[m] <= tt) a = m;
        else b = m;
    }
    const int32_t w = tile_width(hi[a] - lo[a], start[a + 1] - start[a]);
    Tile r;
    r.e = a;
    r.row0 = lo[a] + (tt - start[a]) * w;
    r.rows = min(w, hi[a] - r.row0);
    r.n0 = (t - tt * p.wtiles) * kRowsW;
    return r;
}

// One epilogue warp's 32 columns (tokens c0 .. c0 + 31 of the tile): this lane's row of W is output n.
template <int ACT, typename T>
__device__ __forceinline__ void store_chunk(const MxParams &p, float (&v)[32], const Tile &t, int c0, int n, float bias) {
    const int left = t.rows - c0;
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] += bias;
    if constexpr (ACT == ILW_ACT_SILU_GATE) {
        // even lanes hold gates, odd lanes the rows they gate: each lane of a pair finishes every other token
        const int odd = n & 1;
        T *y = (T *)p.Y + (int64_t)(t.row0 + c0 + odd) * p.ldy + (n >> 1);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, odd ? v[2 * i] : v[2 * i + 1], 1);
            const float gate = odd ? other : v[2 * i], up = odd ? v[2 * i + 1] : other;
            if (2 * i + odd < left && n < p.N) y[(int64_t)(2 * i) * p.ldy] = to_out<T>(gate / (1.0f + expf(-gate)) * up);
        }
    } else {
        T *y = (T *)p.Y + (int64_t)(t.row0 + c0) * p.ldy + n;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float z = v[i];
            if constexpr (ACT == ILW_ACT_GELU) z = 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
            if (i < left && n < p.N) y[(int64_t)i * p.ldy] = to_out<T>(z);
        }
    }
}

template <int ACT, typename T, bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1) mx_gemm_kernel(const __grid_constant__ MxParams p) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kMaxStages + 2 * kMaxScaleStages + 9];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t data0 = (su32(smem_raw) + 1023) & ~1023u;
    const uint32_t scale0 = data0 + p.stages * p.stage_bytes;
    int32_t *start = (int32_t *)(smem_raw + (scale0 - su32(smem_raw)) + p.sstages * p.sstage_bytes);
    int32_t *lo = start + p.E + 1, *hi = lo + p.E;

    const uint32_t b0 = su32(bars);
    auto full = [&](int i) { return b0 + 8 * i; };
    auto empty = [&](int i) { return b0 + 8 * (kMaxStages + i); };
    auto sfull = [&](int i) { return b0 + 8 * (2 * kMaxStages + i); };
    auto sempty = [&](int i) { return b0 + 8 * (2 * kMaxStages + kMaxScaleStages + i); };
    constexpr int kB = 2 * kMaxStages + 2 * kMaxScaleStages;
    auto tfull = [&](int i) { return b0 + 8 * (kB + i); };        // scales in tensor memory
    auto tempty = [&](int i) { return b0 + 8 * (kB + 2 + i); };
    auto afull = [&](int i) { return b0 + 8 * (kB + 4 + i); };    // accumulators
    auto aempty = [&](int i) { return b0 + 8 * (kB + 6 + i); };
    const uint32_t drain = b0 + 8 * (kB + 8);

    if (threadIdx.x == 0) {
        abort_flag = 0;
        for (int i = 0; i < kMaxStages; ++i) bar_init(full(i), 1), bar_init(empty(i), 1);
        for (int i = 0; i < kMaxScaleStages; ++i) bar_init(sfull(i), 1), bar_init(sempty(i), 4);
        for (int i = 0; i < 2; ++i) bar_init(tfull(i), 4), bar_init(tempty(i), 1), bar_init(afull(i), 1), bar_init(aempty(i), kEpiWarps);
        bar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(su32(&tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    grid_wait();
    // the list of tiles: the row range of each expert, and start[e] = token tiles of the experts before e.  The ranges are
    // held in order, apart and inside [0, M], whatever the offsets say.
    if (warp == 2) {
        const int32_t M = (int32_t)p.M;
        int32_t sum = 0, before = 0;  // token tiles, and the end of the last range, of the experts before this round
        for (int e0 = 0; e0 < p.E; e0 += 32) {
            const int e = e0 + lane;
            int32_t l = 0, h = M;
            if (p.offsets && e < p.E) {
                l = max(0, min(p.offsets[e], M));
                h = max(0, min(p.offsets[e + 1], M));
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t y = __shfl_up_sync(0xffffffffu, h, d);
                if (lane >= d) h = max(h, y);
            }
            h = max(h, before);
            const int32_t prev = __shfl_up_sync(0xffffffffu, h, 1);
            l = min(max(l, lane ? prev : before), h);
            before = __shfl_sync(0xffffffffu, h, 31);
            const int32_t n = e < p.E ? (h - l + p.nt - 1) / p.nt : 0;
            int32_t x = n;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            if (e < p.E) {
                lo[e] = l;
                hi[e] = h;
                start[e] = sum + x - n;
            }
            sum += __shfl_sync(0xffffffffu, x, 31);
        }
        if (lane == 0) start[p.E] = sum;
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_base;
    const int32_t tiles = start[p.E] * p.wtiles;
    const int32_t rank = SPLIT ? (int32_t)(blockIdx.x % p.splits) : 0;
    const int32_t first = SPLIT ? (int32_t)(blockIdx.x / p.splits) : (int32_t)blockIdx.x;
    const int32_t step = SPLIT ? (int32_t)(gridDim.x / p.splits) : (int32_t)gridDim.x;
    const int32_t sb_lo = SPLIT ? (int32_t)((int64_t)p.nsb * rank / p.splits) : 0;
    const int32_t sb_hi = SPLIT ? (int32_t)((int64_t)p.nsb * (rank + 1) / p.splits) : p.nsb;
    const int ncol = (p.nt + 31) / 32;  // scale columns of A's rows

    // (split form: a cluster has one tile at most, the host gives it as many clusters as there can be tiles)
    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0, st = 0;  // data and scale stages loaded
            for (int32_t t = first; t < tiles && !abort_flag; t += step) {
                const Tile x = find_tile(p, start, lo, hi, t);
                const int loads = (x.rows + p.abox - 1) / p.abox;
                for (int32_t sb = sb_lo; sb < sb_hi; ++sb) {
                    const uint32_t ss = st % p.sstages;
                    if (!wait_bar(sempty(ss), ((st / p.sstages) & 1) ^ 1, &abort_flag, p, kStatusTimeoutFree)) break;
                    const uint32_t sd = scale0 + ss * p.sstage_bytes;
                    bar_expect_tx(sfull(ss), kRowsW * 16 + p.nt * 16);
                    tma_3d(sd, &p.ws, sb * 16, x.n0, x.e, sfull(ss));
                    tma_2d(sd + kRowsW * 16, &p.as, sb * 16, x.row0, sfull(ss));
                    ++st;
                    for (int32_t kb = 2 * sb; kb < min(2 * sb + 2, p.nkb); ++kb) {
                        const uint32_t s = it % p.stages;
                        if (!wait_bar(empty(s), ((it / p.stages) & 1) ^ 1, &abort_flag, p, kStatusTimeoutFree)) break;
                        const uint32_t d = data0 + s * p.stage_bytes;
                        if ((int32_t)it != p.dbg_skip) {
                            bar_expect_tx(full(s), kRowsW * 128 + loads * p.abox * 128);
                            tma_3d(d, &p.wc, kb * 128, x.n0, x.e, full(s));
                            for (int i = 0; i < loads; ++i)
                                tma_2d(d + kRowsW * 128 + i * p.abox * 128, &p.ac, kb * 128, x.row0 + i * p.abox, full(s));
                        }
                        ++it;
                    }
                    if (abort_flag) break;
                }
            }
            if (abort_flag) {  // the loads in flight end (bounded) before the CTA can exit
                const long long t0 = clock64();
                auto ends = [&](uint32_t b, uint32_t parity) {
                    while (!bar_try(b, parity) && clock64() - t0 < p.wait_cycles) {
                    }
                };
                for (uint32_t i = it > (uint32_t)p.stages ? it - p.stages : 0; i < it; ++i)
                    if ((int32_t)i != p.dbg_skip) ends(full(i % p.stages), (i / p.stages) & 1);
                for (uint32_t i = st > (uint32_t)p.sstages ? st - p.sstages : 0; i < st; ++i) ends(sfull(i % p.sstages), (i / p.sstages) & 1);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t one = elect_one();
        uint32_t it = 0, n = 0;
        bool ok = true;
        for (int32_t t = first; ok && t < tiles; t += step, ++n) {
            const Tile x = find_tile(p, start, lo, hi, t);
            const uint32_t acc = n & 1, d = tmem + acc * kMaxTok;
            const uint32_t id = idesc_mx((x.rows + 15) & ~15, 0);
            ok = wait_warp(aempty(acc), ((n >> 1) & 1) ^ 1, &abort_flag, p, kStatusTimeoutFree);
            const int32_t kb1 = min(2 * sb_hi, p.nkb);
            for (int32_t kb = 2 * sb_lo; ok && kb < kb1; ++kb, ++it) {
                const uint32_t s = it % p.stages, tb = it & 1;
                ok = wait_warp(full(s), (it / p.stages) & 1, &abort_flag, p, kStatusTimeoutTma) &&
                     wait_warp(tfull(tb), (it >> 1) & 1, &abort_flag, p, kStatusTimeoutOperand);
                if (!ok) break;
                fence_after();
                const uint64_t wd = desc_sw128(data0 + s * p.stage_bytes), ad = desc_sw128(data0 + s * p.stage_bytes + kRowsW * 128);
                const uint32_t sc = tmem + kScaleCol + tb * kScaleCols;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = j >> 1, sf = (j & 1) * 2;
                    mma_mx(d, wd + 2 * j, ad + 2 * j, id | (sf << 4) | (sf << 29), sc + 4 * w, sc + 8 + 8 * w,
                           kb > 2 * sb_lo || j > 0, one);
                }
                commit_if(empty(s), one);
                commit_if(tempty(tb), one);
            }
            if (ok) commit_if(afull(acc), one);
        }
        if (!ok) {  // the MMAs in flight end before tensor memory is freed
            commit_if(drain, one);
            const long long t0 = clock64();
            while (!bar_try(drain, 0) && clock64() - t0 < p.wait_cycles) {
            }
        }
        __syncwarp();
    } else if (warp >= kScaleWarp0 && warp < kScaleWarp0 + 4) {
        const uint32_t quarter = (uint32_t)(warp & 3) << 21;  // lane field of this warp's 32 lanes
        uint32_t it = 0, st = 0;
        bool ok = true;
        for (int32_t t = first; ok && t < tiles; t += step) {
            for (int32_t sb = sb_lo; ok && sb < sb_hi; ++sb, ++st) {
                const uint32_t ss = st % p.sstages;
                ok = wait_warp(sfull(ss), (st / p.sstages) & 1, &abort_flag, p, kStatusTimeoutTma);
                if (!ok) break;
                const uint32_t src = scale0 + ss * p.sstage_bytes + lane * 16;
                uint32_t w[4][4], a[8][4];
#pragma unroll
                for (int c = 0; c < 4; ++c) lds128(src + c * 512, w[c]);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    a[c][0] = a[c][1] = a[c][2] = a[c][3] = 0;
                    if (c < ncol) lds128(src + kRowsW * 16 + c * 512, a[c]);
                }
                __syncwarp();
                if (lane == 0) bar_arrive(sempty(ss));
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (2 * sb + h >= p.nkb) break;
                    const uint32_t tb = it & 1;
                    ok = wait_warp(tempty(tb), ((it >> 1) & 1) ^ 1, &abort_flag, p, kStatusTimeoutMma);
                    if (!ok) break;
                    fence_after();
                    __syncwarp();
                    const uint32_t sc = tmem + quarter + kScaleCol + tb * kScaleCols;
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const int k = 2 * h + g;
                        tst4(sc + 4 * g, w[0][k], w[1][k], w[2][k], w[3][k]);
                        tst4(sc + 8 + 8 * g, a[0][k], a[1][k], a[2][k], a[3][k]);
                        if (ncol > 4) tst4(sc + 12 + 8 * g, a[4][k], a[5][k], a[6][k], a[7][k]);
                    }
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(tfull(tb));
                    ++it;
                }
            }
        }
    } else if (warp >= kEpiWarp0) {
        const uint32_t quarter = (uint32_t)(warp & 3) << 21;
        const int half = (warp - kEpiWarp0) >> 2;
        const int row = 32 * (warp & 3) + lane;
        uint32_t n = 0;
        for (int32_t t = first; t < tiles; t += step, ++n) {
            const Tile x = find_tile(p, start, lo, hi, t);
            const uint32_t acc = n & 1;
            const int nn = x.n0 + row;
            const float bias = !SPLIT && p.bias && nn < p.N ? p.bias[(int64_t)x.e * p.N + nn] : 0.0f;
            if (!wait_warp(afull(acc), (n >> 1) & 1, &abort_flag, p, kStatusTimeoutMma)) break;
            __syncwarp();
            fence_after();
            for (int c0 = 32 * half; c0 < x.rows; c0 += 64) {
                uint32_t u[32];
                tld<32>(tmem + quarter + acc * kMaxTok + c0, u);
                twait<32>(u);
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(u[i]);
                if constexpr (SPLIT) {  // this CTA's part of the sums: [token][row of W] over the stages, which are all read
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(data0 + ((c0 + i) * kRowsW + row) * 4), "f"(v[i]) : "memory");
                } else {
                    store_chunk<ACT, T>(p, v, x, c0, nn, bias);
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(aempty(acc));
        }
    }
    if constexpr (SPLIT) {
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (first < tiles && !abort_flag) {
            // each CTA of the cluster finishes some chunks of 32 tokens x 32 rows of W
            const Tile x = find_tile(p, start, lo, hi, first);
            const int chunks = 4 * ((x.rows + 31) / 32);
            for (int c = warp + 16 * rank; c < chunks; c += 16 * p.splits) {
                const int c0 = 32 * (c >> 2), row = 32 * (c & 3) + lane, nn = x.n0 + row;
                const float bias = p.bias && nn < p.N ? p.bias[(int64_t)x.e * p.N + nn] : 0.0f;
                float v[32];
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = 0.0f;
                for (int r = 0; r < p.splits; ++r) {
                    uint32_t at;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(data0 + (c0 * kRowsW + row) * 4), "r"(r));
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        float y;
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(y) : "r"(at + i * kRowsW * 4) : "memory");
                        v[i] += y;
                    }
                }
                store_chunk<ACT, T>(p, v, x, c0, nn, bias);
            }
        }
        asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
    // rows of no expert are zero
    if (p.offsets) {
        const int64_t wide = ACT == ILW_ACT_SILU_GATE ? p.N / 2 : p.N;
        const int64_t head = lo[0], tail = hi[p.E - 1];
        const int64_t total = (head + p.M - tail) * wide;
        for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kThreads) {
            const int64_t r = i / wide;
            ((T *)p.Y)[(r < head ? r : r - head + tail) * p.ldy + (i - r * wide)] = to_out<T>(0.0f);
        }
    }
    fence_before();
    __syncthreads();
    if (warp == 0) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// A tensor map over rows of bytes: [z, rows, cols], boxes of box_rows x box_cols bytes.
bool byte_map(CUtensorMap *m, const void *base, int64_t cols, int64_t rows, int64_t ld, int64_t z, int64_t zstride, int box_cols,
              int box_rows, bool swizzle) {
    EncodeTiledTc fn = encode_tc();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)(z > 0 ? z : 1)};
    cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)zstride};
    cuuint32_t box[3] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, z > 0 ? 3 : 2, const_cast<void *>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int ACT, typename T, bool SPLIT>
cudaError_t launch(const MxParams &p, int grid, size_t smem, cudaStream_t s) {
    static SmemLimit limit;
    cudaError_t e = raise_smem_limit(limit, (const void *)mx_gemm_kernel<ACT, T, SPLIT>, kSmemLimit - 1024);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = kThreads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = SPLIT ? p.splits : 1;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = SPLIT ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, mx_gemm_kernel<ACT, T, SPLIT>, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}
template <int ACT, typename T>
cudaError_t launch_split(const MxParams &p, int grid, size_t smem, cudaStream_t s) {
    return p.splits > 1 ? launch<ACT, T, true>(p, grid, smem, s) : launch<ACT, T, false>(p, grid, smem, s);
}
template <int ACT>
cudaError_t launch_form(const MxParams &p, int32_t form, int grid, size_t smem, cudaStream_t s) {
    if (form == ILW_FP32) return launch_split<ACT, float>(p, grid, smem, s);
    if (form == ILW_FP16) return launch_split<ACT, __half>(p, grid, smem, s);
    return launch_split<ACT, __nv_bfloat16>(p, grid, smem, s);
}

}  // namespace

cudaError_t launch_mx_gemm(const MxGemmProblem &g, cudaStream_t s) {
    if (g.M == 0 || g.N == 0) return cudaSuccess;
    MxParams p;
    memset(&p, 0, sizeof(p));
    p.offsets = g.offsets;
    p.bias = g.bias;
    p.Y = g.Y;
    p.ldy = g.ldy;
    p.M = g.M;
    p.N = g.N;
    p.K = g.K;
    p.E = g.experts;
    p.nkb = (g.K + 255) / 256;
    p.nsb = (g.K + 511) / 512;
    p.wtiles = (g.N + kRowsW - 1) / kRowsW;
    p.status = status_word_ptr();
    gemm_debug_wait(&p.dbg_skip, &p.wait_cycles);
    const int64_t sms = sm_count();

    // Tokens a tile: as wide as the tokens (of an expert, twice the mean) fill, at most 224.
    const int64_t per = g.offsets ? (2 * g.M + g.experts - 1) / g.experts : g.M;
    p.nt = (int32_t)std::min<int64_t>(kMaxTok, (std::min(per, g.M) + 15) / 16 * 16);
    const int64_t token_tiles = g.offsets ? std::min<int64_t>(g.M, g.M / p.nt + g.experts) : (g.M + p.nt - 1) / p.nt;
    const int64_t tiles = token_tiles * p.wtiles;  // at most
    if (tiles > INT32_MAX) return cudaErrorInvalidValue;
    p.abox = p.nt <= 32 || !g.offsets ? p.nt : 32;
    if (p.nt % p.abox) p.nt += 16;  // (whole boxes; 224 is a multiple of 32)
    p.stage_bytes = kRowsW * 128 + p.nt * 128;
    p.sstage_bytes = kRowsW * 16 + (p.nt + 31) / 32 * 512;
    // few tiles: as many CTAs to a tile as the chip has room for, each with whole scale stages of K
    p.splits = 1;
    while (p.splits < 8 && 2 * p.splits * tiles <= sms && 2 * p.splits <= p.nsb) p.splits *= 2;

    p.sstages = 4;
    const int table = (3 * g.experts + 2) * 4, fixed = 1024 + 1024 + table;  // (barriers and alignment)
    p.stages = std::min<int32_t>(kMaxStages, (kSmemLimit - fixed - p.sstages * p.sstage_bytes) / p.stage_bytes);
    p.sstages = std::min<int32_t>(kMaxScaleStages, std::max(4, (p.stages + 1) / 2 + 1));
    p.stages = std::min<int32_t>(kMaxStages, (kSmemLimit - fixed - p.sstages * p.sstage_bytes) / p.stage_bytes);
    const size_t smem = 1024 + (size_t)p.stages * p.stage_bytes + (size_t)p.sstages * p.sstage_bytes + table;

    const int64_t kc = (int64_t)(g.K + 31) / 32 * 16, kb = (g.K + 31) / 32;
    if (!byte_map(&p.wc, g.w_codes, kc, g.N, g.w_ldc, g.experts, g.w_codes_stride, 128, kRowsW, true) ||
        !byte_map(&p.ws, g.w_scales, kb, g.N, g.w_lds, g.experts, g.w_scales_stride, 16, kRowsW, false) ||
        !byte_map(&p.ac, g.a_codes, kc, g.M, g.a_ldc, 0, 0, 128, p.abox, true) ||
        !byte_map(&p.as, g.a_scales, kb, g.M, g.a_lds, 0, 0, 16, p.nt, false))
        return cudaErrorInvalidValue;
    const int grid = (int)(p.splits > 1 ? tiles * p.splits : std::min<int64_t>(tiles, sms));
    if (g.act == ILW_ACT_GELU) return launch_form<ILW_ACT_GELU>(p, g.form, grid, smem, s);
    if (g.act == ILW_ACT_SILU_GATE) return launch_form<ILW_ACT_SILU_GATE>(p, g.form, grid, smem, s);
    return launch_form<ILW_ACT_NONE>(p, g.form, grid, smem, s);
}

}  // namespace ilw
