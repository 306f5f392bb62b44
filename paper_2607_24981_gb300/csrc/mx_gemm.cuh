#pragma once
// mx_gemm.cuh -- products of microscaled 4-bit (MXFP4) matrices on the 5th-generation tensor cores
// (tcgen05.mma kind::mxf4, sm_103a): Y = act(A W^T + bias), for one weight or for one weight per expert
// with ragged groups of rows.
//
//   z[m, n] = sum over blocks b of 2^(sa[m,b] + sw[n,b] - 254) sum_{k in b} a[m,k] w[n,k]  + bias[n]
//
// The tensor core multiplies the 4-bit codes and the block scales exactly and accumulates in fp32 in
// tensor memory; activation and rounding to the output type happen once, in the epilogue.
//
// Tiles.  The rows of W take the 128 lanes of a tile and the rows of A (tokens) its columns: a tile is 128
// outputs x up to 224 tokens, with the number of tokens set at run time in steps of 16.  So one kernel
// serves a single token (the 128 rows of W stream past one 16-wide MMA), a ragged group of an expert
// (the columns past its end are neither computed beyond the next 16 nor stored) and a long batch.
//
// Three forms.  ONE: a CTA a tile.  SPLIT, for few tiles: the K range of a tile is shared by the CTAs of a
// cluster, whose partial sums meet in distributed shared memory and are added in a fixed order.  PAIR, for
// many: two SMs share a tile of 256 outputs (cta_group::2), each with its own 128 rows of W and half of
// the tokens.  One CTA's shared memory takes 45 KB of operands for each 256 of K of its tile and gives them to the
// tensor core once, at 128 bytes a clock 700 clocks for MMAs of 450; in a pair it is 30 KB.  8192 cubed: 168 us in pairs (6.5
// PFLOP/s; some 50 bytes a clock reach each SM, of nominally 64; back to back for seconds, at the power limit, 182 to 187 us), 194 us
// without.  Tensor pipe active 63 % of the time (4096 x 4096 x 8192).
//
// Scales are stored row-major, 16 bytes of a row for 512 values of K.  Four pairs of warps take turns (a turn is a chain of
// latencies of some 2000 clocks, the MMAs of 512 values are done in 900) to bring them in by asynchronous copies
// of 16 bytes (TMA boxes 16 bytes wide held up the loads of the codes behind them), a lane its own rows, and to
// write them, still in shared memory, in the order in which tcgen05.cp brings them to tensor memory (lane i,
// column c: row 32 c + i; the four scales of 128 values of K to a word), so rows may start anywhere; the copies
// and the MMAs that read them follow one another in the tensor pipe without a wait.
//
// One CTA per SM, 28 warps: the loads of W and of A, the MMAs, 8 scale warps, 16 epilogue warps (four on each scheduler:
// with two, the activation's chains of latency set the time of a short K).  A wait on a barrier takes a warp some
// 100 clocks even when there is nothing to wait for, and 256 of K are 450 clocks of MMAs, so each of these roles waits
// once in that time: everything that a block of K needs arrives at one barrier.  Two accumulators let a tile's
// epilogue overlap the next tile's MMAs.  Tiles are dealt out in turn; with experts each CTA works out the list
// of experts that have rows from the offsets itself, so no count has to reach the host, and the last warp finds each tile's
// rows ahead of the others (a role that did so itself lost some 2000 clocks a tile: code that runs once a tile is never
// in the instruction caches that so many roles share).
//
// Every mbarrier wait is bounded; on expiry the kernel latches the device status word, stops issuing
// work, waits for its loads and MMAs in flight and frees its tensor memory.
#include <climits>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_ptx.cuh"
#include "ilwdetr.h"
#include "ilw_kernels.h"
#include "mx_kernels.h"

namespace ilw {

constexpr int kMxRowsW = 128;   // rows of W a CTA
constexpr int kMxMaxTok = 224;  // tokens a tile; a multiple of 32, as tiles of pairs are
constexpr int kMxMaxStages = 16, kMxMinStages = 4;
constexpr int kMxScaleWarp0 = 3, kMxScaleSets = 4;  // pairs of scale warps
constexpr int kMxEpiWarp0 = kMxScaleWarp0 + 2 * kMxScaleSets, kMxEpiWarps = 16, kMxTileWarp = kMxEpiWarp0 + kMxEpiWarps;
constexpr int kMxThreads = 32 * (kMxTileWarp + 1);
constexpr int kMxTiles = 16;    // tiles found ahead
constexpr int kMxAtom = 512;    // bytes of the scales of 128 rows and 128 values of K
constexpr int kMxPatch = 512;   // bytes of shared memory in which an epilogue warp turns 2-byte results
constexpr int kMxSmemLimit = 226 * 1024;  // dynamic; the barriers are static

enum MxMode { MX_ONE = 0, MX_SPLIT = 1, MX_PAIR = 2 };

struct MxExpert {
    int32_t start, row, end, width;  // first token tile, its rows [row, end), rows a tile
};

struct MxParams {
    CUtensorMap wc, ac[4];  // codes of W [E, N, .]; of A [M, .] in boxes of 16, 32, 64 and 128 rows
    const uint8_t *w_scales, *a_scales;
    int64_t w_lds, w_scales_stride, a_lds;
    int32_t nb;             // scale bytes of a row
    const int32_t *offsets;
    const float *bias;
    void *Y;
    int64_t ldy, M;
    int32_t N, E;
    int32_t nkb, nsb;       // K in blocks of 256 (a data stage) and 512 (a scale stage)
    int32_t wtiles;         // tiles of rows of W (128, or 256 a pair)
    uint32_t wdiv_m, wdiv_s;  // division by wtiles
    int32_t nt;             // most tokens a tile, a multiple of 16 (a pair's: of 32)
    int32_t stages;         // stages of codes
    int32_t stage_bytes, raw_bytes, scale_bytes;
    int32_t wide;           // 2-byte rows of Y take 16-byte stores
    int32_t splits;         // CTAs of a cluster that share a tile's K (SPLIT)
    int32_t mode;
    int32_t dbg_skip;
    long long wait_cycles;
    int *status;
};

template <typename T>
cudaError_t launch_mx(const MxParams &p, int32_t act, int grid, size_t smem, cudaStream_t s);

namespace {

struct Tile {
    int32_t e, row0, rows, n0;
};

// Bounded wait: false (after latching `code` and raising the abort flag) when it ran out, or when another role aborted.
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
// The same for a lane that issues loads or MMAs on its own, with the long way out of line: its loop then keeps the operands in
// uniform registers and a wait with nothing to wait for costs next to nothing (a block of K: 225 clocks for 6 copies and 4
// MMAs of 16 tokens, what they take; with a vote of the warp 395).
__device__ __noinline__ bool wait_long(uint32_t b, uint32_t parity, volatile int *abort, const MxParams *p, int code) {
    return wait_bar(b, parity, abort, *p, code);
}
__device__ __forceinline__ bool wait_lane(uint32_t b, uint32_t parity, volatile int *abort, const MxParams &p, int code) {
    return bar_try(b, parity) || wait_long(b, parity, abort, &p, code);
}

// This barrier's address in CTA `rank` of the cluster, and an arrival there.  What the arrivals of a pair order is read by the
// tensor core alone, through the async proxy, to which its writers hand it themselves (TMA, or fence.proxy.async
// after the stores); a release at cluster scope on top of that held each arrival up by some 1000 clocks.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *m) {
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)m) : "memory");
}

// A value that is the same in every lane, in a uniform register: the operands of TMA loads and MMAs are uniform
// registers, and each one that has to be moved there at its instruction costs some 50 clocks (with values that the
// compiler could not know to be uniform a TMA load took 300 clocks, which was the rate of every product).
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
// Of a pair (PAIR) only the first CTA issues, for both.  All by one lane.
template <bool PAIR>
__device__ __forceinline__ void mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t acc) {
    if constexpr (PAIR)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
            " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(acc)
            : "memory");
}
// An arrival at `bar` (of a pair: in both CTAs, unless `local`) when the MMAs and copies issued so far have ended.
template <bool PAIR>
__device__ __forceinline__ void commit_mma(uint32_t bar, bool local = false) {
    if constexpr (PAIR) {
        if (!local)
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                         "h"((uint16_t)3)
                         : "memory");
        else
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    } else {
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    }
}
// Descriptor of scales in order: rows of 16 bytes, eight of them (128 bytes) a core matrix, no swizzle
__device__ __forceinline__ uint64_t scale_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}
// Shared memory to tensor memory (of a pair: in both CTAs, each its own): 32 rows of 16 bytes to 4 columns of 32 lanes, the
// same for each quarter of the lanes.
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t t, uint64_t d) {
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(t), "l"(d) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(t), "l"(d) : "memory");
}
__device__ __forceinline__ void lds128(uint32_t a, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(a)
                 : "memory");
}

// Instruction descriptor of kind::mxf4: E2M1 operands (format 1), UE8M0 scales, M = m, N = n, both
// operands K-major; `id` (0 or 2) is the byte of a scale word at which this MMA's two scales begin.
__device__ __forceinline__ uint32_t idesc_mx(uint32_t m, uint32_t n, uint32_t id) {
    return (id << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (1u << 23) | ((m >> 4) << 24) | (id << 29);
}

template <typename T> __device__ __forceinline__ T to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ __half to_out<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// (By a whole warp.) Tile t: the tile of W's rows runs fastest, so CTAs that run together share a token tile's rows.  tab: the
// experts that have rows, n of them (n <= 1024: two probes of 32), and an end.
template <int MODE>
__device__ __forceinline__ Tile find_tile(const MxParams &p, const MxExpert *tab, const int32_t *id, int n, int32_t t, uint32_t rank) {
    const int lane = threadIdx.x & 31;
    const int32_t tt = (int32_t)((__umulhi((uint32_t)t, p.wdiv_m) + (uint32_t)t) >> p.wdiv_s);  // t / wtiles
    int a = 0;  // the expert with start <= tt < the next one's
    if (n > 32) a = 32 * (__popc(__ballot_sync(0xffffffffu, 32 * lane < n && tab[min(32 * lane, n)].start <= tt)) - 1);
    a += __popc(__ballot_sync(0xffffffffu, a + lane < n && tab[min(a + lane, n)].start <= tt)) - 1;
    const int4 x = *(const int4 *)(tab + a);
    Tile r;
    r.e = id[a];
    r.row0 = x.y + (tt - x.x) * x.w;
    r.rows = min(x.w, x.z - r.row0);
    r.n0 = (t - tt * p.wtiles) * (MODE == MX_PAIR ? 2 * kMxRowsW : kMxRowsW) + (MODE == MX_PAIR ? rank * kMxRowsW : 0);
    return r;
}

// Two floats at a time.
__device__ __forceinline__ uint64_t pack2(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpack2(uint64_t v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t both(float v) { return pack2(v, v); }
__device__ __forceinline__ float rcp_fast(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// z (1 + erf(z / sqrt 2)) / 2 of two values.  With c = |z| / 2 it is z/2 + |z/2| - c erfc(sqrt 2 c), and log2 erfc(sqrt 2 c) is close to a
// polynomial: this one, of degree 10 without a constant and in -c, was fitted to leave c erfc(sqrt 2 c) an error of at most 1.6e-10 (minimax over
// c <= 2.9; past that it falls on, and so does the product).  One operation of the special-function unit a value.  Error in fp32:
// that of its roundings, smaller than with erff (12800 x 1536 x 384 in fp32: 20.4 us, with erff 28.8).
__device__ __forceinline__ void gelu2(float &a, float &b) {
    const float ha = 0.5f * a, hb = 0.5f * b;
    const uint64_t m = pack2(fmaxf(-fabsf(ha), -32.0f), fmaxf(-fabsf(hb), -32.0f));
    uint64_t q = fma2(m, both(-5.52892634e-05f), both(-6.89682201e-04f));
    q = fma2(q, m, both(-3.80723737e-03f));
    q = fma2(q, m, both(-1.19131086e-02f));
    q = fma2(q, m, both(-2.04908401e-02f));
    q = fma2(q, m, both(-1.81822665e-03f));
    q = fma2(q, m, both(1.10451736e-01f));
    q = fma2(q, m, both(4.19400901e-01f));
    q = fma2(q, m, both(-1.83689129e+00f));
    q = fma2(q, m, both(2.30220842e+00f));
    const float2 e = unpack2(mul2(q, m));
    const float2 r = unpack2(fma2(m, pack2(exp2_fast(e.x), exp2_fast(e.y)), pack2(ha + fabsf(ha), hb + fabsf(hb))));
    a = r.x;
    b = r.y;
}
// gate / (1 + exp(-gate)) up for results of type T, by the reciprocal of (1 + exp(-gate)) / 4: that of 1 + exp(-gate) would be flushed to
// zero before the exponential overflows.  exp(-gate) = 2^t (1 + d), where t = -gate log2 e is rounded and d is what that leaves, for
// gates of -80 a hundred roundings of fp32.  Results of two bytes hide it; for those of four the reciprocal takes the factor
// 1 - d 2^t / (1 + 2^t), with t and d of gates past 64 and -100 from there, which gives 1 and 0 as theirs would (t may be
// infinite, and d no number).  16384 rows of 32 experts, 8192 x 2048, fp32: 134 us, without the factor 130.
template <typename T>
__device__ __forceinline__ float silu_gate(float gate, float up) {
    const float q = 0.25f * gate;
    if constexpr (sizeof(T) == 2) return q * rcp_fast(exp2_fast(fmaf(gate, -1.44269504f, -2.0f)) + 0.25f) * up;
    const float x = fmaxf(fminf(gate, 64.0f), -100.0f), t = x * -1.44269504f;
    const float d = fmaf(t, -1.90465421e-09f, fmaf(t, 0.693147182f, x));  // -d, with ln 2 in two parts
    const float r = rcp_fast(fmaf(exp2_fast(t), 0.25f, 0.25f));
    return q * fmaf(r * d, fmaf(r, -0.25f, 1.0f), r) * up;
}

// One warp's 32 rows of W (this lane: row n) x 16 tokens (c0 .. c0 + 15 of the tile).  A lane holds one output of 16
// tokens, so its own stores are 2 bytes wide; where there is an activation and rows of Y allow it (`wide`), 2-byte results
// pass through the warp's patch of shared memory [token][output] and leave in 16-byte pieces (12800 x 1536 x 384 with GELU:
// 20.2 us, 20.9 without; 32 rows of 64 experts, gated, 21.3 and 21.7; 16384 rows of 32, gated, either way 125; without
// activation 8192 cubed takes 181 us so and 169 as it is, 12800 x 1536 x 384 15.8 and 14.9).
template <int ACT, typename T>
__device__ __forceinline__ void store_chunk(const MxParams &p, float (&v)[16], const Tile &t, int c0, int n, float bias, uint32_t patch,
                                            int lane) {
    const int left = t.rows - c0;
    constexpr bool kGate = ACT == ILW_ACT_SILU_GATE;
    constexpr int kCols = kGate ? 16 : 32, kVals = kGate ? 8 : 16;  // outputs of the warp's rows of W, results of a lane
    if (p.bias) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += bias;
    }
    if constexpr (kGate) {
        // even lanes hold gates, odd lanes the rows they gate: each lane of a pair finishes every other token
        const bool odd = lane & 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, odd ? v[2 * i] : v[2 * i + 1], 1);
            v[i] = silu_gate<T>(odd ? other : v[2 * i], odd ? v[2 * i + 1] : other);
        }
    } else if constexpr (ACT == ILW_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) gelu2(v[2 * i], v[2 * i + 1]);
    }
    const int out0 = (kGate ? n >> 1 : n) - (kGate ? lane >> 1 : lane);  // first output of the warp
    const int width = kGate ? p.N / 2 : p.N;
    if constexpr (sizeof(T) == 2 && ACT != ILW_ACT_NONE) {
        if (p.wide) {
            const uint32_t at = patch + (kGate ? (lane & 1) * 2 * kCols + (lane & ~1) : 2 * lane);
            constexpr int kPieces = kCols / 8, kTokens = 32 / kPieces;  // pieces of a token, tokens the patch holds
            const int piece = lane % kPieces, token = lane / kPieces;
            T *y = (T *)p.Y + (int64_t)(t.row0 + c0 + token) * p.ldy + out0 + 8 * piece;
            const bool in = out0 + 8 * piece < width;
#pragma unroll
            for (int h = 0; h < 16 / kTokens; ++h) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const T x = to_out<T>(v[8 * h + i]);
                    asm volatile("st.shared.b16 [%0], %1;" ::"r"(at + i * (kGate ? 4 * kCols : 2 * kCols)), "h"(*(const uint16_t *)&x) : "memory");
                }
                __syncwarp();
                uint32_t q[4];
                lds128(patch + lane * 16, q);
                if (in && token + h * kTokens < left) *(uint4 *)(y + (int64_t)h * kTokens * p.ldy) = make_uint4(q[0], q[1], q[2], q[3]);
                __syncwarp();
            }
            return;
        }
    }
    const int col = out0 + (kGate ? lane >> 1 : lane), first = kGate ? lane & 1 : 0;
    T *y = (T *)p.Y + (int64_t)(t.row0 + c0 + first) * p.ldy + col;
    const int64_t step = kGate ? 2 * p.ldy : p.ldy;
#pragma unroll
    for (int i = 0; i < kVals; ++i, y += step)
        if ((kGate ? 2 * i + first : i) < left && col < width) *y = to_out<T>(v[i]);
}

template <int ACT, typename T, int MODE>
__global__ void __launch_bounds__(kMxThreads, 1) mx_gemm_kernel(const __grid_constant__ MxParams p) {
    constexpr bool SPLIT = MODE == MX_SPLIT, PAIR = MODE == MX_PAIR;
    // tensor-memory columns: two accumulators, then two buffers of the scales of 256 values of K (2 x 4 columns of
    // W's rows, 2 x 8 of A's)
    constexpr int kScaleCol = 2 * kMxMaxTok, kScaleCols = 24;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[3 * kMxMaxStages + kMxScaleSets + 2 * kMxTiles + 5];
    __shared__ int4 tile_ring[kMxTiles];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int abort_flag;
    __shared__ int32_t s_experts, s_head, s_tail;  // experts with rows; rows before the first and from the end of the last
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t data0 = (su32(smem_raw) + 1023) & ~1023u;
    const uint32_t raw0 = data0 + p.stages * p.stage_bytes, scale0 = raw0 + kMxScaleSets * p.raw_bytes;
    const uint32_t patch0 = scale0 + 2 * p.scale_bytes;
    MxExpert *tab = (MxExpert *)(smem_raw + (patch0 - su32(smem_raw)) + (p.wide ? kMxEpiWarps * kMxPatch : 0));
    int32_t *tab_id = (int32_t *)(tab + p.E + 1);

    uint32_t next_bar = su32(bars);
    auto take = [&](int n) {
        const uint32_t at = next_bar;
        next_bar += 8 * n;
        return at;
    };
    // full: a block of K is there, codes and scales (a pair's, at the first CTA: in both); its own: this CTA's codes are, for
    // the second CTA of a pair to pass on
    const uint32_t full = take(kMxMaxStages), empty = take(kMxMaxStages), own = take(kMxMaxStages);
    const uint32_t sfree = take(kMxScaleSets);                          // a place for the scales of a pair's next turn
    const uint32_t tfull = take(kMxTiles), tfree = take(kMxTiles);      // tiles found, and read by every warp
    const uint32_t afull = take(2), aempty = take(2), drain = take(1);  // accumulators

    const uint32_t rank = SPLIT ? blockIdx.x % p.splits : PAIR ? blockIdx.x & 1 : 0;
    const bool leader = !PAIR || rank == 0;
    const int32_t group = SPLIT ? p.splits : PAIR ? 2 : 1, first = (int32_t)blockIdx.x / group;
    if (warp == 0) {
        if (lane == 0) abort_flag = 0;
        if (lane < kMxMaxStages) {
            bar_init(full + 8 * lane, PAIR ? 2 + 1 + 4 : 2 + 2);  // loads, the second CTA's word, scale warps
            bar_init(empty + 8 * lane, 1);
            bar_init(own + 8 * lane, 2);
            bar_init(tfull + 8 * lane, 1);
            bar_init(tfree + 8 * lane, kMxTileWarp);
        } else if (lane < kMxMaxStages + 2) {
            bar_init(afull + 8 * (lane - kMxMaxStages), 1);
            bar_init(aempty + 8 * (lane - kMxMaxStages), PAIR ? 2 * kMxEpiWarps : kMxEpiWarps);
        } else if (lane == kMxMaxStages + 2) {
            bar_init(drain, 1);
        } else if (lane < kMxMaxStages + 3 + kMxScaleSets) {
            bar_init(sfree + 8 * (lane - kMxMaxStages - 3), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32) {
        prefetch_map(&p.wc);
        prefetch_map(&p.ac[0]);
    }
    if (warp == 3) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(su32(&tmem_base)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(su32(&tmem_base)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    grid_wait();
    // the list of tiles: the experts that have rows, in order.  Their ranges are held in order, apart and inside [0, M],
    // whatever the offsets say.
    if (warp == 2) {
        const int32_t M = (int32_t)p.M;
        int32_t sum = 0, count = 0, before = 0, head = M;  // of the experts before this round: tiles, those with rows, end of the last range
        for (int e0 = 0; e0 < p.E; e0 += 32) {
            const int e = e0 + lane;
            int32_t l = 0, h = e < p.E ? M : 0;
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
            if (e0 == 0) head = __shfl_sync(0xffffffffu, l, 0);
            before = __shfl_sync(0xffffffffu, h, 31);
            const int32_t rows = e < p.E ? h - l : 0, tiles = (rows + p.nt - 1) / p.nt;
            int32_t x = tiles;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
                if (lane >= d) x += y;
            }
            const uint32_t with = __ballot_sync(0xffffffffu, rows > 0);
            if (rows > 0) {  // equal tiles of at most nt, multiples of 16 (a pair's: of 32)
                constexpr int kStep = PAIR ? 32 : 16;
                const int i = count + __popc(with & ((1u << lane) - 1));
                *(int4 *)(tab + i) = make_int4(sum + x - tiles, l, h, ((rows + tiles - 1) / tiles + kStep - 1) & ~(kStep - 1));
                tab_id[i] = e;
            }
            sum += __shfl_sync(0xffffffffu, x, 31);
            count += __popc(with);
        }
        if (lane == 0) {
            tab[count].start = sum;
            s_experts = count;
            s_head = head;
            s_tail = before;
        }
        __syncwarp();
        if (first < sum * p.wtiles) {  // the first tile at once; the others follow from the last warp
            const Tile y = find_tile<MODE>(p, tab, tab_id, count, first, rank);
            if (lane == 0) tile_ring[0] = make_int4(y.e, y.row0, y.rows, y.n0);
        }
    }
    fence_before();
    if constexpr (PAIR) cluster_sync();
    else __syncthreads();
    fence_after();
    const uint32_t tmem = uniform(tmem_base);
    const int experts = s_experts;
    const int32_t tiles = tab[experts].start * p.wtiles;
    const int32_t step = (int32_t)gridDim.x / group;
    const int32_t sb_lo = SPLIT ? (int32_t)((int64_t)p.nsb * rank / p.splits) : 0;
    const int32_t sb_hi = SPLIT ? (int32_t)((int64_t)p.nsb * (rank + 1) / p.splits) : p.nsb;
    const int32_t kb_hi = min(2 * sb_hi, p.nkb);
    const int atoms = 1 + (p.nt + 127) / 128;  // of W's rows, and of A's
    // the next tile of this CTA, as the last warp has found it (by a whole warp; false when a wait ran out)
    uint32_t tiles_read = 0;
    auto next_tile = [&](Tile &x) {
        if constexpr (SPLIT) {  // (the only one)
            const int4 v = tile_ring[0];
            x = Tile{v.x, v.y, v.z, v.w};
            return true;
        }
        const uint32_t i = tiles_read % kMxTiles;
        if (tiles_read > 0 && !wait_warp(tfull + 8 * i, (tiles_read / kMxTiles) & 1, &abort_flag, p, kStatusTimeoutOperand)) return false;
        const int4 v = tile_ring[i];
        x = Tile{v.x, v.y, v.z, v.w};
        __syncwarp();
        if (lane == 0) bar_arrive(tfree + 8 * i);
        ++tiles_read;
        return true;
    };
    Tile x = {};  // (an epilogue warp's)
    auto mma_tokens = [&](const Tile &x) { return PAIR ? (x.rows + 31) & ~31 : (x.rows + 15) & ~15; };

    // (SPLIT: a cluster has one tile at most, the host gives it as many clusters as there can be tiles)
    if (warp == 0 || warp == 2) {
        // loads of the codes: warp 0 of W, warp 2 of A
        const uint32_t one = elect_one();
        const uint32_t arrives = leader ? full : own;
        uint32_t it = 0, s = 0, sp = 1;  // stages loaded, the place in the ring, the parity of a free one
        bool ok = true;
        for (int32_t t = first; t < tiles; t += step) {
            Tile x;
            ok = ok && next_tile(x);
            if (!ok) break;
            x.e = uniform(x.e), x.row0 = uniform(x.row0), x.rows = uniform(x.rows), x.n0 = uniform(x.n0);
            // a pair's CTA loads its half of the tokens
            const int part = PAIR ? mma_tokens(x) / 2 : x.rows, row = x.row0 + (PAIR ? (int)rank * part : 0);
            const int units = (part + 15) >> 4;
            const uint32_t bytes = warp == 0 ? kMxRowsW * 128 : units * 2048;
            if (one) {
                for (int32_t kb = 2 * sb_lo; kb < kb_hi; ++kb) {
                    if (!wait_lane(empty + 8 * s, sp, &abort_flag, p, kStatusTimeoutFree)) {
                        ok = false;
                        break;
                    }
                    const uint32_t d = data0 + s * p.stage_bytes + (warp == 0 ? 0 : kMxRowsW * 128), db = arrives + 8 * s;
                    if ((int32_t)it != p.dbg_skip) {
                        bar_expect_tx(db, bytes);
                        if (warp == 0) {
                            tma_3d(d, &p.wc, kb * 128, x.n0, x.e, db);
                        } else {
                            int done = 0;  // (units of 16 rows)
#pragma unroll
                            for (int i = 3; i >= 0; --i)
                                if (units & (1 << i)) {
                                    tma_2d(d + done * 2048, &p.ac[i], kb * 128, row + done * 16, db);
                                    done += 1 << i;
                                }
                        }
                    }
                    ++it;
                    if (++s == (uint32_t)p.stages) s = 0, sp ^= 1;
                }
            }
            ok = __all_sync(0xffffffffu, ok);
        }
        if (one && abort_flag) {  // the loads in flight end (bounded) before the CTA can exit
            // (the barrier may miss other arrivals, so the limit is short: a load takes microseconds)
            const long long t0 = clock64();
            for (uint32_t i = it > (uint32_t)p.stages ? it - p.stages : 0; i < it; ++i)
                while (!bar_try(arrives + 8 * (i % p.stages), (i / p.stages) & 1) && clock64() - t0 < 2000000) {
                }
        }
        __syncwarp();
    } else if (warp == 1 && leader) {
        const uint32_t one = elect_one();
        uint32_t n = 0, s = 0, sp = 0, st = 0, at = 0;  // at: the stage's offset in units of 16 bytes, as descriptors hold it
        const uint64_t desc0 = desc_sw128(data0), scales0 = scale_desc(scale0);
        uint64_t scales = scales0;  // the stage of scales: one of two
        const uint32_t scol = tmem + kScaleCol, half = 2 * kMxAtom * atoms / 16;
        bool ok = true;
        for (int32_t t = first; ok && t < tiles; t += step, ++n) {
            Tile x;
            ok = next_tile(x);
            if (!ok) break;
            const uint32_t acc = n & 1, d = tmem + acc * kMxMaxTok;
            const uint32_t id = idesc_mx(PAIR ? 256 : 128, uniform(mma_tokens(x)), 0);
            ok = wait_warp(aempty + 8 * acc, ((n >> 1) & 1) ^ 1, &abort_flag, p, kStatusTimeoutFree);
            if (!ok) break;
            fence_after();
            // one block of 256 of K: its scales to the columns from sc on, then 4 MMAs of 64
            auto block = [&](uint32_t sc, uint64_t src, bool add) {
                if (!wait_lane(full + 8 * s, sp, &abort_flag, p, kStatusTimeoutTma)) return false;
                fence_after();
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    copy_scales<PAIR>(sc + 4 * w, src);
                    copy_scales<PAIR>(sc + 8 + 8 * w, src + kMxAtom / 16);
                    if (atoms > 2) copy_scales<PAIR>(sc + 12 + 8 * w, src + 2 * kMxAtom / 16);
                    src += kMxAtom * atoms / 16;
                }
                const uint64_t wd = desc0 + at, ad = wd + kMxRowsW * 128 / 16;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t w = j >> 1, sf = (j & 1) * 2;
                    mma_mx<PAIR>(d, wd + 2 * j, ad + 2 * j, id | (sf << 4) | (sf << 29), sc + 4 * w, sc + 8 + 8 * w, add || j > 0);
                }
                commit_mma<PAIR>(empty + 8 * s);
                at += p.stage_bytes / 16;
                if (++s == (uint32_t)p.stages) s = 0, at = 0, sp ^= 1;
                return true;
            };
            if (one) {
                for (int32_t kb = 2 * sb_lo; kb < kb_hi; kb += 2) {  // a stage of scales: two blocks, the last one may be alone
                    ok = block(scol, scales, kb > 2 * sb_lo);
                    if (!ok) break;
                    if (kb + 1 < kb_hi) {
                        ok = block(scol + kScaleCols, scales + half, true);
                        if (!ok) break;
                    }
                    scales = scales == scales0 ? scales0 + p.scale_bytes / 16 : scales0;
                    commit_mma<PAIR>(sfree + 8 * ((st++ + 2) % kMxScaleSets));  // (the turn after the next takes the place of these scales)
                }
                if (ok) commit_mma<PAIR>(afull + 8 * acc);
            }
            ok = __all_sync(0xffffffffu, ok);
        }
        if (!ok && one) {  // the MMAs in flight end before tensor memory is freed
            commit_mma<PAIR>(drain, true);
            const long long t0 = clock64();
            while (!bar_try(drain, 0) && clock64() - t0 < p.wait_cycles) {
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        // a pair's second CTA tells the first what has arrived here
        uint32_t s = 0, sp = 0;
        bool ok = true;
        for (int32_t t = first; ok && t < tiles; t += step) {
            Tile x;
            ok = next_tile(x);  // (read like everyone's, so that its place can be filled again)
            for (int32_t kb = 2 * sb_lo; ok && kb < kb_hi; ++kb) {
                ok = wait_warp(own + 8 * s, sp, &abort_flag, p, kStatusTimeoutTma);
                if (ok && lane == 0) arrive_cluster(in_cta(full + 8 * s, 0));
                if (++s == (uint32_t)p.stages) s = 0, sp ^= 1;
            }
        }
        __syncwarp();
    } else if (warp < kMxEpiWarp0) {
        // scales to the tensor core's order, a stage of 512 values of K a turn; the first warp of a pair: W's rows, the second: the
        // tokens, in one or two parts of 128.  A lane copies the 16 bytes of its rows 32 c + lane into the pair's place when it is
        // done with a turn's, and is the only one to read them there.
        const uint32_t total = first < tiles ? (uint32_t)((tiles - first + step - 1) / step) * (uint32_t)(sb_hi - sb_lo) : 0;
        const uint32_t turn = (warp - kMxScaleWarp0) >> 1;
        const int part = (warp - kMxScaleWarp0) & 1, parts = part == 0 ? 1 : atoms - 1;
        const int64_t pitch = part == 0 ? p.w_lds : p.a_lds;
        const uint32_t raw = raw0 + turn * p.raw_bytes + part * kMxRowsW * 16 + lane * 16;
        int32_t lt = first, lsb = sb_lo;  // the stage to load next
        const uint8_t *base = nullptr;    // its rows: from `base` on, `pitch` apart, `rows` of them
        int rows = 0;
        bool ok = true;
        auto begin = [&] {
            Tile x;
            if (lt >= tiles || !(ok = ok && next_tile(x))) return;
            base = part == 0 ? p.w_scales + x.e * p.w_scales_stride + x.n0 * p.w_lds : p.a_scales + x.row0 * p.a_lds;
            rows = part == 0 ? p.N - x.n0 : x.rows;
        };
        auto skip = [&](int n) {  // n stages on
            lsb += n;
            while (lsb >= sb_hi) {
                lsb -= sb_hi - sb_lo;
                lt += step;
                begin();
            }
        };
        auto load = [&] {
            if (lt >= tiles || !ok) return;
            const uint32_t n = min(p.nb - 16 * lsb, 16);
            const uint8_t *src = base + 16 * lsb + lane * pitch;
            const int last = part == 0 ? 4 : (p.nt + 31) / 32;
            for (int c = 0; c < last; ++c, src += 32 * pitch) {
                const bool in = 32 * c + lane < rows;
                cpa16(raw + c * 512, in ? src : p.a_scales, in ? n : 0);  // (of a row past the end nothing is read: zeros)
            }
        };
        begin();
        skip(turn);
        load();
        // Two stages of scales in order: stage st takes the place of st - 2, whose MMAs then complete a phase of this pair's barrier:
        // one a turn, and none before the last has been seen, for the MMAs of st need what is written here
        uint32_t s = 0, fp = 0;
        int32_t sb = sb_lo;
        for (uint32_t st = 0; ok && st < total; ++st) {
            const int blocks = min(2, p.nkb - 2 * sb);
            if (++sb == sb_hi) sb = sb_lo;
            const bool mine = st % kMxScaleSets == turn;
            uint32_t w[2][4][4];
            if (mine) {
                asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        w[i][c][0] = w[i][c][1] = w[i][c][2] = w[i][c][3] = 0;
                        if (i < parts && (part == 0 || 128 * i + 32 * c < p.nt)) lds128(raw + i * kMxRowsW * 16 + c * 512, w[i][c]);
                    }
            }
            if (mine && st >= 2) {
                ok = wait_warp(sfree + 8 * turn, fp, &abort_flag, p, kStatusTimeoutFree);
                if (!ok) break;
                fp ^= 1;
            }
            if (mine) {
                const uint32_t dst = scale0 + (st & 1) * p.scale_bytes + part * kMxAtom + lane * 16;
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (i < parts) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + i * kMxAtom + j * kMxAtom * atoms),
                                         "r"(w[i][0][j]), "r"(w[i][1][j]), "r"(w[i][2][j]), "r"(w[i][3][j])
                                         : "memory");
                    }
                fence_async_smem();
                __syncwarp();
            }
            for (int i = 0; i < blocks; ++i) {
                if (mine && lane == 0) {
                    if constexpr (PAIR) arrive_cluster(in_cta(full + 8 * s, 0));
                    else bar_arrive(full + 8 * s);
                }
                if (++s == (uint32_t)p.stages) s = 0;
            }
            if (mine) {  // (what is overwritten has gone into the stores above)
                skip(kMxScaleSets);
                load();
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp < kMxTileWarp) {
        const uint32_t quarter = (uint32_t)(warp & 3) << 21;  // lane field of the warp's 32 lanes
        const int part = (warp - kMxEpiWarp0) >> 2, row = 32 * (warp & 3) + lane;
        const uint32_t patch = patch0 + (warp - kMxEpiWarp0) * kMxPatch;
        const uint32_t free0 = PAIR ? in_cta(aempty, 0) : aempty;
        uint32_t n = 0;
        auto bias_of = [&](const Tile &y) {
            const int nn = y.n0 + row;
            return !SPLIT && p.bias && nn < p.N ? p.bias[(int64_t)y.e * p.N + nn] : 0.0f;
        };
        Tile next = {};  // (read, with its bias, while a tile is stored)
        float next_bias = 0.0f;
        if (first < tiles && next_tile(next)) next_bias = bias_of(next);
        for (int32_t t = first; t < tiles; t += step, ++n) {
            const uint32_t acc = n & 1;
            x = next;
            const float bias = next_bias;
            const int nn = x.n0 + row;
            if (!wait_warp(afull + 8 * acc, (n >> 1) & 1, &abort_flag, p, kStatusTimeoutMma)) break;
            fence_after();
            if (t + step < tiles && next_tile(next)) next_bias = bias_of(next);
            for (int c0 = 16 * part; c0 < x.rows; c0 += 64) {
                uint32_t u[16];
                tld<16>(tmem + quarter + acc * kMxMaxTok + c0, u);
                twait<16>(u);
                float v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(u[i]);
                if constexpr (SPLIT) {  // this CTA's part of the sums: [token][row of W] over the stages, which are all read
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        asm volatile("st.shared.f32 [%0], %1;" ::"r"(data0 + ((c0 + i) * kMxRowsW + row) * 4), "f"(v[i]) : "memory");
                } else {
                    store_chunk<ACT, T>(p, v, x, c0, nn, bias, patch, lane);
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) arrive_cluster(free0 + 8 * acc);
                else bar_arrive(aempty + 8 * acc);
            }
        }
    } else if constexpr (!SPLIT) {
        // the tiles of this CTA, one after the other
        uint32_t n = 0;
        for (int32_t t = first; t < tiles; t += step, ++n) {
            const uint32_t i = n % kMxTiles;
            if (n >= kMxTiles && !wait_warp(tfree + 8 * i, (n / kMxTiles - 1) & 1, &abort_flag, p, kStatusTimeoutFree)) break;
            if (n > 0) {
                const Tile y = find_tile<MODE>(p, tab, tab_id, experts, t, rank);
                if (lane == 0) tile_ring[i] = make_int4(y.e, y.row0, y.rows, y.n0);
            }
            if (lane == 0) bar_arrive(tfull + 8 * i);
            __syncwarp();
        }
    }
    if constexpr (SPLIT) {
        __syncwarp();
        cluster_sync();
        if (first < tiles && !abort_flag && warp >= kMxEpiWarp0 && warp < kMxTileWarp) {
            // each warp of the cluster finishes the 32 rows of W of a quarter for four tokens at a time
            const int w = warp - kMxEpiWarp0, units = 4 * ((x.rows + 3) / 4);
            for (int u = w + kMxEpiWarps * rank; u < units; u += kMxEpiWarps * p.splits) {
                const int c0 = u & ~3, row = 32 * (u & 3) + lane, nn = x.n0 + row;
                const float bias = p.bias && nn < p.N ? p.bias[(int64_t)x.e * p.N + nn] : 0.0f;
                float v[8][4], z[4];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.splits) {
                        const uint32_t at = in_cta(data0 + (c0 * kMxRowsW + row) * 4, r);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r][i]) : "r"(at + i * kMxRowsW * 4) : "memory");
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    z[i] = v[0][i];
#pragma unroll
                    for (int r = 1; r < 8; ++r)
                        if (r < p.splits) z[i] += v[r][i];
                    z[i] += bias;
                }
                constexpr bool kGate = ACT == ILW_ACT_SILU_GATE;
                const int width = kGate ? p.N / 2 : p.N, col = kGate ? nn >> 1 : nn;
                if constexpr (ACT == ILW_ACT_GELU) gelu2(z[0], z[1]), gelu2(z[2], z[3]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (kGate) z[i] = silu_gate<T>(z[i], __shfl_down_sync(0xffffffffu, z[i], 1));  // (even lanes: gate, odd: gated)
                    if (c0 + i < x.rows && col < width && !(kGate && lane & 1)) ((T *)p.Y)[(int64_t)(x.row0 + c0 + i) * p.ldy + col] = to_out<T>(z[i]);
                }
            }
        }
    }
    // rows of no expert are zero
    if (p.offsets) {
        const int64_t wide = ACT == ILW_ACT_SILU_GATE ? p.N / 2 : p.N;
        const int64_t head = s_head, tail = s_tail, total = (head + p.M - tail) * wide;
        for (int64_t i = blockIdx.x * (int64_t)kMxThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kMxThreads) {
            const int64_t r = i / wide;
            ((T *)p.Y)[(r < head ? r : r - head + tail) * p.ldy + (i - r * wide)] = to_out<T>(0.0f);
        }
    }
    fence_before();
    __syncwarp();
    if constexpr (MODE != MX_ONE) cluster_sync();  // nothing of this CTA is read or signalled any more
    else __syncthreads();
    if (warp == 3) {
        fence_after();
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int ACT, typename T, int MODE>
cudaError_t launch_mode(const MxParams &p, int grid, size_t smem, cudaStream_t s) {
    static SmemLimit limit;
    cudaError_t e = raise_smem_limit(limit, (const void *)mx_gemm_kernel<ACT, T, MODE>, kMxSmemLimit);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = kMxThreads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = MODE == MX_SPLIT ? p.splits : 2;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = MODE == MX_ONE ? 1 : 2;
    e = cudaLaunchKernelEx(&cfg, mx_gemm_kernel<ACT, T, MODE>, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}
template <int ACT, typename T>
cudaError_t launch_act(const MxParams &p, int grid, size_t smem, cudaStream_t s) {
    if (p.mode == MX_SPLIT) return launch_mode<ACT, T, MX_SPLIT>(p, grid, smem, s);
    if (p.mode == MX_PAIR) return launch_mode<ACT, T, MX_PAIR>(p, grid, smem, s);
    return launch_mode<ACT, T, MX_ONE>(p, grid, smem, s);
}

}  // namespace

template <typename T>
cudaError_t launch_mx(const MxParams &p, int32_t act, int grid, size_t smem, cudaStream_t s) {
    if (act == ILW_ACT_GELU) return launch_act<ILW_ACT_GELU, T>(p, grid, smem, s);
    if (act == ILW_ACT_SILU_GATE) return launch_act<ILW_ACT_SILU_GATE, T>(p, grid, smem, s);
    return launch_act<ILW_ACT_NONE, T>(p, grid, smem, s);
}

}  // namespace ilw
