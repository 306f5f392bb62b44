#pragma once
// i8_gemm.cuh -- products of int8 rows with float scales on the 5th-generation tensor cores (sm_103a): Y = act(sa sw A W^T + bias),
// for one weight or for one weight per expert with ragged groups of rows.
//
//   z[m, n] = sa[m] sw[n] sum_k a[m, k] w[n, k] + bias[n]
//
// This chip's tcgen05 has no int8 kind.  Every int8 number is an fp16 number, so the codes are widened on the way to tcgen05.mma.kind::f16,
// whose products of them are exact and whose fp32 sums are exact below 2^24, so those of 1024 of K are.  HBM and L2 carry 8 bits all the same.
//
// Past 2^24 the tensor core cuts off what does not fit, at every 16 of K and always toward zero: sums of codes of one sign lose 4e-6 of themselves at K = 8192,
// 6e-5 at 32768, 5e-4 at 131071 (a library's fp32 product 1e-6, 2e-6, 5e-6).  Results of two bytes round by more than that up to kI8ShortK.  For
// fp32 results past K = 1024, and for others past kI8ShortK, the sums of each 1024 of K are taken out of tensor memory and added up in shared
// memory as 32-bit whole numbers, by the epilogue's warps while the next 1024 are summed in the other accumulator.  The room for that is a tile of
// 128 tokens' at most.  8192 cubed with fp32 results takes 814 us so (in fp32 sums 567), 2000 cubed 22.3 (19.5), 300 x 4096 x 4096 19.2 (19.8).
//
// Widening is what has to keep up with the tensor core.  64 of K of a tile are 384 clocks of MMAs (192 tokens), in which shared memory moves
// 48 KB.  The codes come by TMA (14 KB in a pair of SMs) and are read once; W's rows, the lanes of a tile, go from registers to tensor
// memory, where the MMA takes its first operand from without touching shared memory; only the tokens are written back there, as 12 KB of
// fp16 that the MMA reads.  (0x6400 | b ^ 0x80 is 1152 + b in fp16: an exclusive or, two byte permutes and two packed subtractions
// widen four codes.)  The chain of a stage, from its barrier over loads, arithmetic and stores to the barrier of the MMAs, is some 1300
// clocks long (loads 350, W's rows 290, the tokens 400, barriers 250), so four sets of warps work at four stages: with three 8192
// cubed took a tenth more, with two a fifth.  It takes 549 us, 2.00 PFLOP/s, the rate of a bf16 product of the library (1.94); at that point a
// stage takes 430 of the 384 clocks that its MMAs need, in tiles of 128 tokens 390 of 256.  A short K is bound by the epilogue, 16 tokens
// of 32 rows a warp and some 900 clocks (reading tensor memory 330, scales 130, stores 450; GELU 700 more).  Taken back: codes widened before
// their place is free (780 us), the next stage's loaded before this one is handed over (617), the next sums on their way from tensor
// memory while the last are stored (12800 x 1536 x 384: 24.0 us, without 21.0), 32 tokens at a time (26.9).
//
// Tiles and the three forms (one CTA a tile, several CTAs of a cluster to a tile's K, pairs of SMs) are those of mx_gemm.cuh.
//
// One CTA per SM, 28 warps: the loads of W and of the tokens, the MMAs, the list of tiles, four sets of four warps that widen (in turn: 64 of
// K a turn, a set's warp the 32 rows of W whose lanes it reaches and a quarter of the tokens), 8 epilogue warps.  Codes wait in a ring of
// stages of 128 of K, widened ones in a ring of four of 64 of K.  A set always takes the same of these four, and with an even number of
// stages of codes and whole blocks of 128 of K always the same halves of the same stages: it sees every phase of the
// barriers that it waits on, so none is taken for the one before.  Two accumulators let a tile's epilogue overlap the next tile's MMAs.
//
// Every mbarrier wait is bounded, as in mx_gemm.cuh.
#include <climits>
#include <cstdint>
#include <type_traits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "i8_kernels.h"
#include "ilwdetr.h"
#include "tile_gemm.cuh"

namespace ilw {

constexpr int kI8MaxTok = 192;  // tokens a tile; a multiple of 32, as tiles of pairs are
constexpr int kI8MaxTokOne = 128;  // of one CTA, which with more has no room for two stages of codes to spare
constexpr int kI8LongTok = 128;  // of any form where sums are kept in shared memory
constexpr int kI8ExactK = 1024;     // 2^14 kI8ExactK = 2^24
constexpr int kI8ShortK = 16384;    // 2^-23 kI8ShortK / 16 = 2^-13 of the sum of magnitudes at most, and half of it as a rule; fp16 rounds by 2^-11
constexpr int kI8MaxStages = 8, kI8MinStages = 2;
constexpr int kI8Sets = 4;      // sets of four widening warps
constexpr int kI8MaxWide = 2 * kI8Sets;  // stages of widened codes at most: one or two a set
constexpr int kI8TileWarp = 3, kI8WidenWarp0 = 4, kI8EpiWarp0 = kI8WidenWarp0 + 4 * kI8Sets, kI8EpiWarps = 8;
constexpr int kI8Warps = kI8EpiWarp0 + kI8EpiWarps, kI8Threads = 32 * kI8Warps;
constexpr int kI8Tiles = 16;    // tiles found ahead
constexpr int kI8Patch = 512;   // bytes of shared memory in which an epilogue warp turns 2-byte results
constexpr int kI8SmemLimit = 224 * 1024;  // dynamic; barriers and token scales are static
static_assert(kI8Sets == 4 && kI8MaxStages % 2 == 0 && kI8MinStages % 2 == 0, "a set has its own stages");
static_assert(kI8WidenWarp0 % 4 == 0 && kI8EpiWarp0 % 4 == 0, "a warp reaches the lanes of its number modulo 4");

struct I8Params {
    CUtensorMap wc, ac[4];  // codes of W [E, N, K]; of A [M, K] in boxes of 16, 32, 64 and 128 rows
    const float *a_scales, *w_scales;
    const int32_t *offsets;
    const float *bias;
    void *Y;
    int64_t ldy, M;
    int32_t N, E;
    int32_t nkb;            // K in blocks of 128: a stage of codes, two of widened ones
    int32_t wtiles;         // tiles of rows of W (128, or 256 a pair)
    uint32_t wdiv_m, wdiv_s;  // division by wtiles
    int32_t nt;             // most tokens a tile, a multiple of 16 (a pair's: of 32)
    int32_t stages;         // stages of codes
    int32_t wides;          // stages of widened codes
    int32_t stage_bytes, wide_bytes;
    int32_t wide;           // 2-byte rows of Y take 16-byte stores
    int32_t splits;         // CTAs of a cluster that share a tile's K (TILE_SPLIT)
    int32_t part;           // (LONG) stages of 64 of K after which sums are taken out of an accumulator
    int32_t sums_bytes;     // (LONG) whole sums [token][row of W] of a tile
    int32_t mode;
    int32_t dbg_skip;
    long long wait_cycles;
    int *status;
};

// LONG: sums are taken out of the accumulators every p.part stages.
template <typename T, bool LONG>
cudaError_t launch_i8(const I8Params &p, int32_t act, int grid, size_t smem, cudaStream_t s);

namespace {

// D += A B of 16 of K: A [128 or 2 x 128 rows] in tensor memory, B the tokens' fp16 rows.  By one lane.
template <bool PAIR>
__device__ __forceinline__ void mma_f16(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    if constexpr (PAIR)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a),
                     "l"(b), "r"(idesc), "r"(acc)
                     : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d), "r"(a),
                     "l"(b), "r"(idesc), "r"(acc)
                     : "memory");
}
// fp16 operands (format 0), both K-major, fp32 sums, M = m, N = n
__device__ __forceinline__ uint32_t idesc_f16(uint32_t m, uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((m >> 4) << 24); }
// Four codes to fp16.
__device__ __forceinline__ void widen4(uint32_t w, uint32_t &lo, uint32_t &hi) {
    const __half2 base = __half2half2(__ushort_as_half((unsigned short)0x6480));
    const uint32_t x = w ^ 0x80808080u;
    uint32_t a = __byte_perm(x, 0x64646464u, 0x4140), b = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 l = __hsub2(*reinterpret_cast<__half2 *>(&a), base), h = __hsub2(*reinterpret_cast<__half2 *>(&b), base);
    lo = *reinterpret_cast<const uint32_t *>(&l);
    hi = *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ void sts32(uint32_t a, int32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ int32_t lds32(uint32_t a) {
    int32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
// 16 columns of this thread's lane of tensor memory
__device__ __forceinline__ void tst16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
                 "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                 "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
                 : "memory");
}

// Two values to 2 bytes each, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pair_out(float a, float b);
template <> __device__ __forceinline__ uint32_t pair_out<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
template <> __device__ __forceinline__ uint32_t pair_out<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Four 8 x 8 matrices of 2-byte values, each transposed; lane l gives the address of row l % 8 of matrix l / 8.
__device__ __forceinline__ void load_turned(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

// One warp's 32 rows of W (this lane: row n) x 16 tokens (c0 .. c0 + 15 of the tile): activation and stores.  A lane holds one output of
// 16 tokens.  Where rows of Y allow it (`wide`), 2-byte results pass through the warp's patch of shared memory, [output][token], two to
// a word, and come back transposed, the outputs of a token side by side in 16-byte (gated: 8-byte) pieces: some 20 instructions where
// 16 stores of 2 bytes with their addresses and conditions are 100.
template <int ACT, typename T>
__device__ __forceinline__ void store_tokens(const I8Params &p, float (&v)[16], const Tile &t, int c0, int n, uint32_t patch, int lane) {
    const int left = t.rows - c0;
    constexpr bool kGate = ACT == ILW_ACT_SILU_GATE;
    const int width = kGate ? p.N / 2 : p.N;
    if constexpr (kGate) {
        // even lanes hold gates, odd lanes the rows they gate: the even lane of a pair finishes the first eight tokens, the odd one the others
        const bool odd = lane & 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float other = __shfl_xor_sync(0xffffffffu, odd ? v[i] : v[8 + i], 1);
            v[i] = silu_gate<T>(odd ? other : v[i], odd ? v[8 + i] : other);
        }
    } else if constexpr (ACT == ILW_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) gelu2(v[2 * i], v[2 * i + 1]);
    }
    const int out0 = kGate ? (n - lane) >> 1 : n - lane;  // first output of the warp
    if constexpr (sizeof(T) == 2) {
        if (p.wide) {
            // place of row r of the patch: such that neither the eight lanes that write together nor the eight rows of a matrix meet in a bank
            auto place = [&](int r) { return patch + 16 * (r ^ (r >> 3 & 3) << 1); };
            // lane 4 i + j: token i of eight; rows 2 j and 2 j + 1 of each matrix
            const int m = lane >> 3, r = lane & 7, i = lane >> 2, j = lane & 3;
            uint32_t q[4];
            if constexpr (kGate) {  // matrices 0, 1: tokens 0 .. 7, outputs 4 j .. 4 j + 3; matrices 2, 3: tokens 8 .. 15
                sts128(place(lane >> 1 | (lane & 1) << 4), pair_out<T>(v[0], v[1]), pair_out<T>(v[2], v[3]), pair_out<T>(v[4], v[5]), pair_out<T>(v[6], v[7]));
                __syncwarp();
                load_turned(place(4 * (r >> 1) + 2 * (m & 1) + (r & 1) | (m >> 1) << 4), q);
                T *y = (T *)p.Y + (int64_t)(t.row0 + c0 + i) * p.ldy + out0 + 4 * j;
                const bool in = out0 + 4 * j < width;
                if (in && i < left) *(uint2 *)y = make_uint2(q[0], q[1]);
                if (in && i + 8 < left) *(uint2 *)(y + 8 * p.ldy) = make_uint2(q[2], q[3]);
                __syncwarp();
            } else {
                T *y = (T *)p.Y + (int64_t)(t.row0 + c0 + i) * p.ldy + out0 + 8 * j;
                const bool in = out0 + 8 * j < width;
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // eight tokens: outputs 8 j + 2 m, + 1 from matrix m
                    sts128(place(lane), pair_out<T>(v[8 * h], v[8 * h + 1]), pair_out<T>(v[8 * h + 2], v[8 * h + 3]), pair_out<T>(v[8 * h + 4], v[8 * h + 5]),
                           pair_out<T>(v[8 * h + 6], v[8 * h + 7]));
                    __syncwarp();
                    load_turned(place(8 * (r >> 1) + 2 * m + (r & 1)), q);
                    if (in && i + 8 * h < left) *(uint4 *)(y + 8 * h * p.ldy) = make_uint4(q[0], q[1], q[2], q[3]);
                    __syncwarp();
                }
            }
            return;
        }
    }
    const int col = out0 + (kGate ? lane >> 1 : lane), first = kGate ? 8 * (lane & 1) : 0;
    constexpr int kVals = kGate ? 8 : 16;
    T *y = (T *)p.Y + (int64_t)(t.row0 + c0 + first) * p.ldy + col;
    if (col < width) {
        if (left >= 16) {
#pragma unroll
            for (int i = 0; i < kVals; ++i) y[i * p.ldy] = to_out<T>(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kVals; ++i)
                if (first + i < left) y[i * p.ldy] = to_out<T>(v[i]);
        }
    }
}

template <int ACT, typename T, int MODE, bool LONG>
__global__ void __launch_bounds__(kI8Threads, 1) i8_gemm_kernel(const __grid_constant__ I8Params p) {
    constexpr bool SPLIT = MODE == TILE_SPLIT, PAIR = MODE == TILE_PAIR;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kI8MaxStages + 2 * kI8MaxWide + 2 * kI8Tiles + 5];
    __shared__ int4 tile_ring[kI8Tiles];
    __shared__ __align__(16) float token_scales[kI8EpiWarps][2][16];
    __shared__ uint32_t tmem_base;
    __shared__ volatile int abort_flag;
    __shared__ int32_t s_experts, s_head, s_tail;  // experts with rows; rows before the first and from the end of the last
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t data0 = (su32(smem_raw) + 1023) & ~1023u;
    const uint32_t wide0 = data0 + p.stages * p.stage_bytes, sums0 = wide0 + p.wides * p.wide_bytes, patch0 = LONG ? sums0 + p.sums_bytes : sums0;
    TileExpert *tab = (TileExpert *)(smem_raw + (patch0 - su32(smem_raw)) + (p.wide ? kI8EpiWarps * kI8Patch : 0));
    int32_t *tab_id = (int32_t *)(tab + p.E + 1);

    uint32_t next_bar = su32(bars);
    auto take = [&](int n) {
        const uint32_t at = next_bar;
        next_bar += 8 * n;
        return at;
    };
    const uint32_t full = take(kI8MaxStages), empty = take(kI8MaxStages);  // stages of codes, a CTA's own
    const uint32_t ready = take(kI8MaxWide), wfree = take(kI8MaxWide);           // stages of widened codes (a pair's `ready`: at the first CTA, of both)
    const uint32_t tfull = take(kI8Tiles), tfree = take(kI8Tiles);         // tiles found, and read by every warp
    const uint32_t afull = take(2), aempty = take(2), drain = take(1);     // accumulators

    const uint32_t rank = SPLIT ? blockIdx.x % p.splits : PAIR ? blockIdx.x & 1 : 0;
    const bool leader = !PAIR || rank == 0;
    const int32_t group = SPLIT ? p.splits : PAIR ? 2 : 1, first = (int32_t)blockIdx.x / group;
    if (warp == 0) {
        if (lane == 0) abort_flag = 0;
        if (lane < kI8MaxStages) {
            bar_init(full + 8 * lane, 2);
            bar_init(empty + 8 * lane, 8);  // four warps for each half of a block of K
        }
        if (lane < kI8MaxWide) {
            bar_init(ready + 8 * lane, PAIR ? 8 : 4);
            bar_init(wfree + 8 * lane, 1);
        }
        if (lane < kI8Tiles) {
            bar_init(tfull + 8 * lane, 1);
            bar_init(tfree + 8 * lane, kI8Warps - 1);
        }
        if (lane < 2) {
            bar_init(afull + 8 * lane, 1);
            bar_init(aempty + 8 * lane, PAIR ? 2 * kI8EpiWarps : kI8EpiWarps);
        }
        if (lane == 0) bar_init(drain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x == 32) {
        prefetch_map(&p.wc);
        prefetch_map(&p.ac[0]);
    }
    if (warp == kI8TileWarp) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(su32(&tmem_base)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(su32(&tmem_base)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    grid_wait();
    if (warp == 2) {
        int32_t sum, count, head, tail;
        list_tiles<PAIR ? 32 : 16>(p, tab, tab_id, lane, sum, count, head, tail);
        if (lane == 0) {
            s_experts = count;
            s_head = head;
            s_tail = tail;
        }
        if (first < sum * p.wtiles) {  // the first tile at once; the others follow from a warp of their own
            const Tile y = find_tile<MODE>(p, tab, tab_id, count, first, rank);
            if (lane == 0) tile_ring[0] = make_int4(y.e, y.row0, y.rows, y.n0);
        }
    }
    fence_before();
    if constexpr (PAIR) cluster_sync();
    else __syncthreads();
    fence_after();
    const uint32_t tmem = uniform(tmem_base), wcol = tmem + 2 * p.nt;  // columns: two accumulators, then the widened rows of W, 32 a stage
    const int experts = s_experts;
    const int32_t tiles = tab[experts].start * p.wtiles;
    const int32_t step = (int32_t)gridDim.x / group;
    const int32_t kb_lo = SPLIT ? (int32_t)((int64_t)p.nkb * rank / p.splits) : 0;
    const int32_t kb_hi = SPLIT ? (int32_t)((int64_t)p.nkb * (rank + 1) / p.splits) : p.nkb;
    const int32_t ks_lo = 2 * kb_lo, ks_hi = 2 * kb_hi;
    // the next tile of this CTA, as its warp has found it (by a whole warp; false when a wait ran out)
    uint32_t tiles_read = 0;
    auto next_tile = [&](Tile &x) {
        if constexpr (SPLIT) {  // (the only one)
            const int4 v = tile_ring[0];
            x = Tile{v.x, v.y, v.z, v.w};
            return true;
        }
        const uint32_t i = tiles_read % kI8Tiles;
        if (tiles_read > 0 && !wait_lean(tfull + 8 * i, (tiles_read / kI8Tiles) & 1, &abort_flag, p, kStatusTimeoutOperand)) return false;
        const int4 v = tile_ring[i];
        x = Tile{v.x, v.y, v.z, v.w};
        __syncwarp();
        if (lane == 0) bar_arrive(tfree + 8 * i);
        ++tiles_read;
        return true;
    };
    Tile x = {};  // (an epilogue warp's)
    auto mma_tokens = [&](const Tile &x) { return PAIR ? (x.rows + 31) & ~31 : (x.rows + 15) & ~15; };
    // tokens whose codes this CTA loads and widens: of a pair half of them each
    auto my_tokens = [&](const Tile &x) { return PAIR ? mma_tokens(x) / 2 : mma_tokens(x); };

    // (SPLIT: a cluster has one tile at most, the host gives it as many clusters as there can be tiles)
    if (warp == 0 || warp == 2) {
        // loads of the codes: warp 0 of W, warp 2 of the tokens
        const uint32_t one = elect_one();
        uint32_t it = 0, s = 0, sp = 1;  // stages loaded, the place in the ring, the parity of a free one
        bool ok = true;
        for (int32_t t = first; t < tiles; t += step) {
            Tile x;
            ok = ok && next_tile(x);
            if (!ok) break;
            x.e = uniform(x.e), x.row0 = uniform(x.row0), x.rows = uniform(x.rows), x.n0 = uniform(x.n0);
            const int part = my_tokens(x), row = x.row0 + (PAIR ? (int)rank * part : 0);
            const int units = part >> 4;
            const uint32_t bytes = warp == 0 ? kTileRowsW * 128 : units * 2048;
            if (one) {
                for (int32_t kb = kb_lo; kb < kb_hi; ++kb) {
                    if (!wait_lane(empty + 8 * s, sp, &abort_flag, p, kStatusTimeoutFree)) {
                        ok = false;
                        break;
                    }
                    const uint32_t d = data0 + s * p.stage_bytes + (warp == 0 ? 0 : kTileRowsW * 128), db = full + 8 * s;
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
                while (!bar_try(full + 8 * (i % p.stages), (i / p.stages) & 1) && clock64() - t0 < 2000000) {
                }
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t one = elect_one();
        const int32_t part = LONG ? p.part : ks_hi - ks_lo;  // of K, to one accumulator
        uint32_t n = 0, cs = 0, cp = 0;
        const uint64_t desc0 = desc_sw128(wide0);
        uint64_t bd = desc0;
        uint32_t at = wcol;
        bool ok = true;
        for (int32_t t = first; ok && t < tiles; t += step) {
            Tile x;
            ok = next_tile(x);
            if (!ok || !leader) continue;  // (a pair's second CTA only reads its tiles, so that their places can be filled again)
            const uint32_t id = idesc_f16(PAIR ? 256 : 128, uniform(mma_tokens(x)));
            for (int32_t lo = ks_lo; ok && lo < ks_hi; lo += part, ++n) {
                const uint32_t acc = n & 1, d = tmem + acc * p.nt;
                const int32_t hi = LONG ? min(lo + part, ks_hi) : ks_hi;
                ok = wait_lean(aempty + 8 * acc, ((n >> 1) & 1) ^ 1, &abort_flag, p, kStatusTimeoutFree);
                if (!ok) break;
                fence_after();
                if (one) {
                    for (int32_t ks = lo; ks < hi; ++ks) {
                        if (!wait_lane(ready + 8 * cs, cp, &abort_flag, p, kStatusTimeoutOperand)) {
                            ok = false;
                            break;
                        }
                        fence_after();
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma_f16<PAIR>(d, at + 8 * j, bd + 2 * j, id, ks > lo || j > 0);
                        commit_mma<PAIR>(wfree + 8 * cs);
                        at += 32;
                        bd += p.wide_bytes / 16;
                        if (++cs == (uint32_t)p.wides) cs = 0, cp ^= 1, at = wcol, bd = desc0;
                    }
                    if (ok) commit_mma<PAIR>(afull + 8 * acc);
                }
                ok = __all_sync(0xffffffffu, ok);
            }
        }
        if (!ok && one && leader) {  // the MMAs in flight end before tensor memory is freed
            commit_mma<PAIR>(drain, true);
            const long long t0 = clock64();
            while (!bar_try(drain, 0) && clock64() - t0 < p.wait_cycles) {
            }
        }
        __syncwarp();
    } else if (warp == kI8TileWarp) {
        // the tiles of this CTA, one after the other
        if constexpr (!SPLIT) {
            uint32_t n = 0;
            for (int32_t t = first; t < tiles; t += step, ++n) {
                const uint32_t i = n % kI8Tiles;
                if (n >= kI8Tiles && !wait_lean(tfree + 8 * i, (n / kI8Tiles - 1) & 1, &abort_flag, p, kStatusTimeoutFree)) break;
                if (n > 0) {
                    const Tile y = find_tile<MODE>(p, tab, tab_id, experts, t, rank);
                    if (lane == 0) tile_ring[i] = make_int4(y.e, y.row0, y.rows, y.n0);
                }
                if (lane == 0) bar_arrive(tfull + 8 * i);
                __syncwarp();
            }
        }
    } else if (warp < kI8EpiWarp0) {
        // widening: this set's stages of 64 of K.  Lane i of warp q: row 32 q + i of W, to its lane of tensor memory; of the tokens eight
        // rows and four pieces of 16 codes at a time, so that the eight lanes that are served together meet in no bank
        const uint32_t set = (warp - kI8WidenWarp0) >> 2, q = warp & 3;
        const uint32_t wrow = (32 * q + lane) * 128, wx = lane & 7;
        const uint32_t trow = lane & 7, tc = lane >> 3;
        constexpr int kHeld = kI8MaxTok / 64;  // pieces of a warp: all that a pair's CTA has
        const uint32_t tdst = wcol + (q << 21), ready0 = PAIR ? in_cta(ready, 0) : ready;
        const uint32_t nks = ks_hi - ks_lo;
        uint32_t g = 0;             // stages of widened codes before this tile (an even number)
        uint32_t cs = set, cp = 1;  // this set's next stage of widened codes, the parity of a free one
        bool ok = true;
        for (int32_t t = first; ok && t < tiles; t += step, g += nks) {
            Tile x;
            ok = next_tile(x);
            if (!ok) break;
            const int groups = my_tokens(x) >> 3;
            uint32_t ks = (set - g) & (kI8Sets - 1);
            const uint32_t block = (g + ks) >> 1, h = set & 1;
            uint32_t s = block % p.stages, sp = (block / p.stages) & 1;
            uint32_t w[4][4], a[kHeld][4];
            auto load = [&] {
                const uint32_t src = data0 + s * p.stage_bytes, tsrc = src + kTileRowsW * 128 + (8 * q + trow) * 128 + (((4 * h + tc) ^ trow) << 4);
#pragma unroll
                for (int c = 0; c < 4; ++c) lds128(src + wrow + (((4 * h + c) ^ wx) << 4), w[c]);
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if ((int)q + 4 * i < groups) lds128(tsrc + i * 4096, a[i]);
            };
            for (; ks < nks; ks += kI8Sets) {
                ok = wait_lean(full + 8 * s, sp, &abort_flag, p, kStatusTimeoutTma);
                if (!ok) break;
                load();
                ok = wait_lean<120>(wfree + 8 * cs, cp, &abort_flag, p, kStatusTimeoutFree);
                if (!ok) break;
                fence_after();
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t v[16];
#pragma unroll
                    for (int j = 0; j < 8; ++j) widen4(w[2 * i + j / 4][j % 4], v[2 * j], v[2 * j + 1]);
                    tst16(tdst + 32 * cs + 16 * i, v);
                }
                const uint32_t trows = wide0 + cs * p.wide_bytes + (8 * q + trow) * 128;
                auto put = [&](int i, const uint32_t (&b)[4]) {
                    uint32_t v[8];
#pragma unroll
                    for (int j = 0; j < 4; ++j) widen4(b[j], v[2 * j], v[2 * j + 1]);
                    sts128(trows + i * 4096 + (((2 * tc) ^ trow) << 4), v[0], v[1], v[2], v[3]);
                    sts128(trows + i * 4096 + (((2 * tc + 1) ^ trow) << 4), v[4], v[5], v[6], v[7]);
                };
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if ((int)q + 4 * i < groups) put(i, a[i]);
                if constexpr (!PAIR) {
                    const uint32_t tsrc = data0 + s * p.stage_bytes + kTileRowsW * 128 + (8 * q + trow) * 128 + (((4 * h + tc) ^ trow) << 4);
#pragma unroll
                    for (int i = kHeld; i < kI8MaxTokOne / 32; ++i)
                        if ((int)q + 4 * i < groups) {
                            lds128(tsrc + i * 4096, a[0]);
                            put(i, a[0]);
                        }
                }
                const uint32_t done = s;
                s += kI8Sets / 2;
                if (s >= (uint32_t)p.stages) s -= p.stages, sp ^= 1;
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                fence_before();
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) arrive_cluster(ready0 + 8 * cs);
                    else bar_arrive(ready + 8 * cs);
                    bar_arrive(empty + 8 * done);
                }
                cs += kI8Sets;
                if (cs >= (uint32_t)p.wides) cs = set, cp ^= 1;
            }
        }
        __syncwarp();
    } else {
        const uint32_t quarter = (uint32_t)(warp & 3) << 21;  // lane field of the warp's 32 lanes
        const int part = (warp - kI8EpiWarp0) >> 2, row = 32 * (warp & 3) + lane;
        const uint32_t patch = patch0 + (warp - kI8EpiWarp0) * kI8Patch;
        const uint32_t free0 = PAIR ? in_cta(aempty, 0) : aempty;
        uint32_t n = 0, turn = 0;
        float next_scale = 0.0f, next_bias = 0.0f;
        auto read_row = [&](const Tile &y) {  // of this lane's row of W
            const int nn = y.n0 + row;
            if (SPLIT || nn >= p.N) return;
            next_scale = __ldg(p.w_scales + (int64_t)y.e * p.N + nn);
            if (p.bias) next_bias = __ldg(p.bias + (int64_t)y.e * p.N + nn);
        };
        // (LONG) all parts of K but the last to the whole sums: each thread its own, which no other reads
        auto take_parts = [&](const Tile &y, uint32_t &n) {
            for (int32_t lo = ks_lo; lo + p.part < ks_hi; lo += p.part, ++n) {
                const uint32_t acc = n & 1;
                if (!wait_lean<200>(afull + 8 * acc, (n >> 1) & 1, &abort_flag, p, kStatusTimeoutMma)) return false;
                fence_after();
                for (int c0 = 16 * part; c0 < y.rows; c0 += 4 * kI8EpiWarps) {
                    uint32_t u[16];
                    tld<16>(tmem + quarter + acc * p.nt + c0, u);
                    twait<16>(u);
                    const uint32_t at = sums0 + (c0 * kTileRowsW + row) * 4;
#pragma unroll
                    for (int i = 0; i < 16; ++i) sts32(at + i * kTileRowsW * 4, __float2int_rn(__uint_as_float(u[i])) + (lo > ks_lo ? lds32(at + i * kTileRowsW * 4) : 0));
                }
                fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) arrive_cluster(free0 + 8 * acc);
                    else bar_arrive(aempty + 8 * acc);
                }
            }
            return true;
        };
        Tile next = {};  // (read, with its scale and bias, while a tile is stored)
        if (first < tiles && next_tile(next)) read_row(next);
        const bool parts = LONG && p.part < ks_hi - ks_lo;
        for (int32_t t = first; t < tiles; t += step, ++n) {
            x = next;
            if (LONG && !take_parts(x, n)) break;
            const uint32_t acc = n & 1;
            const float scale = next_scale, bias = next_bias;
            const int nn = x.n0 + row;
            // scales of 16 tokens, a lane one of them
            auto token_scale = [&](int c0) { return !SPLIT && c0 + (lane & 15) < x.rows ? __ldg(p.a_scales + x.row0 + c0 + (lane & 15)) : 0.0f; };
            float sa = token_scale(16 * part);
            if (!wait_lean<200>(afull + 8 * acc, (n >> 1) & 1, &abort_flag, p, kStatusTimeoutMma)) break;
            fence_after();
            if (t + step < tiles && next_tile(next)) read_row(next);
            // a tile's columns, with the order of scaled_sum known where the warp's rows have one (as a choice for each value it took the GELU of 12800 x 1536 x
            // 384 from 30.6 us to 31.8)
            auto columns = [&](auto channel_first) {
                for (int c0 = 16 * part; c0 < x.rows; c0 += 4 * kI8EpiWarps) {
                    uint32_t u[16];
                    tld<16>(tmem + quarter + acc * p.nt + c0, u);
                    const uint32_t scales = su32(token_scales[warp - kI8EpiWarp0][turn & 1]);
                    if constexpr (!SPLIT) {  // (through shared memory every lane gets all 16)
                        if (lane < 16) asm volatile("st.shared.f32 [%0], %1;" ::"r"(scales + 4 * lane), "f"(sa) : "memory");
                        __syncwarp();
                        ++turn;
                    }
                    sa = token_scale(c0 + 4 * kI8EpiWarps);
                    twait<16>(u);
                    if (SPLIT || LONG) {  // this CTA's whole sums
                        const uint32_t at = (c0 * kTileRowsW + row) * 4;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int32_t sum = __float2int_rn(__uint_as_float(u[i])) + (parts ? lds32(sums0 + at + i * kTileRowsW * 4) : 0);
                            if constexpr (SPLIT) sts32(data0 + at + i * kTileRowsW * 4, sum);  // (over the stages, which are all read)
                            else u[i] = __float_as_uint((float)sum);
                        }
                    }
                    if constexpr (!SPLIT) {
                        float v[16];
                        const uint64_t sw = both(scale), b = both(bias);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t s[4];
                            lds128(scales + 16 * i, s);
#pragma unroll
                            for (int j = 0; j < 4; j += 2) {
                                const float u0 = __uint_as_float(u[4 * i + j]), u1 = __uint_as_float(u[4 * i + j + 1]), a0 = __uint_as_float(s[j]), a1 = __uint_as_float(s[j + 1]);
                                if constexpr (decltype(channel_first)::value) {
                                    const float2 z = unpack2(fma2(mul2(pack2(u0, u1), sw), pack2(a0, a1), b));
                                    v[4 * i + j] = z.x, v[4 * i + j + 1] = z.y;
                                } else {
                                    v[4 * i + j] = scaled_sum(u0, a0, scale, bias), v[4 * i + j + 1] = scaled_sum(u1, a1, scale, bias);
                                }
                            }
                        }
                        store_tokens<ACT, T>(p, v, x, c0, nn, patch, lane);
                    }
                }
            };
            if (SPLIT || __all_sync(0xffffffffu, fabsf(scale) <= 1.0f)) columns(std::true_type());
            else columns(std::false_type());
            fence_before();
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) arrive_cluster(free0 + 8 * acc);
                else bar_arrive(aempty + 8 * acc);
            }
        }
    }
    if constexpr (SPLIT) {
        __syncwarp();
        cluster_sync();
        if (first < tiles && !abort_flag && warp >= kI8EpiWarp0) {
            // each warp of the cluster finishes the 32 rows of W of a quarter for four tokens at a time
            const int w = warp - kI8EpiWarp0, units = 4 * ((x.rows + 3) / 4);
            for (int u = w + kI8EpiWarps * rank; u < units; u += kI8EpiWarps * p.splits) {
                const int c0 = u & ~3, row = 32 * (u & 3) + lane, nn = x.n0 + row;
                const int64_t of = (int64_t)x.e * p.N + nn;
                const float scale = nn < p.N ? p.w_scales[of] : 0.0f, bias = p.bias && nn < p.N ? p.bias[of] : 0.0f;
                int32_t v[8][4];
                float z[4];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < p.splits) {
                        const uint32_t at = in_cta(data0 + (c0 * kTileRowsW + row) * 4, r);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v[r][i]) : "r"(at + i * kTileRowsW * 4) : "memory");
                    }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    int32_t sum = v[0][i];
#pragma unroll
                    for (int r = 1; r < 8; ++r)
                        if (r < p.splits) sum += v[r][i];
                    z[i] = scaled_sum((float)sum, c0 + i < x.rows ? p.a_scales[x.row0 + c0 + i] : 0.0f, scale, bias);
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
        for (int64_t i = blockIdx.x * (int64_t)kI8Threads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kI8Threads) {
            const int64_t r = i / wide;
            ((T *)p.Y)[(r < head ? r : r - head + tail) * p.ldy + (i - r * wide)] = to_out<T>(0.0f);
        }
    }
    fence_before();
    __syncwarp();
    if constexpr (MODE != TILE_ONE) cluster_sync();  // nothing of this CTA is read or signalled any more
    else __syncthreads();
    if (warp == kI8TileWarp) {
        fence_after();
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int ACT, typename T, int MODE, bool LONG>
cudaError_t launch_mode(const I8Params &p, int grid, size_t smem, cudaStream_t s) {
    static SmemLimit limit;
    cudaError_t e = raise_smem_limit(limit, (const void *)i8_gemm_kernel<ACT, T, MODE, LONG>, kI8SmemLimit);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = kI8Threads;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = MODE == TILE_SPLIT ? p.splits : 2;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = MODE == TILE_ONE ? 1 : 2;
    e = cudaLaunchKernelEx(&cfg, i8_gemm_kernel<ACT, T, MODE, LONG>, p);
    return e != cudaSuccess ? e : cudaGetLastError();
}
template <int ACT, typename T, bool LONG>
cudaError_t launch_act(const I8Params &p, int grid, size_t smem, cudaStream_t s) {
    if (p.mode == TILE_SPLIT) return launch_mode<ACT, T, TILE_SPLIT, LONG>(p, grid, smem, s);
    if (p.mode == TILE_PAIR) return launch_mode<ACT, T, TILE_PAIR, LONG>(p, grid, smem, s);
    return launch_mode<ACT, T, TILE_ONE, LONG>(p, grid, smem, s);
}

}  // namespace

template <typename T, bool LONG>
cudaError_t launch_i8(const I8Params &p, int32_t act, int grid, size_t smem, cudaStream_t s) {
    if (act == ILW_ACT_GELU) return launch_act<ILW_ACT_GELU, T, LONG>(p, grid, smem, s);
    if (act == ILW_ACT_SILU_GATE) return launch_act<ILW_ACT_SILU_GATE, T, LONG>(p, grid, smem, s);
    return launch_act<ILW_ACT_NONE, T, LONG>(p, grid, smem, s);
}

}  // namespace ilw
