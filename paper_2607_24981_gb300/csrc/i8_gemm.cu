// i8_gemm.cu -- host side of the int8 products: tile sizes, the form of the kernel (i8_gemm.cuh), tensor maps, and which products
// go to the kernel for few tokens (i8_few.cu).
#include <algorithm>
#include <climits>
#include <cmath>
#include <cstring>

#include "divisor.cuh"
#include "i8_gemm.cuh"

namespace ilw {
void gemm_debug_wait(int32_t *skip, long long *cycles);
extern template cudaError_t launch_i8<float, false>(const I8Params &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_i8<__half, false>(const I8Params &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_i8<__nv_bfloat16, false>(const I8Params &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_i8<float, true>(const I8Params &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_i8<__half, true>(const I8Params &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_i8<__nv_bfloat16, true>(const I8Params &, int32_t, int, size_t, cudaStream_t);
namespace {

// A tensor map over rows of codes, [z, rows, cols] bytes (z 0: no such dimension), in swizzled boxes of box_rows x 128.
bool code_map(CUtensorMap *m, const void *base, int64_t cols, int64_t rows, int64_t ld, int64_t z, int64_t zstride, int box_rows) {
    EncodeTiledTc fn = encode_tc();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)(z > 0 ? z : 1)};
    cuuint64_t strides[2] = {(cuuint64_t)ld, (cuuint64_t)zstride};
    cuuint32_t box[3] = {128, (cuuint32_t)box_rows, 1}, es[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, z > 0 ? 3 : 2, const_cast<void *>(base), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether sums are taken out of the accumulators on the way (i8_gemm.cuh).
bool long_sums(const I8GemmProblem &g) { return g.K > (g.form == ILW_FP32 ? kI8ExactK : kI8ShortK); }

// What a product will take on `sms` SMs, by a model in ns of what the forms were measured to: the forms differ by factors where sizes do,
// and by a few percent where the model errs.
//   few tokens (i8_few.cu)  2200 + the weights once for every eight tokens of an expert at 4.4 TB/s, of two tokens or fewer at 5.8, and no less
//                           than 1000 + 2 K (K <= 1024) for each turn of the warps (4096 x 4096: one token 3.7 us, 8 6.0, 16 9.4; 32 rows of 64 experts, 4096 x
//                           2048, 34 and by tiles 36, 128 rows 82 and 71)
//   tiles                   3700, a pair's 4300, and for each round of tiles the longer of its stages of 64 of K, 185 + n / 2 each of n tokens (a
//                           pair's 150 + 0.4 n), and its epilogue, 250 + 14.5 n (GELU 21 n; of one CTA a quarter more); for all of them no less
//                           than the weights at 6 TB/s, of one CTA 5.6 (8192 cubed in pairs of 192, 160 and 128 tokens 549, 626 and 677 us, one CTA of 128 and
//                           64 860 and 1315; 2000 cubed in pairs of 192 and 128 22.8 and 19.1, one CTA of 128 22.1; 12800 x 1536 x 384 22.2, 22.0
//                           and 25.4; 300 x 1001 x 1030 in pairs of 128 and 32 9.3 and 7.6)
//   K shared by CTAs        2800 + 10 n for the join (32 x 4096 x 4096 by one CTA 15.3 us, two 12.5, four 9.6)
struct Choice {
    int mode;  // TILE_*, or -1 for the few
    int32_t nt, splits;
    double ns;
};
Choice choose(const I8GemmProblem &g, int64_t sms) {
    const double M = (double)g.M, weights = (double)g.N * g.K;
    // experts that have rows, about, and their rows
    const double met = g.offsets ? std::max(1.0, g.experts * (1.0 - std::exp(-M / g.experts))) : 1.0, mean = M / met;
    const double units = g.offsets ? std::max(met, M / 8 + met / 2) : std::ceil(M / 8);
    const double turns = std::ceil(units * ((g.N + 3) / 4) / (16.0 * sms));
    const bool countable = (M / 8 + g.experts + 1) * ((g.N + 3) / 4) < INT32_MAX;  // (pieces of work of the few)
    Choice best = {-1, 8, 1, countable ? 2200 + std::max(units * weights / (mean > 2 ? 4400 : 5800), (1000 + 2 * std::min(g.K, 1024)) * turns) : INFINITY};
    const int32_t nkb = (g.K + 127) / 128, top = (int32_t)std::min<double>(kI8MaxTok, std::ceil((g.offsets ? 4 * mean : M) / 32) * 32);
    const double epilogue = g.act == ILW_ACT_GELU ? 21 : 14.5;
    const int32_t widest = long_sums(g) ? kI8LongTok : kI8MaxTok;
    for (const bool pair : {true, false})
        for (int32_t n = pair ? 32 : 16; n <= std::min(top, pair ? widest : kI8MaxTokOne); n += pair ? 32 : 16) {
            const int64_t wtiles = (g.N + (pair ? 2 : 1) * kTileRowsW - 1) / ((pair ? 2 : 1) * kTileRowsW);
            const double about = g.offsets ? std::min(M, std::max(met, M / n + met / 2)) : std::ceil(M / n);
            const double tokens = std::min<double>(n, std::ceil(mean / 16) * 16), stage = pair ? 150 + 0.4 * tokens : 185 + 0.5 * tokens;
            const double rounds = std::ceil(about * wtiles / (pair ? sms / 2 : sms));
            const double ns = (pair ? 4300 : 3700) + std::max(rounds * std::max(2 * nkb * stage, (pair ? 1.0 : 1.25) * (250 + epilogue * tokens)), met * weights / (pair ? 6000 : 5600));
            if (ns <= best.ns) best = {pair ? TILE_PAIR : TILE_ONE, n, 1, ns};
            if (pair) continue;
            // clusters of all tiles at once, which have to fit side by side: 16 of 8 CTAs do not
            const int64_t most = (g.offsets ? std::min<int64_t>(g.M, g.M / n + g.experts) : (g.M + n - 1) / n) * wtiles;
            for (int32_t c = 2; c <= 8; c *= 2) {
                const int64_t room = c == 8 ? sms / 2 : c == 4 ? sms * 7 / 8 : sms;
                if (c > nkb || c * most > room) continue;
                const double split = 3700 + 2 * ((nkb + c - 1) / c) * stage + 2800 + 10 * tokens;
                if (split < best.ns) best = {TILE_SPLIT, n, c, split};
            }
        }
    return best;
}

// The parameters of a form, with the number of tiles at most and the shared memory of a CTA.
bool lay_out(const I8GemmProblem &g, const Choice &c, I8Params &p, int64_t &tiles, int &smem) {
    p.M = g.M, p.N = g.N, p.E = g.experts;
    p.nkb = (g.K + 127) / 128;
    p.mode = c.mode, p.nt = c.nt, p.splits = c.splits;
    const int64_t out = g.act == ILW_ACT_SILU_GATE ? g.N / 2 : g.N;
    p.wide = g.form != ILW_FP32 && out % 8 == 0 && (uintptr_t)g.Y % 16 == 0 && g.ldy % 8 == 0;
    const int rows_w = p.mode == TILE_PAIR ? 2 * kTileRowsW : kTileRowsW;
    p.wtiles = (g.N + rows_w - 1) / rows_w;
    const Divisor by = divisor(p.wtiles);
    p.wdiv_m = by.m, p.wdiv_s = by.s;
    tiles = (g.offsets ? std::min<int64_t>(g.M, g.M / p.nt + g.experts) : (g.M + p.nt - 1) / p.nt) * p.wtiles;
    const int32_t tokens = p.mode == TILE_PAIR ? p.nt / 2 : p.nt;  // whose codes a CTA loads
    p.stage_bytes = kTileRowsW * 128 + tokens * 128;
    p.wide_bytes = tokens * 128;
    p.part = kI8ExactK / 64;
    p.sums_bytes = long_sums(g) ? kTileRowsW * p.nt * 4 : 0;
    const int fixed = 1024 + p.sums_bytes + (g.experts + 1) * (int)sizeof(TileExpert) + g.experts * 4 + (p.wide ? kI8EpiWarps * kI8Patch : 0);
    auto bytes = [&] { return fixed + p.stages * p.stage_bytes + p.wides * p.wide_bytes; };
    // two stages of widened codes a set where tensor memory and shared memory have room, then as many stages of codes as fit
    for (p.wides = 2 * p.nt + 32 * kI8MaxWide <= 512 ? kI8MaxWide : kI8Sets;; p.wides = kI8Sets) {
        for (p.stages = kI8MaxStages; p.stages >= kI8MinStages && bytes() > kI8SmemLimit; p.stages -= 2) {
        }
        if (p.wides == kI8Sets || p.stages >= 4) break;
    }
    smem = bytes();
    return p.stages >= kI8MinStages && tiles <= INT32_MAX - 4096;
}

}  // namespace

void i8_gemm_form(const I8GemmProblem &g, int32_t sms, int32_t (&form)[3]) {
    const Choice c = choose(g, sms ? sms : sm_count());
    form[0] = c.mode < 0 ? 3 : c.mode, form[1] = c.splits, form[2] = c.nt;
}

cudaError_t launch_i8_gemm(const I8GemmProblem &g, cudaStream_t s) {
    if (g.M == 0 || g.N == 0) return cudaSuccess;
    const int64_t sms = sm_count();
    Choice c = choose(g, sms);
    if (c.mode < 0) return launch_i8_few(g, s);
    I8Params p;
    memset(&p, 0, sizeof(p));
    p.offsets = g.offsets;
    p.bias = g.bias;
    p.Y = g.Y;
    p.ldy = g.ldy;
    p.status = status_word_ptr();
    gemm_debug_wait(&p.dbg_skip, &p.wait_cycles);
    int64_t tiles;
    int smem;
    if (!lay_out(g, c, p, tiles, smem)) return cudaErrorInvalidValue;
    p.w_scales = g.w_scales, p.a_scales = g.a_scales;
    if (!code_map(&p.wc, g.w_codes, g.K, g.N, g.w_ldc, g.experts, g.w_codes_stride, kTileRowsW) || !code_map(&p.ac[0], g.a_codes, g.K, g.M, g.a_ldc, 0, 0, 16))
        return cudaErrorInvalidValue;
    for (int i = 1; i < 4; ++i)
        if (!code_map(&p.ac[i], g.a_codes, g.K, g.M, g.a_ldc, 0, 0, 16 << i)) return cudaErrorInvalidValue;
    int grid = (int)std::min<int64_t>(tiles, sms);
    if (p.mode == TILE_SPLIT) grid = (int)tiles * p.splits;
    if (p.mode == TILE_PAIR) grid = 2 * (int)std::min<int64_t>(tiles, sms / 2);
    auto launch = [&](auto plain, auto with_long_sums) { return (long_sums(g) ? with_long_sums : plain)(p, g.act, grid, (size_t)smem, s); };
    if (g.form == ILW_FP32) return launch(launch_i8<float, false>, launch_i8<float, true>);
    if (g.form == ILW_FP16) return launch(launch_i8<__half, false>, launch_i8<__half, true>);
    return launch(launch_i8<__nv_bfloat16, false>, launch_i8<__nv_bfloat16, true>);
}

}  // namespace ilw
