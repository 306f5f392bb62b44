// mx_gemm.cu -- host side of the MXFP4 products: tile sizes, the form of the kernel (mx_gemm.cuh), tensor maps.
#include <algorithm>
#include <climits>
#include <cstring>

#include "mx_gemm.cuh"

namespace ilw {
void gemm_debug_wait(int32_t *skip, long long *cycles);
extern template cudaError_t launch_mx<float>(const MxParams &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_mx<__half>(const MxParams &, int32_t, int, size_t, cudaStream_t);
extern template cudaError_t launch_mx<__nv_bfloat16>(const MxParams &, int32_t, int, size_t, cudaStream_t);
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

// The form that a product takes on `sms` SMs, in p: mode, tiles, stages, with the number of tiles at most and the shared memory of a CTA.
bool choose_form(const MxGemmProblem &g, int64_t sms, MxParams &p, int64_t &tiles, int &smem) {
    p.M = g.M;
    p.N = g.N;
    p.E = g.experts;
    p.nkb = (g.K + 255) / 256;
    p.nsb = (g.K + 511) / 512;

    const int64_t out = g.act == ILW_ACT_SILU_GATE ? g.N / 2 : g.N;
    p.wide = g.act != ILW_ACT_NONE && g.form != ILW_FP32 && out % 8 == 0 && (uintptr_t)g.Y % 16 == 0 && g.ldy % 8 == 0;
    const int fixed = 1024 + (g.experts + 1) * (int)sizeof(TileExpert) + g.experts * 4 + (p.wide ? kMxEpiWarps * kMxPatch : 0);
    auto bytes = [&] { return fixed + p.stages * p.stage_bytes + kMxScaleSets * p.raw_bytes + 2 * p.scale_bytes; };

    // Tokens a tile: as wide as the tokens (of an expert, twice the mean: with the mean alone more experts of unequal ones take two
    // tiles; 1000 rows of 32 experts, N 4096, K 1024: 18.8 to 20.1 us as they are dealt out, 21.3 to 22.1 with the mean; 4096
    // rows, K 2048, 34.7 to 36.8 and 34.3 to 38.6) fill, at most 224, and what leaves room for four stages.
    const int64_t per = g.offsets ? (2 * g.M + g.experts - 1) / g.experts : g.M;
    p.nt = (int32_t)std::min<int64_t>(kMxMaxTok, (std::min(per, g.M) + 15) / 16 * 16);
    if (p.nt > 32) p.nt = (p.nt + 31) / 32 * 32;
    // tiles of n tokens: at most, and (every other expert's last tile half full) about
    auto most = [&](int64_t n) { return g.offsets ? std::min<int64_t>(g.M, g.M / n + g.experts) : (g.M + n - 1) / n; };
    auto about = [&](int64_t n) { return g.offsets ? std::min<int64_t>(g.M, g.M / n + g.experts / 2 + 1) : (g.M + n - 1) / n; };
    for (;; p.nt = (p.nt - 1) / 32 * 32) {  // (a pair's: a multiple of 32)
        // Pairs start and end some 1.5 us later and then take a sixth less time a block of K, so they are for a K above 1024 and 20 blocks
        // or more a pair of SMs (one CTA a tile against pairs, in us: 12800 x 384 x 1536, 9 blocks, 9.7 and 12.2; 6400 x 2048 x
        // 1536, 18 blocks, 16.6 and 16.8; 12800 x 1536 x 1536, 27 blocks, 21.8 and 20.8; 8192 cubed 194 and 169), and for
        // tiles of 64 tokens or more, whose MMAs take longer than their rows of W
        const int64_t pair_tiles = most(p.nt) * ((g.N + 2 * kTileRowsW - 1) / (2 * kTileRowsW));
        p.mode = p.nt >= 64 && g.N > kTileRowsW && p.nkb > 4 && 2 * pair_tiles * p.nkb >= 20 * sms ? TILE_PAIR : TILE_ONE;
        const int rows_w = p.mode == TILE_PAIR ? 2 * kTileRowsW : kTileRowsW;
        p.wtiles = (g.N + rows_w - 1) / rows_w;
        if (p.mode == TILE_ONE) {
            // The width, from 64 tokens on, at which the CTA with the most tiles reads the fewest rows of W and tokens (at 224 tokens and so, in
            // us: 12800 x 384 x 1536, 128 tokens, 11.5 and 9.7; 6400 x 1536 x 384, 176, 11.5 and 10.4; 224 x 4096 x 4096, 64, 10.8
            // and 8.9; narrower still, 32 and 16 tokens, 12.3 and 15.6; 2048 rows of 16 experts, 768 x 1024, 7.2 and 6.6)
            int64_t least = INT64_MAX;
            for (int32_t top = p.nt, n = top; n >= std::min(top, 64); n -= 16) {
                const int64_t rows = (about(n) * p.wtiles + sms - 1) / sms * (n + kTileRowsW);
                if (rows < least) least = rows, p.nt = n;
            }
        }
        tiles = most(p.nt) * p.wtiles;
        const int32_t tokens = p.mode == TILE_PAIR ? p.nt / 2 : p.nt;  // whose codes a CTA loads
        p.stage_bytes = kTileRowsW * 128 + tokens * 128;
        p.raw_bytes = kTileRowsW * 16 + (p.nt + 31) / 32 * 512;
        p.scale_bytes = 4 * kMxAtom * (1 + (p.nt + 127) / 128);
        // as many stages as fit
        for (p.stages = kMxMaxStages; p.stages >= kMxMinStages && bytes() > kMxSmemLimit; --p.stages) {
        }
        if (p.stages >= kMxMinStages) break;
        if (p.nt <= 32) return false;  // (never)
    }
    smem = bytes();
    if (tiles > INT32_MAX) return false;
    // t / wtiles for t < 2^31 (round-up reciprocal of Granlund and Montgomery, 1994)
    while ((1ll << p.wdiv_s) < p.wtiles) ++p.wdiv_s;
    p.wdiv_m = (uint32_t)((((uint64_t)1 << 32) * ((1ull << p.wdiv_s) - p.wtiles)) / p.wtiles + 1);
    // Few tiles and a long K: 8, 4 or 2 CTAs to a tile, each with whole scale stages of K.  The cluster and its join cost what six
    // stages of 512 do, more with many tokens (one CTA and split, in us: one token, N 4096, K 4096, by 4, 7.1 and 7.0; K 16384,
    // 17.7 and 10.8; N 1024 by 8, 16.9 and 7.6; 224 tokens, N and K 4096, by 4, 10.8 and 12.0, which is why it is not split),
    // and the clusters have to fit side by side: 16 of 8 CTAs do not (N 2048, K 4096: 11.4 us, by 4 6.7).
    p.splits = 1;
    if (p.mode == TILE_ONE)
        for (int c = 8; c > 1 && p.splits == 1; c /= 2) {
            const int64_t room = c == 8 ? sms / 2 : c == 4 ? sms * 7 / 8 : sms;
            if (c <= p.nsb && c * tiles <= room && p.nsb - (p.nsb + c - 1) / c >= 6 + p.nt / 128) p.splits = c;
        }
    if (p.splits > 1) p.mode = TILE_SPLIT;
    return true;
}

}  // namespace

bool mx_gemm_form(const MxGemmProblem &g, int32_t sms, int32_t (&form)[3]) {
    MxParams p;
    memset(&p, 0, sizeof(p));
    int64_t tiles;
    int smem;
    if (!choose_form(g, sms ? sms : sm_count(), p, tiles, smem)) return false;
    form[0] = p.mode, form[1] = p.splits, form[2] = p.nt;
    return true;
}

cudaError_t launch_mx_gemm(const MxGemmProblem &g, cudaStream_t s) {
    if (g.M == 0 || g.N == 0) return cudaSuccess;
    MxParams p;
    memset(&p, 0, sizeof(p));
    p.offsets = g.offsets;
    p.bias = g.bias;
    p.Y = g.Y;
    p.ldy = g.ldy;
    p.status = status_word_ptr();
    gemm_debug_wait(&p.dbg_skip, &p.wait_cycles);
    const int64_t sms = sm_count();
    int64_t tiles;
    int smem;
    if (!choose_form(g, sms, p, tiles, smem)) return cudaErrorInvalidValue;

    p.nb = (g.K + 31) / 32;
    p.w_scales = g.w_scales, p.w_lds = g.w_lds, p.w_scales_stride = g.w_scales_stride;
    p.a_scales = g.a_scales, p.a_lds = g.a_lds;
    if (!code_map(&p.wc, g.w_codes, 16 * p.nb, g.N, g.w_ldc, g.experts, g.w_codes_stride, kTileRowsW) ||
        !code_map(&p.ac[0], g.a_codes, 16 * p.nb, g.M, g.a_ldc, 0, 0, 16))
        return cudaErrorInvalidValue;
    for (int i = 1; i < 4; ++i)
        if (!code_map(&p.ac[i], g.a_codes, 16 * p.nb, g.M, g.a_ldc, 0, 0, 16 << i)) return cudaErrorInvalidValue;
    int grid = (int)std::min<int64_t>(tiles, sms);
    if (p.mode == TILE_SPLIT) grid = (int)tiles * p.splits;
    if (p.mode == TILE_PAIR) grid = 2 * (int)std::min<int64_t>(tiles, sms / 2);
    if (g.form == ILW_FP32) return launch_mx<float>(p, g.act, grid, smem, s);
    if (g.form == ILW_FP16) return launch_mx<__half>(p, g.act, grid, smem, s);
    return launch_mx<__nv_bfloat16>(p, g.act, grid, smem, s);
}

}  // namespace ilw
