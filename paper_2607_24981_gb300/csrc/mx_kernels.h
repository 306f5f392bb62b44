// mx_kernels.h -- internal launch interface of the microscaled 4-bit (MXFP4) operators and of the
// mixture-of-experts routing around them.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "divisor.cuh"
#include "ilwdetr.h"

namespace ilw {

// Element forms of a float (or int8) tensor: the C-ABI's codes.
struct MxQuantParams {
    const void *X;
    int32_t form;           // 8 (int8), ILW_FP32, ILW_FP16, ILW_BF16
    int64_t ldx, x_rows;    // elements between rows; rows of X
    const int32_t *gather;  // source row of each row, or NULL (row i is row i)
    int64_t rows;
    int32_t K;
    uint8_t *codes;
    int64_t ldc;
    uint8_t *scales;
    int64_t lds;
    int *status;
};
cudaError_t launch_mx_quantize(const MxQuantParams &p, cudaStream_t s);

struct MxDequantParams {
    const uint8_t *codes;
    int64_t ldc;
    const uint8_t *scales;
    int64_t lds, rows;
    int32_t K;
    void *Y;
    int32_t form;  // ILW_FP32, ILW_FP16, ILW_BF16
    int64_t ldy;
};
cudaError_t launch_mx_dequantize(const MxDequantParams &p, cudaStream_t s);

struct MxGemmProblem {
    const uint8_t *a_codes, *a_scales, *w_codes, *w_scales;
    int64_t a_ldc, a_lds, w_ldc, w_lds, w_codes_stride, w_scales_stride;
    const float *bias;         // [experts, N] or NULL
    int64_t M;
    int32_t N, K, experts;
    const int32_t *offsets;    // [experts + 1] device, or NULL (one group of all rows)
    int32_t act;               // ILW_ACT_*
    int32_t form;              // ILW_FP32, ILW_FP16, ILW_BF16
    void *Y;
    int64_t ldy;
};
constexpr int kMxMaxExperts = 1024;
// What launch_mx_gemm would take on `sms` SMs (0: as many as the current device has): form 0 (a CTA a tile), 1 (several) or 2 (a
// pair), CTAs that share a tile's K, most tokens a tile.
bool mx_gemm_form(const MxGemmProblem &g, int32_t sms, int32_t (&form)[3]);
cudaError_t launch_mx_gemm(const MxGemmProblem &p, cudaStream_t s);

struct MoeRouteParams {
    const void *logits;
    int32_t form;
    int64_t ld;
    int32_t T, E, k, renormalize;
    int32_t *expert;   // [T, k]
    float *weight;     // [T, k]
    int32_t *offsets;  // [E + 1]
    int32_t *source;   // [T k]
    int32_t *slot;     // [T, k]
    int32_t *counts;   // workspace [chunks, E]
};
// How experts are taken and weighted beside plain softmax (ilw_moe_scores_t).
struct RouteScores {
    int32_t score;             // ILW_SCORE_*
    const float *bias;         // [E] or NULL
    int32_t groups, top_groups, group_best, group_size;
    Divisor per_group;         // by group_size
    float scale;
};
struct MoeScoredParams : MoeRouteParams {
    RouteScores scores;
};
constexpr int kRouteMaxExperts = ILW_MOE_MAX_EXPERTS, kRouteMaxTop = ILW_MOE_MAX_TOP;
size_t moe_route_workspace(int32_t T, int32_t E);
cudaError_t launch_moe_route(const MoeRouteParams &p, cudaStream_t s);
cudaError_t launch_moe_route_scored(const MoeScoredParams &p, cudaStream_t s);  // (fills in what follows from groups and E)
// For the latter: whether one CTA takes all, and the order from chunks' counts (chunks of 256 or 512 tokens).
bool moe_route_in_one(int32_t T, int32_t E);
cudaError_t launch_moe_place(const MoeRouteParams &p, int32_t chunk, cudaStream_t s);

struct MoeCombineParams {
    const void *Y;
    int32_t form;
    int64_t ldy, rows;
    const int32_t *slot;
    const float *weight;
    int32_t T, k, N;
    const void *res;  // or NULL
    int64_t ldr;
    void *out;
    int64_t ldo;
    int *status;
};
cudaError_t launch_moe_combine(const MoeCombineParams &p, cudaStream_t s);

}  // namespace ilw
