// i8_kernels.h -- internal launch interface of the int8 operators with float scales.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "ilwdetr.h"

namespace ilw {

struct I8QuantParams {
    const void *X;
    int32_t form;           // ILW_FP32, ILW_FP16, ILW_BF16
    int64_t ldx, x_rows;    // elements between rows; rows of X
    const int32_t *gather;  // source row of each row, or NULL (row i is row i)
    int64_t rows;
    int32_t K;
    int8_t *codes;
    int64_t ldc;
    float *scales;
    int *status;
};
cudaError_t launch_i8_quantize(const I8QuantParams &p, cudaStream_t s);

struct I8DequantParams {
    const int8_t *codes;
    int64_t ldc;
    const float *scales;
    int64_t rows;
    int32_t K;
    void *Y;
    int32_t form;  // ILW_FP32, ILW_FP16, ILW_BF16
    int64_t ldy;
};
cudaError_t launch_i8_dequantize(const I8DequantParams &p, cudaStream_t s);

struct I8GemmProblem {
    const int8_t *a_codes, *w_codes;
    const float *a_scales, *w_scales;  // [M], [experts, N]
    int64_t a_ldc, w_ldc, w_codes_stride;
    const float *bias;                 // [experts, N] or NULL
    int64_t M;
    int32_t N, K, experts;
    const int32_t *offsets;            // [experts + 1] device, or NULL (one group of all rows)
    int32_t act;                       // ILW_ACT_*
    int32_t form;                      // ILW_FP32, ILW_FP16, ILW_BF16
    void *Y;
    int64_t ldy;
};
constexpr int kI8MaxExperts = 1024;
constexpr int kI8MaxK = (1 << 17) - 1;  // |sum| <= 2^14 K < 2^31
// What launch_i8_gemm would take on `sms` SMs (0: as many as the current device has): form 0 (a CTA a tile), 1 (several), 2 (a pair) or 3
// (launch_i8_few), CTAs that share a tile's K, most tokens a tile.
void i8_gemm_form(const I8GemmProblem &g, int32_t sms, int32_t (&form)[3]);
cudaError_t launch_i8_few(const I8GemmProblem &g, cudaStream_t s);
cudaError_t launch_i8_gemm(const I8GemmProblem &g, cudaStream_t s);

}  // namespace ilw
