// i8_abi.cu -- the C-ABI entry points of the int8 operators with float scales: argument checks and dispatch.
#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "i8_kernels.h"
#include "ilw_kernels.h"
#include "ilwdetr.h"

namespace {

int fail(int code, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return ilw::report_error(code, buf);
}
int done(cudaError_t e, const char *what) {
    return e == cudaSuccess ? ILW_OK : fail(ILW_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
bool aligned(const void *p, size_t a) { return (uintptr_t)p % a == 0; }
int form_size(int32_t form) { return form == ILW_FP32 ? 4 : form == ILW_FP16 || form == ILW_BF16 ? 2 : 0; }
// An int8 matrix: codes in rows of K bytes on 16-byte boundaries, and scales.
int i8_matrix(const char *what, const char *name, const int8_t *codes, int64_t ld, const float *scales, int32_t K) {
    if (!codes || !aligned(codes, 16)) return fail(ILW_ERR_INVALID_ARG, "%s: codes of %s NULL or not 16-byte aligned", what, name);
    if (ld < K || ld % 16 || ld >= (int64_t)1 << 40)
        return fail(ILW_ERR_INVALID_ARG, "%s: rows of %s are %lld bytes apart: a multiple of 16, at least %d", what, name, (long long)ld, K);
    if (!scales || !aligned(scales, 4)) return fail(ILW_ERR_INVALID_ARG, "%s: scales of %s NULL or misaligned", what, name);
    return ILW_OK;
}

#define ILW_TRY(x) \
    if (const int rc_ = (x)) return rc_

// Checks a product's arguments and puts them into g; those of an empty one (M or N 0) need no tensors.
int gemm_problem(const ilw_i8_gemm_t *p, ilw::I8GemmProblem &g) {
    if (!p || p->struct_size != sizeof(ilw_i8_gemm_t)) return fail(ILW_ERR_INVALID_ARG, "i8_gemm: struct_size");
    if (p->act < ILW_ACT_NONE || p->act > ILW_ACT_SILU_GATE) return fail(ILW_ERR_INVALID_ARG, "i8_gemm: act=%d", p->act);
    if (!form_size(p->y_form)) return fail(ILW_ERR_INVALID_ARG, "i8_gemm: y_form=%d", p->y_form);
    if (p->M < 0 || p->N < 0 || p->K < 1 || p->experts < 1 || (!p->offsets && p->experts != 1))
        return fail(ILW_ERR_INVALID_ARG, "i8_gemm: bad sizes M=%lld N=%d K=%d experts=%d", (long long)p->M, p->N, p->K, p->experts);
    const bool gate = p->act == ILW_ACT_SILU_GATE;
    if (gate && p->N % 2) return fail(ILW_ERR_INVALID_ARG, "i8_gemm: a gated product's N=%d must be even", p->N);
    if (p->M > INT32_MAX - 1024 || p->N > (1 << 24) || p->K > ilw::kI8MaxK || p->experts > ilw::kI8MaxExperts)
        return fail(ILW_ERR_UNSUPPORTED, "i8_gemm: M < 2^31 - 1024, N <= 2^24, K < 2^17, experts <= %d", ilw::kI8MaxExperts);
    // (tiles are counted in 32 bits; products of this size take those of 32 tokens or more)
    if ((p->M / 32 + p->experts + 1) * (((int64_t)p->N + 127) / 128) > INT32_MAX - 4096) return fail(ILW_ERR_UNSUPPORTED, "i8_gemm: M x N too large for one call");
    g = {};
    g.M = p->M, g.N = p->N;
    if (p->M == 0 || p->N == 0) return ILW_OK;
    ILW_TRY(i8_matrix("i8_gemm", "A", p->a_codes, p->a_ldc, p->a_scales, p->K));
    ILW_TRY(i8_matrix("i8_gemm", "W", p->w_codes, p->w_ldc, p->w_scales, p->K));
    const bool one = !p->offsets || p->experts == 1;
    if (!one && (p->w_codes_stride % 16 || p->w_codes_stride < 16 || p->w_codes_stride >= (int64_t)1 << 40))
        return fail(ILW_ERR_INVALID_ARG, "i8_gemm: the stride between experts is a positive multiple of 16 bytes");
    if (!aligned(p->bias, 4) || !aligned(p->offsets, 4)) return fail(ILW_ERR_INVALID_ARG, "i8_gemm: bias or offsets misaligned");
    if (!p->Y || !aligned(p->Y, form_size(p->y_form)) || p->ldy < (gate ? p->N / 2 : p->N))
        return fail(ILW_ERR_INVALID_ARG, "i8_gemm: Y NULL, misaligned or of short rows");
    g.a_codes = p->a_codes, g.a_scales = p->a_scales, g.w_codes = p->w_codes, g.w_scales = p->w_scales;
    g.a_ldc = p->a_ldc, g.w_ldc = p->w_ldc;
    g.w_codes_stride = one ? p->w_ldc : p->w_codes_stride;  // (one matrix: any stride that a tensor map takes)
    g.bias = p->bias, g.K = p->K, g.experts = p->experts, g.offsets = p->offsets;
    g.act = p->act, g.form = p->y_form, g.Y = p->Y, g.ldy = p->ldy;
    return ILW_OK;
}

}  // namespace

extern "C" {

int ilwdetr_i8_quantize(const void *X, int32_t x_form, int64_t ldx, int64_t x_rows, const int32_t *gather, int64_t rows,
                        int32_t K, int8_t *codes, int64_t ldc, float *scales, ilw_stream_t stream) {
    const int size = form_size(x_form);
    if (!size) return fail(ILW_ERR_INVALID_ARG, "i8_quantize: x_form=%d", x_form);
    if (K < 1 || K > INT32_MAX - 8192 || rows < 0 || rows > INT32_MAX || x_rows < 0 || x_rows > INT32_MAX || ldx < K || (!gather && rows > x_rows))
        return fail(ILW_ERR_INVALID_ARG, "i8_quantize: bad sizes rows=%lld x_rows=%lld K=%d", (long long)rows, (long long)x_rows, K);
    if (rows == 0) return ILW_OK;
    if ((!X && x_rows > 0) || !aligned(X, size) || !aligned(gather, 4))
        return fail(ILW_ERR_INVALID_ARG, "i8_quantize: X NULL, or X or gather misaligned");
    ILW_TRY(i8_matrix("i8_quantize", "the result", codes, ldc, scales, K));
    if (ilw::validate_only()) return ILW_OK;
    const ilw::I8QuantParams p{X, x_form, ldx, x_rows, gather, rows, K, codes, ldc, scales, nullptr};
    return done(ilw::launch_i8_quantize(p, (cudaStream_t)stream), "i8_quantize");
}

int ilwdetr_i8_dequantize(const int8_t *codes, int64_t ldc, const float *scales, int64_t rows, int32_t K, void *Y,
                          int32_t y_form, int64_t ldy, ilw_stream_t stream) {
    if (!form_size(y_form)) return fail(ILW_ERR_INVALID_ARG, "i8_dequantize: y_form=%d", y_form);
    if (K < 1 || K > INT32_MAX - 8192 || rows < 0 || rows > INT32_MAX || ldy < K)
        return fail(ILW_ERR_INVALID_ARG, "i8_dequantize: bad sizes rows=%lld K=%d", (long long)rows, K);
    if (rows == 0) return ILW_OK;
    if (!Y || !aligned(Y, form_size(y_form))) return fail(ILW_ERR_INVALID_ARG, "i8_dequantize: Y NULL or misaligned");
    ILW_TRY(i8_matrix("i8_dequantize", "the matrix", codes, ldc, scales, K));
    if (ilw::validate_only()) return ILW_OK;
    const ilw::I8DequantParams p{codes, ldc, scales, rows, K, Y, y_form, ldy};
    return done(ilw::launch_i8_dequantize(p, (cudaStream_t)stream), "i8_dequantize");
}

int ilwdetr_i8_gemm(const ilw_i8_gemm_t *p, ilw_stream_t stream) {
    ilw::I8GemmProblem g;
    ILW_TRY(gemm_problem(p, g));
    if (g.M == 0 || g.N == 0 || ilw::validate_only()) return ILW_OK;
    return done(ilw::launch_i8_gemm(g, (cudaStream_t)stream), "i8_gemm");
}

int ilwdetr_debug_i8_form(const ilw_i8_gemm_t *p, int32_t sms, int32_t *form) {
    ilw::I8GemmProblem g;
    ILW_TRY(gemm_problem(p, g));
    if (!form || sms < 0 || g.M == 0 || g.N == 0) return fail(ILW_ERR_INVALID_ARG, "debug_i8_form: NULL result, negative sms or empty product");
    int32_t f[3];
    ilw::i8_gemm_form(g, sms, f);
    for (int i = 0; i < 3; ++i) form[i] = f[i];
    return ILW_OK;
}

}  // extern "C"
