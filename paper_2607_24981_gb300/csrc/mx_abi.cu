// mx_abi.cu -- the C-ABI entry points of the microscaled 4-bit and mixture-of-experts operators: argument
// checks and dispatch.
#include <climits>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "mx_kernels.h"

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
// One of the two arrays of an MXFP4 matrix: `bytes` of each row are used.
int mx_array(const char *what, const char *name, const void *p, int64_t ld, int64_t bytes) {
    if (!p || !aligned(p, 16)) return fail(ILW_ERR_INVALID_ARG, "%s: %s NULL or not 16-byte aligned", what, name);
    if (ld < bytes || ld % 16 || ld >= (int64_t)1 << 40)
        return fail(ILW_ERR_INVALID_ARG, "%s: %s rows of %lld bytes: a multiple of 16, at least %lld", what, name, (long long)ld, (long long)bytes);
    return ILW_OK;
}
int64_t code_bytes(int32_t K) { return ((int64_t)K + 31) / 32 * 16; }
int64_t scale_bytes(int32_t K) { return ((int64_t)K + 31) / 32; }

#define ILW_TRY(x) \
    if (const int rc_ = (x)) return rc_

// Checks a product's arguments and puts them into g; those of an empty one (M or N 0) need no tensors.
int gemm_problem(const ilw_mx_gemm_t *p, ilw::MxGemmProblem &g) {
    if (!p || p->struct_size != sizeof(ilw_mx_gemm_t)) return fail(ILW_ERR_INVALID_ARG, "mx_gemm: struct_size");
    if (p->act < ILW_ACT_NONE || p->act > ILW_ACT_SILU_GATE) return fail(ILW_ERR_INVALID_ARG, "mx_gemm: act=%d", p->act);
    if (!form_size(p->y_form)) return fail(ILW_ERR_INVALID_ARG, "mx_gemm: y_form=%d", p->y_form);
    if (p->M < 0 || p->N < 0 || p->K < 1 || p->experts < 1 || (!p->offsets && p->experts != 1))
        return fail(ILW_ERR_INVALID_ARG, "mx_gemm: bad sizes M=%lld N=%d K=%d experts=%d", (long long)p->M, p->N, p->K, p->experts);
    const bool gate = p->act == ILW_ACT_SILU_GATE;
    if (gate && p->N % 2) return fail(ILW_ERR_INVALID_ARG, "mx_gemm: a gated product's N=%d must be even", p->N);
    if (p->M > INT32_MAX - 1024 || p->N > (1 << 24) || p->K > (1 << 24) || p->experts > ilw::kMxMaxExperts)
        return fail(ILW_ERR_UNSUPPORTED, "mx_gemm: M < 2^31 - 1024, N and K <= 2^24, experts <= %d", ilw::kMxMaxExperts);
    // (the tiles a call can come to, counted in 32 bits by the kernel)
    if ((p->M / 16 + p->experts + 1) * ((p->N + 127) / 128) > INT32_MAX) return fail(ILW_ERR_UNSUPPORTED, "mx_gemm: M x N too large for one call");
    g = {};
    g.M = p->M, g.N = p->N;
    if (p->M == 0 || p->N == 0) return ILW_OK;
    ILW_TRY(mx_array("mx_gemm", "a_codes", p->a_codes, p->a_ldc, code_bytes(p->K)));
    ILW_TRY(mx_array("mx_gemm", "a_scales", p->a_scales, p->a_lds, scale_bytes(p->K)));
    ILW_TRY(mx_array("mx_gemm", "w_codes", p->w_codes, p->w_ldc, code_bytes(p->K)));
    ILW_TRY(mx_array("mx_gemm", "w_scales", p->w_scales, p->w_lds, scale_bytes(p->K)));
    const bool one = !p->offsets || p->experts == 1;
    if (!one && (p->w_codes_stride % 16 || p->w_scales_stride % 16 || p->w_codes_stride < 16 || p->w_scales_stride < 16 ||
                 p->w_codes_stride >= (int64_t)1 << 40 || p->w_scales_stride >= (int64_t)1 << 40))
        return fail(ILW_ERR_INVALID_ARG, "mx_gemm: strides between experts are positive multiples of 16 bytes");
    if (!aligned(p->bias, 4) || !aligned(p->offsets, 4)) return fail(ILW_ERR_INVALID_ARG, "mx_gemm: bias or offsets misaligned");
    if (!p->Y || !aligned(p->Y, form_size(p->y_form)) || p->ldy < (gate ? p->N / 2 : p->N))
        return fail(ILW_ERR_INVALID_ARG, "mx_gemm: Y NULL, misaligned or of short rows");
    g.a_codes = p->a_codes, g.a_scales = p->a_scales, g.w_codes = p->w_codes, g.w_scales = p->w_scales;
    g.a_ldc = p->a_ldc, g.a_lds = p->a_lds, g.w_ldc = p->w_ldc, g.w_lds = p->w_lds;
    // (one matrix: any stride that a tensor map takes)
    g.w_codes_stride = one ? p->w_ldc : p->w_codes_stride, g.w_scales_stride = one ? p->w_lds : p->w_scales_stride;
    g.bias = p->bias, g.K = p->K, g.experts = p->experts, g.offsets = p->offsets;
    g.act = p->act, g.form = p->y_form, g.Y = p->Y, g.ldy = p->ldy;
    return ILW_OK;
}

}  // namespace

extern "C" {

int ilwdetr_mx_quantize(const void *X, int32_t x_form, int64_t ldx, int64_t x_rows, const int32_t *gather, int64_t rows,
                        int32_t K, uint8_t *codes, int64_t ldc, uint8_t *scales, int64_t lds, ilw_stream_t stream) {
    const int size = x_form == 8 ? 1 : form_size(x_form);
    if (!size) return fail(ILW_ERR_INVALID_ARG, "mx_quantize: x_form=%d", x_form);
    if (K < 1 || K > INT32_MAX - 1024 || rows < 0 || rows > INT32_MAX || x_rows < 0 || ldx < K || (!gather && rows > x_rows) || x_rows > INT32_MAX)
        return fail(ILW_ERR_INVALID_ARG, "mx_quantize: bad sizes rows=%lld x_rows=%lld K=%d", (long long)rows, (long long)x_rows, K);
    if (rows == 0) return ILW_OK;
    if ((!X && x_rows > 0) || !aligned(X, size) || !aligned(gather, 4))
        return fail(ILW_ERR_INVALID_ARG, "mx_quantize: X NULL, or X or gather misaligned");
    ILW_TRY(mx_array("mx_quantize", "codes", codes, ldc, code_bytes(K)));
    ILW_TRY(mx_array("mx_quantize", "scales", scales, lds, (scale_bytes(K) + 15) / 16 * 16));
    if (ilw::validate_only()) return ILW_OK;
    const ilw::MxQuantParams p{X, x_form, ldx, x_rows, gather, rows, K, codes, ldc, scales, lds, nullptr};
    return done(ilw::launch_mx_quantize(p, (cudaStream_t)stream), "mx_quantize");
}

int ilwdetr_mx_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t lds, int64_t rows, int32_t K,
                          void *Y, int32_t y_form, int64_t ldy, ilw_stream_t stream) {
    if (!form_size(y_form)) return fail(ILW_ERR_INVALID_ARG, "mx_dequantize: y_form=%d", y_form);
    if (K < 1 || K > INT32_MAX - 1024 || rows < 0 || rows > INT32_MAX || ldy < K) return fail(ILW_ERR_INVALID_ARG, "mx_dequantize: bad sizes rows=%lld K=%d", (long long)rows, K);
    if (rows == 0) return ILW_OK;
    if (!Y || !aligned(Y, form_size(y_form))) return fail(ILW_ERR_INVALID_ARG, "mx_dequantize: Y NULL or misaligned");
    ILW_TRY(mx_array("mx_dequantize", "codes", codes, ldc, code_bytes(K)));
    ILW_TRY(mx_array("mx_dequantize", "scales", scales, lds, scale_bytes(K)));
    if (ilw::validate_only()) return ILW_OK;
    const ilw::MxDequantParams p{codes, ldc, scales, lds, rows, K, Y, y_form, ldy};
    return done(ilw::launch_mx_dequantize(p, (cudaStream_t)stream), "mx_dequantize");
}

int ilwdetr_mx_gemm(const ilw_mx_gemm_t *p, ilw_stream_t stream) {
    ilw::MxGemmProblem g;
    ILW_TRY(gemm_problem(p, g));
    if (g.M == 0 || g.N == 0 || ilw::validate_only()) return ILW_OK;
    return done(ilw::launch_mx_gemm(g, (cudaStream_t)stream), "mx_gemm");
}

int ilwdetr_debug_mx_form(const ilw_mx_gemm_t *p, int32_t sms, int32_t *form) {
    ilw::MxGemmProblem g;
    ILW_TRY(gemm_problem(p, g));
    if (!form || sms < 0 || g.M == 0 || g.N == 0) return fail(ILW_ERR_INVALID_ARG, "debug_mx_form: NULL result, negative sms or empty product");
    int32_t f[3];
    if (!ilw::mx_gemm_form(g, sms, f)) return fail(ILW_ERR_UNSUPPORTED, "debug_mx_form: no form");
    for (int i = 0; i < 3; ++i) form[i] = f[i];
    return ILW_OK;
}

size_t ilwdetr_moe_route_workspace_bytes(int32_t T, int32_t E) {
    if (T < 0 || E < 1) return 0;
    return ilw::moe_route_workspace(T, E);
}

int ilwdetr_moe_route(const void *logits, int32_t form, int64_t ld, int32_t T, int32_t E, int32_t k, int32_t renormalize,
                      int32_t *expert, float *weight, int32_t *offsets, int32_t *source, int32_t *slot, void *workspace,
                      size_t workspace_bytes, ilw_stream_t stream) {
    if (!form_size(form)) return fail(ILW_ERR_INVALID_ARG, "moe_route: form=%d", form);
    if (T < 0 || E < 1 || k < 1 || k > E || ld < E) return fail(ILW_ERR_INVALID_ARG, "moe_route: bad sizes T=%d E=%d k=%d", T, E, k);
    if (E > ilw::kRouteMaxExperts || k > ilw::kRouteMaxTop || (int64_t)T * k > INT32_MAX)
        return fail(ILW_ERR_UNSUPPORTED, "moe_route: E <= %d, k <= %d, T k < 2^31", ilw::kRouteMaxExperts, ilw::kRouteMaxTop);
    if (T > 0 && (!logits || !expert || !weight || !source || !slot))
        return fail(ILW_ERR_INVALID_ARG, "moe_route: NULL tensor");
    if (!offsets || !aligned(logits, form_size(form)) || !aligned(expert, 4) || !aligned(weight, 4) || !aligned(offsets, 4) ||
        !aligned(source, 4) || !aligned(slot, 4))
        return fail(ILW_ERR_INVALID_ARG, "moe_route: offsets NULL or a tensor misaligned");
    const size_t need = ilw::moe_route_workspace(T, E);
    if (need && (!workspace || !aligned(workspace, 4) || workspace_bytes < need))
        return fail(ILW_ERR_INVALID_ARG, "moe_route: workspace NULL, misaligned or smaller than %zu bytes", need);
    if (ilw::validate_only()) return ILW_OK;
    const ilw::MoeRouteParams p{logits, form, ld, T, E, k, renormalize, expert, weight, offsets, source, slot, (int32_t *)workspace};
    return done(ilw::launch_moe_route(p, (cudaStream_t)stream), "moe_route");
}

int ilwdetr_moe_combine(const void *Y, int32_t form, int64_t ldy, int64_t rows, const int32_t *slot, const float *weight,
                        int32_t T, int32_t k, int32_t N, const void *res, int64_t ldr, void *out, int64_t ldo,
                        ilw_stream_t stream) {
    const int size = form_size(form);
    if (!size) return fail(ILW_ERR_INVALID_ARG, "moe_combine: form=%d", form);
    if (T < 0 || k < 1 || N < 0 || rows < 0 || ldy < N || ldo < N || (res && ldr < N))
        return fail(ILW_ERR_INVALID_ARG, "moe_combine: bad sizes T=%d k=%d N=%d", T, k, N);
    if (T == 0 || N == 0) return ILW_OK;
    if ((!Y && rows > 0) || !slot || !weight || !out) return fail(ILW_ERR_INVALID_ARG, "moe_combine: NULL tensor");
    if (!aligned(Y, size) || !aligned(res, size) || !aligned(out, size) || !aligned(slot, 4) || !aligned(weight, 4))
        return fail(ILW_ERR_INVALID_ARG, "moe_combine: misaligned");
    if (ilw::validate_only()) return ILW_OK;
    const ilw::MoeCombineParams p{Y, form, ldy, rows, slot, weight, T, k, N, res, ldr, out, ldo, nullptr};
    return done(ilw::launch_moe_combine(p, (cudaStream_t)stream), "moe_combine");
}

}  // extern "C"
