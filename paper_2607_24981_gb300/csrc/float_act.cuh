// float_act.cuh -- the floating-point ends of products: rounding to the result's type, and the activations (GELU, SiLU gates).
#pragma once
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

namespace ilw {
namespace {

template <typename T> __device__ __forceinline__ T to_out(float v);
template <> __device__ __forceinline__ float to_out<float>(float v) { return v; }
template <> __device__ __forceinline__ __half to_out<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 to_out<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

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
// sum sa sw + bias of a whole sum, with two roundings: sw first, unless it is above 1.  Then no step overflows, or falls below the normal numbers, where the result
// does not: |sum| >= 1, so sum sw lies between the normal sw and |sum| <= 2^31, and a sum sa that overflows does so before it grows.
__device__ __forceinline__ float scaled_sum(float sum, float sa, float sw, float bias) {
    const bool small = fabsf(sw) <= 1.0f;
    return fmaf(sum * (small ? sw : sa), small ? sa : sw, bias);
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

}  // namespace
}  // namespace ilw
