// mx.cu -- rows to microscaled 4-bit floating point (MXFP4) and back.
//
// A block is 32 consecutive values of a row: one E8M0 scale byte b, standing for 2^(b - 127), and 32 E2M1
// codes (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign).  The scale of a block is the power of two that puts its largest
// magnitude into [4, 8) (OCP Microscaling Formats 1.0, section 6.3); values are divided by it, exactly, and
// rounded to the nearest code, ties to the even one, saturating at 6.  A block of zeros has scale byte 0, a
// block with a value that is not finite the NaN byte 255.
//
// Both kernels move bytes and little else.  A warp takes 256 values of a row: each lane 8, four lanes a block.
#include <algorithm>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "mx_kernels.h"

namespace ilw {
namespace {

constexpr int kWarps = 8;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(int8_t v) { return (float)v; }

// 8 consecutive values from x (n of them exist, the rest are 0); VEC: x is aligned to 8 values (16 bytes for 4-byte ones)
template <typename T, bool VEC>
__device__ __forceinline__ void load8(const T *x, int n, float (&v)[8]) {
    if (VEC && n >= 8) {
        union {
            uint32_t w[2 * sizeof(T)];
            T t[8];
        } u;
        if constexpr (sizeof(T) == 1) {
            *(uint2 *)u.w = *(const uint2 *)x;
        } else {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4 *)u.w)[i] = ((const uint4 *)x)[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = to_f(u.t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? to_f(x[i]) : 0.0f;
    }
}

// Two values to two codes of a byte, `lo` in the low nibble: nearest, ties to even, saturating.
__device__ __forceinline__ uint32_t e2m1x2(float lo, float hi) {
    uint16_t r;
    asm("{\n .reg .b8 t;\n cvt.rn.satfinite.e2m1x2.f32 t, %2, %1;\n cvt.u16.u8 %0, t;\n}\n" : "=h"(r) : "f"(lo), "f"(hi));
    return r;
}
// 2^(b - 127) for a scale byte (b = 0 is a subnormal, 255 NaN)
__device__ __forceinline__ float scale_value(uint32_t b) {
    return __uint_as_float(b == 255 ? 0x7fc00000u : b == 0 ? 0x00400000u : b << 23);
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) mx_quantize_kernel(const MxQuantParams p) {
    grid_wait();
    const int lane = threadIdx.x & 31;
    const int32_t segs = (p.K + 255) / 256;
    const int32_t blocks = (p.K + 31) / 32, pad = (blocks + 15) & ~15;
    for (int64_t r = blockIdx.y; r < p.rows; r += gridDim.y) {
        int64_t src = r;
        if (p.gather) {
            src = p.gather[r];
            if (src < 0 || src >= p.x_rows) {
                if (src != -1 && p.status && lane == 0) atomicExch(p.status, kStatusBadIndex);
                src = -1;
            }
        }
        for (int32_t seg = blockIdx.x * kWarps + (threadIdx.x >> 5); seg < segs; seg += gridDim.x * kWarps) {
            const int32_t k = seg * 256 + lane * 8;
            float v[8];
            load8<T, VEC>((const T *)p.X + (src < 0 ? 0 : src) * p.ldx + k, src < 0 ? 0 : p.K - k, v);
            uint32_t m = 0;  // magnitudes as bits: in order, infinities and NaN on top
#pragma unroll
            for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            // floor(log2 amax) - 2 + 127 is the biased exponent less 2, at least 0 (a subnormal's too)
            const uint32_t e = m >> 23;
            const uint32_t b = e == 255 ? 255u : e < 2 ? 0u : e - 2;
            uint32_t w = 0;
            if (e != 255) {
                const float inv = __uint_as_float((254 - b) << 23);  // 2^(127 - b), b <= 252
#pragma unroll
                for (int i = 0; i < 4; ++i) w |= e2m1x2(v[2 * i] * inv, v[2 * i + 1] * inv) << (8 * i);
            }
            if (k < blocks * 32) *(uint32_t *)(p.codes + r * p.ldc + (k >> 1)) = w;
            const int32_t blk = k >> 5;
            if ((lane & 3) == 0 && blk < pad) p.scales[r * p.lds + blk] = (uint8_t)b;
            if (seg == segs - 1 && seg * 8 + 8 + lane < pad) p.scales[r * p.lds + seg * 8 + 8 + lane] = 0;
        }
    }
}

// the two values of a byte of codes
__device__ __forceinline__ float2 from_e2m1x2(uint32_t byte) {
    uint32_t h;
    asm("{\n .reg .b8 t, z;\n mov.b32 {t, z, z, z}, %1;\n cvt.rn.f16x2.e2m1x2 %0, t;\n}\n" : "=r"(h) : "r"(byte));
    return __half22float2(*reinterpret_cast<__half2 *>(&h));
}

template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T, bool VEC>
__global__ void __launch_bounds__(32 * kWarps) mx_dequantize_kernel(const MxDequantParams p) {
    grid_wait();
    const int lane = threadIdx.x & 31;
    const int32_t segs = (p.K + 255) / 256;
    for (int64_t r = blockIdx.y; r < p.rows; r += gridDim.y) {
        for (int32_t seg = blockIdx.x * kWarps + (threadIdx.x >> 5); seg < segs; seg += gridDim.x * kWarps) {
            const int32_t k = seg * 256 + lane * 8, n = p.K - k;
            if (n <= 0) continue;
            const uint32_t w = *(const uint32_t *)(p.codes + r * p.ldc + (k >> 1));
            const float s = scale_value(p.scales[r * p.lds + (k >> 5)]);
            T *y = (T *)p.Y + r * p.ldy + k;
            union {
                uint4 q[sizeof(T) / 2];
                T t[8];
            } u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = from_e2m1x2((w >> (8 * i)) & 255);
                u.t[2 * i] = from_f<T>(f.x * s);
                u.t[2 * i + 1] = from_f<T>(f.y * s);
            }
            if (VEC && n >= 8) {
#pragma unroll
                for (int i = 0; i < (int)sizeof(T) / 2; ++i) ((uint4 *)y)[i] = u.q[i];
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n) y[i] = u.t[i];
            }
        }
    }
}

dim3 row_grid(int64_t rows, int32_t K) {
    const int32_t segs = (K + 255) / 256;
    return dim3((unsigned)((segs + kWarps - 1) / kWarps), (unsigned)std::min<int64_t>(rows, 65535));
}

template <typename T>
cudaError_t quantize(const MxQuantParams &p, cudaStream_t s) {
    const bool vec = (uintptr_t)p.X % 16 == 0 && p.ldx * (int64_t)sizeof(T) % 16 == 0;
    if (vec) return launch_after(mx_quantize_kernel<T, true>, row_grid(p.rows, p.K), 32 * kWarps, 0, s, p);
    return launch_after(mx_quantize_kernel<T, false>, row_grid(p.rows, p.K), 32 * kWarps, 0, s, p);
}
template <typename T>
cudaError_t dequantize(const MxDequantParams &p, cudaStream_t s) {
    const bool vec = (uintptr_t)p.Y % 16 == 0 && p.ldy * (int64_t)sizeof(T) % 16 == 0;
    if (vec) return launch_after(mx_dequantize_kernel<T, true>, row_grid(p.rows, p.K), 32 * kWarps, 0, s, p);
    return launch_after(mx_dequantize_kernel<T, false>, row_grid(p.rows, p.K), 32 * kWarps, 0, s, p);
}

}  // namespace

cudaError_t launch_mx_quantize(const MxQuantParams &q, cudaStream_t s) {
    if (q.rows == 0) return cudaSuccess;
    MxQuantParams p = q;
    p.status = status_word_ptr();
    if (p.form == ILW_FP32) return quantize<float>(p, s);
    if (p.form == ILW_FP16) return quantize<__half>(p, s);
    if (p.form == ILW_BF16) return quantize<__nv_bfloat16>(p, s);
    return quantize<int8_t>(p, s);
}

cudaError_t launch_mx_dequantize(const MxDequantParams &p, cudaStream_t s) {
    if (p.rows == 0) return cudaSuccess;
    if (p.form == ILW_FP32) return dequantize<float>(p, s);
    if (p.form == ILW_FP16) return dequantize<__half>(p, s);
    return dequantize<__nv_bfloat16>(p, s);
}

}  // namespace ilw
