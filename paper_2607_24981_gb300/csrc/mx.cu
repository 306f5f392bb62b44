// mx.cu -- rows to microscaled 4-bit floating point (MXFP4) and back.
//
// A block is 32 consecutive values of a row: one E8M0 scale byte b, standing for 2^(b - 127), and 32 E2M1
// codes (0, .5, 1, 1.5, 2, 3, 4, 6 and a sign).  The scale of a block is the power of two that puts its largest
// magnitude into [4, 8) (OCP Microscaling Formats 1.0, section 6.3); values are divided by it, exactly, and
// rounded to the nearest code, ties to the even one, saturating at 6.  A block of zeros has scale byte 0, a
// block with a value that is not finite the NaN byte 255.
//
// Both move bytes and little else, so what counts is how many are in flight and how few instructions go with them.  Rows on
// 16-byte boundaries: sixteen values a thread and step to quantise (two lanes a block; magnitudes of 16-bit values are
// compared two at a time), eight a thread back, several steps in flight.  Other rows: a warp takes 256 values of a row, one
// after the other in memory, and hands them over through shared memory, so that its accesses stay whole lines
// (eight values a lane in a row of its own would touch every line eight times).  Measured, first form and second: 65536 x 1536 bf16
// to codes 40.1 us (6.4 TB/s) and 78, back 38.3 us (6.7 TB/s) and 77; 16384 x 4096 fp32 to codes 44.2 us (6.9 TB/s) and 52, back 62 and
// 57; int8 65536 x 1536 to codes 66 us (2.3 TB/s) and 74.
#include <algorithm>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "divisor.cuh"
#include "ilw_kernels.h"
#include "ilwdetr.h"
#include "mx_kernels.h"

namespace ilw {
namespace {

constexpr int kThreads = 256;
constexpr int kSteps = 4;  // groups of eight values of a thread in flight, on the way back

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(int8_t v) { return (float)v; }

// 8 values of T (16 or 32 bytes; 8 for int8) as loaded
template <typename T> struct alignas(sizeof(T) == 1 ? 8 : 16) Eight {
    T t[8];
};

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

// Scale byte of a block whose largest magnitude has the bits m (infinities and NaN are above all others), and the factor
// 2^(127 - b) by which its values become codes: floor(log2 amax) - 2 + 127 is the biased exponent less 2, at least 0 (a
// subnormal's too).
__device__ __forceinline__ uint32_t scale_byte(uint32_t m, float &inv) {
    const uint32_t e = m >> 23, b = e == 255 ? 255u : e < 2 ? 0u : e - 2;
    inv = __uint_as_float((254 - min(b, 253u)) << 23);
    return b;
}
__device__ __forceinline__ uint32_t codes8(const float (&v)[8], float inv) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) w |= e2m1x2(v[2 * i] * inv, v[2 * i + 1] * inv) << (8 * i);
    return w;
}
// Scale byte and codes of this lane's 8 values (four lanes a block, all of them here).
__device__ __forceinline__ uint32_t encode8(const float (&v)[8], uint32_t &b) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    float inv;
    b = scale_byte(m, inv);
    return b == 255 ? 0 : codes8(v, inv);
}

// The largest magnitude of 8 values, as the bits of a float.
__device__ __forceinline__ uint32_t magnitude8(const Eight<float> &x) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x.t[i]) & 0x7fffffffu);
    return m;
}
template <typename T>
__device__ __forceinline__ uint32_t magnitude8_16bit(const Eight<T> &x) {
    const uint32_t *w = (const uint32_t *)&x;
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
    return max(m & 0xffffu, m >> 16);
}
__device__ __forceinline__ uint32_t magnitude8(const Eight<__nv_bfloat16> &x) { return magnitude8_16bit(x) << 16; }
__device__ __forceinline__ uint32_t magnitude8(const Eight<__half> &x) {
    return __float_as_uint(__half2float(__ushort_as_half((unsigned short)magnitude8_16bit(x)))) & 0x7fffffffu;
}
__device__ __forceinline__ uint32_t magnitude8(const Eight<int8_t> &x) {
    int m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, abs((int)x.t[i]));
    return __float_as_uint((float)m);
}

// The row of X that row r takes; -1: a row of zeros.
__device__ __forceinline__ int64_t source_row(const MxQuantParams &p, int64_t r) {
    if (!p.gather) return r;
    const int32_t s = p.gather[r];
    if (s >= 0 && s < p.x_rows) return s;
    if (s != -1 && p.status) atomicExch(p.status, kStatusBadIndex);
    return -1;
}

// Rows of X on 16-byte boundaries, K a multiple of 8.  Step i of the grid: row i / per, values 16 (i % per) .. + 15, two lanes a
// block.
template <typename T>
__global__ void __launch_bounds__(kThreads) mx_quantize_kernel(const MxQuantParams p, Divisor per, uint32_t r0, uint32_t total) {
    constexpr int kSteps = 2;
    grid_wait();
    const uint32_t base = blockIdx.x * (kThreads * kSteps) + threadIdx.x;
    Eight<T> x[kSteps][2];
    uint32_t row[kSteps], k[kSteps];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        const uint32_t i = base + j * kThreads;
        row[j] = per.div(i);
        k[j] = (i - row[j] * per.d) * 16;
#pragma unroll
        for (int u = 0; u < 8; ++u) x[j][0].t[u] = x[j][1].t[u] = T(0);
        if (i < total && k[j] < (uint32_t)p.K) {
            const int64_t src = source_row(p, (int64_t)r0 + row[j]);
            if (src >= 0) {
                const Eight<T> *at = (const Eight<T> *)((const T *)p.X + src * p.ldx + k[j]);
                x[j][0] = at[0];
                if (k[j] + 8 < (uint32_t)p.K) x[j][1] = at[1];
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        uint32_t m = max(magnitude8(x[j][0]), magnitude8(x[j][1]));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        if (base + j * kThreads >= total) continue;
        float inv;
        const uint32_t b = scale_byte(m, inv);
        uint2 w = make_uint2(0, 0);
        if (b != 255) {
            float v[8], u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = to_f(x[j][0].t[i]), u[i] = to_f(x[j][1].t[i]);
            w = make_uint2(codes8(v, inv), codes8(u, inv));
        }
        const int64_t r = (int64_t)r0 + row[j];
        const uint32_t blk = k[j] >> 5, half = threadIdx.x & 1;
        *(uint2 *)(p.codes + r * p.ldc + (k[j] >> 1)) = w;
        if (half == 0) p.scales[r * p.lds + blk] = (uint8_t)b;
        if (blk + 1 == per.d / 2)  // the row's last block: its lanes fill up the scale bytes
            for (uint32_t z = blk + 1 + half; z <= (blk | 15); z += 2) p.scales[r * p.lds + z] = 0;
    }
}

// Any rows: a warp takes 256 values of a row at a time.
template <typename T>
__global__ void __launch_bounds__(kThreads) mx_quantize_any_kernel(const MxQuantParams p, Divisor segs, uint32_t r0, uint32_t total) {
    __shared__ __align__(16) float stage[kThreads / 32][256];
    grid_wait();
    const int lane = threadIdx.x & 31;
    float *mine = stage[threadIdx.x >> 5];
    const uint32_t u = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (u >= total) return;
    const uint32_t row = segs.div(u), k0 = (u - row * segs.d) * 256;
    const int64_t r = (int64_t)r0 + row, src = source_row(p, r);
    const uint32_t K = (uint32_t)p.K, blocks = (K + 31) / 32;
    const T *x = (const T *)p.X + src * p.ldx + k0;
#pragma unroll
    for (int i = 0; i < 8; ++i) mine[32 * i + lane] = src >= 0 && k0 + 32 * i + lane < K ? to_f(x[32 * i + lane]) : 0.0f;
    __syncwarp();
    float v[8];
    uint32_t b;
    *(float4 *)v = *(const float4 *)(mine + 8 * lane);
    *(float4 *)(v + 4) = *(const float4 *)(mine + 8 * lane + 4);
    const uint32_t w = encode8(v, b), k = k0 + 8 * lane;
    if (k < blocks * 32) *(uint32_t *)(p.codes + r * p.ldc + (k >> 1)) = w;
    const uint32_t blk = k >> 5;
    if ((k & 31) == 0 && blk < blocks) p.scales[r * p.lds + blk] = (uint8_t)b;
    if (k0 + 256 >= K && lane < 15 && blocks + lane <= ((blocks - 1) | 15)) p.scales[r * p.lds + blocks + lane] = 0;  // (up to a multiple of 16)
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

template <typename T>
__global__ void __launch_bounds__(kThreads) mx_dequantize_kernel(const MxDequantParams p, Divisor per, uint32_t r0, uint32_t total) {
    grid_wait();
    const uint32_t base = blockIdx.x * (kThreads * kSteps) + threadIdx.x;
    uint32_t w[kSteps], b[kSteps], row[kSteps], k[kSteps];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        const uint32_t i = base + j * kThreads;
        row[j] = per.div(i);
        k[j] = (i - row[j] * per.d) * 8;
        w[j] = b[j] = 0;
        if (i < total) {
            const int64_t r = (int64_t)r0 + row[j];
            w[j] = *(const uint32_t *)(p.codes + r * p.ldc + (k[j] >> 1));
            b[j] = p.scales[r * p.lds + (k[j] >> 5)];
        }
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        if (base + j * kThreads >= total) continue;
        const float s = scale_value(b[j]);
        Eight<T> y;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float2 f = from_e2m1x2((w[j] >> (8 * u)) & 255);
            y.t[2 * u] = from_f<T>(f.x * s);
            y.t[2 * u + 1] = from_f<T>(f.y * s);
        }
        *(Eight<T> *)((T *)p.Y + ((int64_t)r0 + row[j]) * p.ldy + k[j]) = y;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) mx_dequantize_any_kernel(const MxDequantParams p, Divisor segs, uint32_t r0, uint32_t total) {
    __shared__ __align__(16) float stage[kThreads / 32][256];
    grid_wait();
    const int lane = threadIdx.x & 31;
    float *mine = stage[threadIdx.x >> 5];
    const uint32_t u = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    if (u >= total) return;
    const uint32_t row = segs.div(u), k0 = (u - row * segs.d) * 256, k = k0 + 8 * lane;
    const int64_t r = (int64_t)r0 + row;
    const uint32_t K = (uint32_t)p.K;
    if (k < K) {
        const uint32_t w = *(const uint32_t *)(p.codes + r * p.ldc + (k >> 1));
        const float s = scale_value(p.scales[r * p.lds + (k >> 5)]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float2 f = from_e2m1x2((w >> (16 * i)) & 255), g = from_e2m1x2((w >> (16 * i + 8)) & 255);
            ((float4 *)(mine + 8 * lane))[i] = make_float4(f.x * s, f.y * s, g.x * s, g.y * s);
        }
    }
    __syncwarp();
    T *y = (T *)p.Y + r * p.ldy + k0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (k0 + 32 * i + lane < K) y[32 * i + lane] = from_f<T>(mine[32 * i + lane]);
}

// Launches `kernel` over `rows` rows of `per` steps each, `step` of them a CTA, as often as 2^30 steps at a time take (a step is a
// thread's or a warp's, so 32 bits hold a step's number but not always a thread's).
template <typename P>
cudaError_t over_rows(void (*kernel)(const P, Divisor, uint32_t, uint32_t), const P &p, int64_t rows, uint32_t per, uint32_t step, cudaStream_t s) {
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / per);
    for (int64_t r0 = 0; r0 < rows; r0 += most) {
        const uint32_t total = (uint32_t)(std::min(most, rows - r0) * per);
        const cudaError_t e = launch_after(kernel, (total + step - 1) / step, kThreads, 0, s, p, divisor(per), (uint32_t)r0, total);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename T>
cudaError_t quantize(const MxQuantParams &p, cudaStream_t s) {
    if ((uintptr_t)p.X % alignof(Eight<T>) == 0 && p.ldx * (int64_t)sizeof(T) % alignof(Eight<T>) == 0 && p.K % 8 == 0)
        return over_rows(mx_quantize_kernel<T>, p, p.rows, (uint32_t)(p.K + 31) / 32 * 2, kThreads * 2, s);
    return over_rows(mx_quantize_any_kernel<T>, p, p.rows, (uint32_t)(p.K + 255) / 256, kThreads / 32, s);
}
template <typename T>
cudaError_t dequantize(const MxDequantParams &p, cudaStream_t s) {
    if ((uintptr_t)p.Y % 16 == 0 && p.ldy * (int64_t)sizeof(T) % 16 == 0 && p.K % 8 == 0)
        return over_rows(mx_dequantize_kernel<T>, p, p.rows, p.K / 8, kThreads * kSteps, s);
    return over_rows(mx_dequantize_any_kernel<T>, p, p.rows, (uint32_t)(p.K + 255) / 256, kThreads / 32, s);
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
