// i8.cu -- rows to int8 codes with a float scale each, and back.
//
// Of a row x with largest magnitude m: scale s = m / 127 rounded to fp32, at least 2^-126 (0 for a row of zeros, NaN where a value is
// not finite), codes x / s rounded to the nearest whole number, ties to the even one.
//
// The codes are those of the exact quotient.  n = rint(x (1 / s)) is it, or its neighbour where x / s lies within 127 roundings of fp32
// of a half; d = x - n s is exact in fp32 (a multiple of the smaller of the units of x and s that is at most about s / 2), and rint(n + d (1 / s)),
// one fma, is the code unless x lies on a half: 2 x is a multiple of the unit u = 2^-23 2^e of s = m 2^e (1 <= m < 2) where it comes close to an odd
// multiple of s, so from the half it is u / 2 s = 2^-24 / m away at least, and 1 / s rounded moves d / s by at most 2^-26 m, which is less.  On
// a half it is right too if 1 / s is exact.  fp32 values may lie on halves of any other scale, 16-bit ones of scales with no more bits than theirs:
// there d is compared with s / 2 (65536 x 1536 bf16 that way 63 us, so 44.8).
//
// Bytes are what it moves.  A row is held in registers between its maximum and its codes, by 8 lanes, a warp, 128 or 512 threads; past 24576
// (512 x 6 pieces of 16 bytes) it is read twice.  Rows on 16-byte boundaries are loaded and stored 16 bytes at a time; others value by value, four
// consecutive ones a thread (whole lines, with the codes exchanged between lanes, were slower: 65536 x 1537 bf16 117 us, so 80).  16384 x 4096
// fp32: 47.8 us (7.0 TB/s), back 49.1 (6.8).  65536 x 1536 bf16: 44.8 us (6.75 TB/s), back 50.2 (6.0).
#include <algorithm>
#include <cstdint>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "divisor.cuh"
#include "float_act.cuh"
#include "i8_kernels.h"
#include "ilw_kernels.h"
#include "ilwdetr.h"

namespace ilw {
namespace {

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }

// V consecutive values of T: 16 bytes of them, or four.
template <typename T, int V> struct alignas(V * sizeof(T) == 16 ? 16 : 4) Unit {
    T t[V];
};

// Values 2 i and 2 i + 1 of a unit (16-bit ones by their common word).
template <int V> __device__ __forceinline__ float2 pair(const Unit<float, V> &x, int i) { return make_float2(x.t[2 * i], x.t[2 * i + 1]); }
template <int V> __device__ __forceinline__ float2 pair(const Unit<__half, V> &x, int i) { return __half22float2(((const __half2 *)&x)[i]); }
template <int V> __device__ __forceinline__ float2 pair(const Unit<__nv_bfloat16, V> &x, int i) {
    const uint32_t w = ((const uint32_t *)&x)[i];
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
// The largest magnitude of a unit as the bits of a T without a sign (infinities and NaN are above all others); of 16-bit ones that of each half of
// the words.
template <int V> __device__ __forceinline__ uint32_t magnitude(const Unit<float, V> &x, uint32_t m) {
#pragma unroll
    for (int i = 0; i < V; ++i) m = max(m, __float_as_uint(x.t[i]) & 0x7fffffffu);
    return m;
}
template <typename T, int V> __device__ __forceinline__ uint32_t magnitude(const Unit<T, V> &x, uint32_t m) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) m = __vmaxu2(m, ((const uint32_t *)&x)[i] & 0x7fff7fffu);
    return m;
}
__device__ __forceinline__ uint32_t of_halves(uint32_t m, float) { return m; }
template <typename T> __device__ __forceinline__ uint32_t of_halves(uint32_t m, T) { return max(m & 0xffffu, m >> 16); }
__device__ __forceinline__ float magnitude_value(uint32_t m, float) { return __uint_as_float(m); }
__device__ __forceinline__ float magnitude_value(uint32_t m, __half) { return __half2float(__ushort_as_half((unsigned short)m)); }
__device__ __forceinline__ float magnitude_value(uint32_t m, __nv_bfloat16) { return __uint_as_float(m << 16); }

constexpr float kMagic = 12582912.0f;  // 1.5 2^23: x + kMagic holds rint(x) in its low bits

// Whether a value of T can lie on a half of s without 1 / s being exact: x = (n + 1/2) s takes a scale of no more bits than T has.
__device__ __forceinline__ bool halves(float, float) { return true; }
__device__ __forceinline__ bool halves_of(float s, uint32_t past) {
    const uint32_t b = __float_as_uint(s);
    return (b & past) == 0 && (b & 0x7fffff) != 0;
}
__device__ __forceinline__ bool halves(float s, __half) { return halves_of(s, 0x1fff); }
__device__ __forceinline__ bool halves(float s, __nv_bfloat16) { return halves_of(s, 0xffff); }

template <int V> __device__ __forceinline__ void code_words(const float (&t)[V], uint32_t (&w)[V / 4]) {
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
        w[i] = __byte_perm(__byte_perm(__float_as_uint(t[4 * i]), __float_as_uint(t[4 * i + 1]), 0x0040),
                           __byte_perm(__float_as_uint(t[4 * i + 2]), __float_as_uint(t[4 * i + 3]), 0x0040), 0x5410);
}
// Codes of a unit, four to a word.
template <typename T, int V> __device__ __forceinline__ void encode(const Unit<T, V> &x, float s, float inv, uint32_t (&w)[V / 4]) {
    float t[V];
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float2 p = pair(x, i / 2);
        const uint64_t v = pack2(p.x, p.y), sum = fma2(v, both(inv), both(kMagic));
        const float2 c = unpack2(fma2(fma2(fma2(sum, both(-1.0f), both(kMagic)), both(s), v), both(inv), sum));
        t[i] = c.x, t[i + 1] = c.y;
    }
    code_words(t, w);
}
// The same where values may lie on a half.
template <typename T, int V> __device__ __forceinline__ void encode_halves(const Unit<T, V> &x, float s, float inv, uint32_t (&w)[V / 4]) {
    float t[V], worst = 0.0f;
#pragma unroll
    for (int i = 0; i < V; i += 2) {
        const float2 p = pair(x, i / 2);
        const uint64_t v = pack2(p.x, p.y), sum = fma2(v, both(inv), both(kMagic));
        const float2 c = unpack2(sum), r = unpack2(fma2(fma2(sum, both(-1.0f), both(kMagic)), both(s), v));
        t[i] = c.x, t[i + 1] = c.y;
        worst = fmaxf(worst, fmaxf(fabsf(r.x), fabsf(r.y)));
    }
    if (worst > 0.4999f * s) {  // near a half
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float v = to_f(x.t[i]), r = fmaf(kMagic - t[i], s, v), half = 0.5f * s;
            if (fabsf(r) > half || (fabsf(r) == half && (__float_as_uint(t[i]) & 1))) t[i] += copysignf(1.0f, r);
        }
    }
    code_words(t, w);
}

// CTAs an SM, so that loads of some rows overlap the arithmetic of others (65536 x 1536 bf16: with three 47.7 us, so 44.8, with five 45.3 and
// spills; 4096 x 8192 fp32: with six 52.3, so 27.5, with ten 32.5; 2000 x 20000 fp32: with one 69.5, so 44.5).
constexpr int quantize_ctas(int G, int held) { return G == 512 ? 3 : G == 128 ? (held > 4 ? 8 : 10) : held > 4 ? 4 : 5; }
// G threads a row (a warp, or the whole CTA); each holds up to kHeld units of it.
template <typename T, bool WIDE, int G, int kHeld>
__global__ void __launch_bounds__(G <= 32 ? 256 : G, quantize_ctas(G, kHeld)) i8_quantize_kernel(const I8QuantParams p) {
    constexpr int V = WIDE ? 16 / (int)sizeof(T) : 4;
    __shared__ uint32_t warp_max[G < 32 ? 1 : G / 32];
    grid_wait();
    const int q = threadIdx.x % G;
    const int64_t r = G <= 32 ? blockIdx.x * (int64_t)(256 / G) + threadIdx.x / G : blockIdx.x;
    if (r >= p.rows) return;  // (all threads of a row)
    int64_t src = r;
    if (p.gather) {
        src = p.gather[r];
        if (src < 0 || src >= p.x_rows) {
            if (src != -1 && q == 0 && p.status) atomicExch(p.status, kStatusBadIndex);
            src = -1;
        }
    }
    const T *x = (const T *)p.X + (src < 0 ? 0 : src) * p.ldx;
    const int32_t K = p.K, units = (K + V - 1) / V;
    auto load = [&](int32_t u) {
        Unit<T, V> y;
        if constexpr (WIDE) {
            if (u < units && src >= 0) return *(const Unit<T, V> *)(x + (int64_t)u * V);
#pragma unroll
            for (int i = 0; i < V; ++i) y.t[i] = T(0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) y.t[i] = src >= 0 && (int64_t)u * V + i < K ? x[(int64_t)u * V + i] : T(0.0f);
        }
        return y;
    };
    Unit<T, V> held[kHeld];
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < kHeld; ++j) held[j] = load(q + j * G);
#pragma unroll
    for (int j = 0; j < kHeld; ++j) m = magnitude(held[j], m);
    for (int32_t u = q + kHeld * G; u < units; u += G) m = magnitude(load(u), m);
    m = of_halves(m, T());
    m = __reduce_max_sync(G < 32 ? ((1u << G % 32) - 1) << (threadIdx.x & 31) / G * G : 0xffffffffu, m);
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) warp_max[threadIdx.x >> 5] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G / 32; ++i) m = max(m, warp_max[i]);
    }
    const float largest = magnitude_value(m, T());
    const bool fine = largest < __int_as_float(0x7f800000);
    const float s = largest > 0.0f ? fmaxf(__fdiv_rn(largest, 127.0f), 1.17549435e-38f) : 0.0f, inv = s > 0.0f && fine ? __frcp_rn(s) : 0.0f;
    if (q == 0) p.scales[r] = fine ? s : __int_as_float(0x7fc00000);
    int8_t *c = p.codes + r * p.ldc;
    auto put = [&](int32_t u, const uint32_t (&w)[V / 4]) {
        int8_t *at = c + (int64_t)u * V;
        if constexpr (V == 8) {
            *(uint2 *)at = make_uint2(w[0], w[1]);
        } else {
            if (WIDE || (int64_t)u * 4 + 4 <= K) *(uint32_t *)at = w[0];
            else
                for (int i = 0; u * 4 + i < K; ++i) at[i] = (int8_t)(w[0] >> (8 * i));
        }
    };
    uint32_t w[V / 4] = {};
    if (!fine) {
        for (int32_t u = q; u < units; u += G) put(u, w);
    } else if (sizeof(T) == 2 && halves(s, T())) {  // (rare: from memory again)
#pragma unroll 1
        for (int32_t u = q; u < units; u += G) {
            encode_halves(load(u), s, inv, w);
            put(u, w);
        }
    } else {
        auto code = [&](int32_t u, const Unit<T, V> &y) {
            if (u >= units) return;
            if constexpr (sizeof(T) == 2) encode(y, s, inv, w);
            else encode_halves(y, s, inv, w);
            put(u, w);
        };
#pragma unroll
        for (int j = 0; j < kHeld; ++j) code(q + j * G, held[j]);
        for (int32_t u = q + kHeld * G; u < units; u += G) code(u, load(u));
    }
}

// A code times s, from byte i of w ^ 0x80808080: 2^23 + 128 + code has that byte at its end (the conversion's own instruction has a quarter of
// the rate).
__device__ __forceinline__ float code_value(uint32_t w, int i, float s) { return (__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7650 + i)) - 8388736.0f) * s; }

// Values.  Rows of Y on 16-byte boundaries: 16 bytes of them a thread and step, several steps in flight.
constexpr int kSteps = 4;
template <typename T>
__global__ void __launch_bounds__(256) i8_dequantize_kernel(const I8DequantParams p, Divisor per, uint32_t r0, uint32_t total) {
    constexpr int V = 16 / sizeof(T);
    struct alignas(V) Codes {
        uint32_t w[V / 4];
    };
    grid_wait();
    const uint32_t base = blockIdx.x * (256 * kSteps) + threadIdx.x;
    Codes c[kSteps];
    float s[kSteps];
    uint32_t row[kSteps], k[kSteps];
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        const uint32_t i = base + j * 256;
        row[j] = per.div(i);
        k[j] = (i - row[j] * per.d) * V;
        if (i < total) {
            c[j] = *(const Codes *)(p.codes + ((int64_t)r0 + row[j]) * p.ldc + k[j]);
            s[j] = p.scales[(int64_t)r0 + row[j]];
        }
    }
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        if (base + j * 256 >= total) continue;
        struct alignas(16) Pack {
            T t[V];
        } o;
#pragma unroll
        for (int i = 0; i < V; ++i) o.t[i] = to_out<T>(code_value(c[j].w[i / 4] ^ 0x80808080u, i % 4, s[j]));
        *(Pack *)((T *)p.Y + ((int64_t)r0 + row[j]) * p.ldy + k[j]) = o;
    }
}
// Any rows: a warp takes 128 codes of a row, four a lane, and each lane stores what is a lane apart, so that accesses stay whole lines.
template <typename T>
__global__ void __launch_bounds__(256) i8_dequantize_any_kernel(const I8DequantParams p, Divisor segs, uint32_t r0, uint32_t total) {
    grid_wait();
    const int lane = threadIdx.x & 31;
    const uint32_t u = blockIdx.x * 8 + (threadIdx.x >> 5);
    if (u >= total) return;
    const uint32_t row = segs.div(u), k0 = (u - row * segs.d) * 128;
    const int64_t r = (int64_t)r0 + row;
    const int32_t left = p.K - (int32_t)k0;  // (codes of whole words are there up to the last one's)
    const int8_t *c = p.codes + r * p.ldc + k0;
    uint32_t w = 0;
    if (4 * lane + 4 <= left) w = *(const uint32_t *)(c + 4 * lane);
    else
        for (int i = 0; 4 * lane + i < left; ++i) w |= (uint32_t)(uint8_t)c[4 * lane + i] << (8 * i);
    const float s = p.scales[r];
    T *y = (T *)p.Y + r * p.ldy + k0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t v = __shfl_sync(0xffffffffu, w, 8 * i + (lane >> 2));
        if (32 * i + lane < left) y[32 * i + lane] = to_out<T>((float)(int8_t)(v >> (8 * (lane & 3))) * s);
    }
}

template <typename T, bool WIDE> cudaError_t quantize_rows(const I8QuantParams &p, cudaStream_t s) {
    const int64_t units = WIDE ? p.K / (16 / (int)sizeof(T)) : ((int64_t)p.K + 3) / 4;
    if constexpr (WIDE)
        if (units <= 8 * 2) return launch_after(i8_quantize_kernel<T, WIDE, 8, 2>, (unsigned)((p.rows + 31) / 32), 256, 0, s, p);
    const unsigned by_warp = (unsigned)((p.rows + 7) / 8);
    if (units <= 32 * 2) return launch_after(i8_quantize_kernel<T, WIDE, 32, 2>, by_warp, 256, 0, s, p);
    if (units <= 32 * 4) return launch_after(i8_quantize_kernel<T, WIDE, 32, 4>, by_warp, 256, 0, s, p);
    if (units <= 32 * 6) return launch_after(i8_quantize_kernel<T, WIDE, 32, 6>, by_warp, 256, 0, s, p);
    if (units <= 128 * 4) return launch_after(i8_quantize_kernel<T, WIDE, 128, 4>, (unsigned)p.rows, 128, 0, s, p);
    if (units <= 128 * 8) return launch_after(i8_quantize_kernel<T, WIDE, 128, 8>, (unsigned)p.rows, 128, 0, s, p);
    return launch_after(i8_quantize_kernel<T, WIDE, 512, 6>, (unsigned)p.rows, 512, 0, s, p);
}
template <typename T> cudaError_t quantize(const I8QuantParams &p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    if ((uintptr_t)p.X % 16 == 0 && p.ldx % V == 0 && p.K % V == 0) return quantize_rows<T, true>(p, s);
    return quantize_rows<T, false>(p, s);
}
// Launches `kernel` over rows of `per` steps each, `step` of them a CTA, as often as 2^30 steps at a time take.
cudaError_t over_rows(void (*kernel)(const I8DequantParams, Divisor, uint32_t, uint32_t), const I8DequantParams &p, uint32_t per, uint32_t step, cudaStream_t s) {
    const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 30) / per);
    for (int64_t r0 = 0; r0 < p.rows; r0 += most) {
        const uint32_t total = (uint32_t)(std::min(most, p.rows - r0) * per);
        const cudaError_t e = launch_after(kernel, (total + step - 1) / step, 256, 0, s, p, divisor(per), (uint32_t)r0, total);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}
template <typename T> cudaError_t dequantize(const I8DequantParams &p, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    if ((uintptr_t)p.Y % 16 == 0 && p.ldy % V == 0 && p.K % V == 0) return over_rows(i8_dequantize_kernel<T>, p, p.K / V, 256 * kSteps, s);
    return over_rows(i8_dequantize_any_kernel<T>, p, ((uint32_t)p.K + 127) / 128, 8, s);
}

}  // namespace

cudaError_t launch_i8_quantize(const I8QuantParams &q, cudaStream_t s) {
    if (q.rows == 0) return cudaSuccess;
    I8QuantParams p = q;
    p.status = status_word_ptr();
    if (p.form == ILW_FP32) return quantize<float>(p, s);
    if (p.form == ILW_FP16) return quantize<__half>(p, s);
    return quantize<__nv_bfloat16>(p, s);
}

cudaError_t launch_i8_dequantize(const I8DequantParams &p, cudaStream_t s) {
    if (p.rows == 0) return cudaSuccess;
    if (p.form == ILW_FP32) return dequantize<float>(p, s);
    if (p.form == ILW_FP16) return dequantize<__half>(p, s);
    return dequantize<__nv_bfloat16>(p, s);
}

}  // namespace ilw
