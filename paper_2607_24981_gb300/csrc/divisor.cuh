// divisor.cuh -- division of 32-bit numbers by a divisor that the host knows.
#pragma once
#include <cstdint>

namespace ilw {
namespace {

// n / d for n < 2^31 (round-up reciprocal of Granlund and Montgomery, 1994)
struct Divisor {
    uint32_t d, m, s;
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, m) + n) >> s; }
};
inline Divisor divisor(uint32_t d) {
    uint32_t s = 0;
    while (((uint64_t)1 << s) < d) ++s;
    return {d, (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - d)) / d + 1), s};
}

}  // namespace
}  // namespace ilw
