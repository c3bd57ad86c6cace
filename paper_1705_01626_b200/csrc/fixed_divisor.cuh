#pragma once

#include <cstdint>
#include <cuda_runtime.h>

namespace cdma {

// Quotient of a 32-bit number and a fixed divisor by a high product (Granlund and Montgomery, "Division by
// invariant integers using multiplication", PLDI 1994).
struct FixedDivisor {
    uint32_t divisor, multiplier, shift1, shift2;
};
inline FixedDivisor make_divisor(uint32_t d) {
    if (d == 0) d = 1;
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    FixedDivisor f;
    f.divisor = d;
    f.multiplier = static_cast<uint32_t>((((1ull << l) - d) << 32) / d + 1);
    f.shift1 = l < 1 ? l : 1;
    f.shift2 = l < 1 ? 0 : l - 1;
    return f;
}
__device__ __forceinline__ uint32_t divide(uint32_t n, const FixedDivisor& f) {
    const uint32_t t = __umulhi(f.multiplier, n);
    return (t + ((n - t) >> f.shift1)) >> f.shift2;
}

}  // namespace cdma
