// Division of x < 2^31 by a number fixed for a launch: (mulhi(x, mul) + x) >> shift.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace tr {

struct Divisor {
    uint32_t mul, shift;
};

__device__ __forceinline__ uint32_t divide(uint32_t x, const Divisor& d) { return (__umulhi(d.mul, x) + x) >> d.shift; }

inline Divisor divisor(uint32_t d)
{
    Divisor v;
    v.shift = 0;
    while ((1ull << v.shift) < d) ++v.shift;
    v.mul = (uint32_t)(((1ull << 32) * ((1ull << v.shift) - d)) / d + 1);
    return v;
}

}  // namespace tr
