// Rotary angles, for the kernels that turn queries and keys (gfx950).
#pragma once

#include <hip/hip_runtime.h>

namespace bf1 {

// p * f radians without its whole turns: the nearest fp32 number of half turns, in
// [-1, 1], and the radians left (below 2^-23).
struct Turn {
    float half_turns, rest;
};
__device__ __forceinline__ Turn turn_of(double p, double f) {
    constexpr double INV = 0x1.45f306dc9c883p-3, INV_LOW = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
    const double a = p * f, a_low = fma(p, f, -a);
    const double t = a * INV, t_low = fma(a, INV, -t) + fma(a, INV_LOW, a_low * INV);
    const double x = 2. * ((t - rint(t)) + t_low);
    const float h = (float)x;
    return {h, (float)((x - (double)h) * 3.141592653589793)};
}

}  // namespace bf1
