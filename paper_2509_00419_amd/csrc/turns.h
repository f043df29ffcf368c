// Angles of positions, the arithmetic that host and kernels share.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>

namespace lvlm {

// position times frequency (radians) in turns, less the whole ones: half a turn either way, and what the first word's rounding hid.  A
// 31-bit number times a 24-bit one does not fit the 53 bits of a product, nor does 1 / (2 pi): both keep what they lose in a second
// word, and the whole turns go before the words meet.  What is left is off by its rounding to fp32, 2^-25 of a turn at most, whatever the
// position (one word each: 2.3 times that beyond position 2^30).  No contraction: it would put into the first word what the second holds.
__host__ __device__ __forceinline__ float part_of_turn(int position, float frequency) {
#pragma clang fp contract(off)
    constexpr double kPerTurn = 0x1.45f306dc9c883p-3, kPerTurnRest = -0x1.6b01ec5417056p-57;    // 1 / (2 pi)
    const double x = (double)position * (double)frequency, x_rest = fma((double)position, (double)frequency, -x);
    const double turns = x * kPerTurn, rest = fma(x, kPerTurn, -turns) + fma(x, kPerTurnRest, x_rest * kPerTurn);
    return (float)((turns - rint(turns)) + rest);
}

}  // namespace lvlm
