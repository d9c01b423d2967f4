// The angle of a rotation without its whole turns.  Runs on the CPU too.
#pragma once
#include "mask.h"

namespace cf {

// position * frequency (radians) in half-turns, -1 .. 1 but for a rounding, off by 2^-24 of one, its rounding to fp32, whatever the position, where the angle is below
// 2^40 radians.  The product has 55 bits and 1 / 2 pi more than any type, so both are taken as a double and what that leaves: with the double alone the error
// grows with the angle, to 2^-21 of a half-turn at 2^30 turns.  (The whole turns' subtraction is exact.)
// Infinities and NaNs become NaN.
CF_BOTH float half_turns(float frequency, int position)
{
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;        // 1 / 2 pi
    const double angle = (double)frequency * position, rest = __builtin_fma((double)frequency, (double)position, -angle);
    const double whole = __builtin_rint(angle * kTurn);
    return (float)(2.0 * (__builtin_fma(angle, kTurn, -whole) + __builtin_fma(angle, kTurnRest, rest * kTurn)));
}

}  // namespace cf
