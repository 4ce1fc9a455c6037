// Frequencies of the rotary positions in units of 2^-64 turns (sa_rotary.hip), on the host.
#pragma once

#include <math.h>
#include <stdint.h>

namespace sa {

// F_t = base^(-2 t / size) / (2 pi) in units of 2^-64 turns, for the size / 2 pairs of an axis of
// `size` elements, in extended precision (64 bits of mantissa).  Every 16th by a power of its own (a
// unit in the last place, 2^-63 relative, at most), the 15 behind it by products with one step: each
// 2^-64 off, and 2^-63 by the step.  So (2 + 2 + 15 * 3) 2^-64 relative of 2^64 / (2 pi) f_t, and half a unit
// by the rounding to an integer: 8.4 units at most.
constexpr double kMaxTurnUnits = 8.4;
inline void turn_units(double base, int size, uint64_t* turn) {
    const long double unit = 0x1p64L / 6.283185307179586476925286766559L, step = powl(base, -2.0L / size);
    long double f = unit;
    for (int t = 0; t < size / 2; ++t, f *= step) {
        if (t > 0 && t % 16 == 0) f = unit * powl(base, -2.0L * t / size);
        turn[t] = (uint64_t)(f + 0.5L);
    }
}

}  // namespace sa
