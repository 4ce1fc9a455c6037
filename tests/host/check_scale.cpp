// Host check of the scale exponents (csrc/sa_e4m3.h) against their definition: the
// least e with amax <= 448 * 2^e, in [-100, 120], at and around every border.
#include <cmath>
#include <cstdio>
#include <cstring>

#include "sa_e4m3.h"

static uint32_t bits(float x) {
    uint32_t u;
    std::memcpy(&u, &x, 4);
    return u;
}

int main() {
    long long checked = 0;
    for (int p = -149; p <= 119; ++p)
        for (int step = -2; step <= 2; ++step) {
            float x = (float)std::ldexp(448.0, p);
            for (int s = 0; s < (step < 0 ? -step : step); ++s) x = std::nextafterf(x, step < 0 ? 0.f : INFINITY);
            if (!std::isfinite(x)) continue;
            int want = sa::kMinExp;
            while (want < sa::kMaxExp && (double)x > std::ldexp(448.0, want)) ++want;
            if (sa::scale_exponent(bits(x)) != want) {
                std::printf("amax %g: %d, want %d\n", x, sa::scale_exponent(bits(x)), want);
                return 1;
            }
            ++checked;
        }
    for (float x : {0.f, 1e-45f, 1e-38f, 3.4028235e38f}) {
        int want = sa::kMinExp;
        while (want < sa::kMaxExp && (double)x > std::ldexp(448.0, want)) ++want;
        if (sa::scale_exponent(bits(x)) != want) return 1;
        ++checked;
    }
    for (int e = sa::kMinExp; e <= sa::kMaxExp; ++e, ++checked) {
        const float x = (float)std::ldexp(1.0, e);
        if (sa::power_bits(e) != bits(x) || sa::exponent_of(bits(x)) != e) return 1;
    }
    // memory that was never stored to: any bits give an exponent in range
    for (uint64_t u = 0; u < (1ull << 32); u += 9973, ++checked) {
        const int e = sa::exponent_of((uint32_t)u);
        if (e < sa::kMinExp || e > sa::kMaxExp) return 1;
    }
    std::printf("ok %lld\n", checked);
    return 0;
}
