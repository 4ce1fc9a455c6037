// Host check of the 32-bit index space that the step over an 8-bit cache walks
// (KeySet) against the order that DecodeSet defines (itself checked against the set
// definitions in check_decode_set.cpp), written out in 64 bits: every key of small sets, and
// first, last, border and spread keys of sets at the furthest positions and widest strides.
#include <cstdio>
#include <initializer_list>

#include "sa_pattern.h"

static long long checked = 0;

// Key t: A1 ascending, then A2 outside it (strided: downwards; fixed: the earlier summary columns upwards).
static long long key(int pattern, int part, long long pos, long long l, long long c, long long w, long long n1, long long lo,
                     long long t) {
    if (part != sa::PART_A2 && t < n1) return lo + t;
    const long long u = part == sa::PART_A2 ? t : t - n1;
    if (pattern == sa::STRIDED) return pos - (u + (part == sa::PART_A2 ? 0 : 2)) * l;
    return u / c * l + w + u % c;
}

static int check(int pattern, int part, int32_t pos, int32_t l, int32_t c, int32_t w, long long most) {
    const sa::DivL dc = sa::make_divl(c > 0 ? c : 1);
    const sa::DecodeSet d(pattern, part, pos, l, c, w, dc);
    const sa::KeySet k(d);
    if (k.count != (uint64_t)d.count) {
        std::printf("count %u, want %lld\n", k.count, (long long)d.count);
        return 1;
    }
    const long long step = d.count > most ? d.count / most : 1;
    auto same = [&](long long t) {
        if (t < 0 || t >= d.count) return true;
        ++checked;
        const long long want = key(pattern, part, pos, l, c, w, d.n1, d.a1_lo, t);
        if (k.at((uint32_t)t) == want) return true;
        std::printf("pattern %d part %d pos %d l %d c %d w %d t %lld: %d, want %lld\n", pattern, part, pos, l, c, w, t,
                    k.at((uint32_t)t), want);
        return false;
    };
    for (long long t = 0; t < d.count; t += step)
        if (!same(t)) return 1;
    for (long long t : {(long long)d.n1 - 1, (long long)d.n1, (long long)d.n1 + 1, (long long)d.count - 1, (long long)d.count - 2})
        if (!same(t)) return 1;
    return 0;
}

int main() {
    const int strided = sa::STRIDED, fixed = sa::FIXED;
    for (int part = 0; part < 3; ++part) {
        for (int l = 1; l <= 20; ++l)
            for (int pos = 0; pos < 90; ++pos) {
                if (check(strided, part, pos, l, 0, 0, 1000)) return 1;
                for (int c = 1; c <= l; ++c)
                    for (int w = 0; w + c <= l; ++w)
                        if (check(fixed, part, pos, l, c, w, 1000)) return 1;
            }
        const int32_t top = 2147483647;
        for (int32_t pos : {top, top - 1, 1 << 30, (1 << 20) + 7})
            for (int32_t l : {1, 2, 3, 1000, 65536, 1 << 30, top - 1, top}) {
                if (check(strided, part, pos, l, 0, 0, 5000)) return 1;
                for (int32_t c : {1, 2, 31, 32, 997, l})
                    if (c <= l && check(fixed, part, pos, l, c, l - c, 5000)) return 1;
            }
    }
    std::printf("ok %lld\n", checked);
    return 0;
}
