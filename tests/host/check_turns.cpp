// Prints the rotary frequencies (csrc/sa_turns.h) of the (base, size) pairs given as arguments: a line for each.
#include <cstdio>
#include <cstdlib>

#include "sa_turns.h"

int main(int argc, char** argv) {
    uint64_t turn[64];
    std::printf("%.17g\n", sa::kMaxTurnUnits);
    for (int i = 1; i + 1 < argc; i += 2) {
        const int size = std::atoi(argv[i + 1]);
        sa::turn_units(std::strtod(argv[i], nullptr), size, turn);
        for (int t = 0; t < size / 2; ++t) std::printf("%llu ", (unsigned long long)turn[t]);
        std::printf("\n");
    }
    return 0;
}
