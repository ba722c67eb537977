// The keys that no token of a unit attends (csrc/paged.h), against the definition key by key.
#include <cstdio>
#include <cstdlib>

#include "paged.h"

using namespace s2a;

int main() {
    std::srand(11);
    for (int round = 0; round < 60000; ++round) {
        const int far = round % 5 == 0 ? (1 << 30) - 2000 : 0;
        const int first = far + std::rand() % 700, last = first + std::rand() % 260, n = round % 2 ? 16 << std::rand() % 4 : 1 + std::rand() % 130;
        const int window = std::rand() % 3 == 0 ? 0 : std::rand() % 9 == 0 ? (1 << 30) : 1 + std::rand() % (std::rand() % 2 ? 20 : 500);
        const int sinks = std::rand() % 3 == 0 ? 0 : std::rand() % 9 == 0 ? (1 << 30) : std::rand() % 300;
        const int key0 = std::rand() % 3 == 0 ? 0 : far + std::rand() % 8 * 128;
        const HiddenKeys h = hidden_keys(first, last, key0, window, sinks);
        const int i0 = (std::rand() % 10) * 16;
        bool any = false, all = true;
        for (int i = 0; i < i0 + n; ++i) {
            const bool hidden = !any_attends(first, last, key0 + i, window, sinks);
            if (hidden != h.has(i)) return std::printf("key %d from %d: %d\n", i, key0, hidden), 1;
            if (i < n) any |= hidden;
            if (i >= i0) all &= hidden;
        }
        if (any != h.any(n)) return std::printf("any of %d from %d: %d\n", n, key0, any), 1;
        if (all != h.all(i0, n)) return std::printf("all of %d from %d: %d\n", n, key0 + i0, all), 1;
    }
    std::printf("ok\n");
}
