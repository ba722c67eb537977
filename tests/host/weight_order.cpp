// weight_order(): whole numbers in the order of the weights that they are made of.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <limits>

#include "evict.h"

static uint32_t order(float x) {
    uint32_t bits;
    std::memcpy(&bits, &x, 4);
    return s2a::weight_order(bits);
}

int main() {
    const float inf = std::numeric_limits<float>::infinity(), nan = std::numeric_limits<float>::quiet_NaN();
    const float rising[] = {-inf, -3e38f, -1.f, -1e-45f, 0.f, 1e-45f, 1e-38f, 0.5f, std::nextafter(0.5f, 1.f), 1.f, 3e38f, inf, nan};
    for (int i = 0; i < 13; ++i)
        for (int j = 0; j < 13; ++j)
            if ((order(rising[i]) < order(rising[j])) != (i < j)) return std::printf("%g %g\n", rising[i], rising[j]), 1;
    if (order(-0.f) != order(0.f) || order(-nan) != order(nan)) return std::printf("zeros or NaN\n"), 1;
    std::printf("ok\n");
    return 0;
}
