// Entries of a table that is longer than 2^31 (csrc/paged.h).
#include <cstdio>

#include "paged.h"

using namespace s2a;

int main() {
    for (int width : {1, 3, 1 << 20, 0x7fffffff})
        for (int b : {0, 1, 2047, 4095, 0x7ffffffe}) {
            const PagedBatch batch{nullptr, nullptr, nullptr, width, 0x7fffffff, 1};
            const unsigned long long want = static_cast<unsigned long long>(b) * static_cast<unsigned long long>(width);
            if (table_row(batch, b) < 0 || static_cast<unsigned long long>(table_row(batch, b)) != want) return std::printf("sequence %d of %d entries\n", b, width), 1;
        }
    std::printf("ok\n");
}
