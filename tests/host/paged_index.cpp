// Where the tokens of a paged batch lie (csrc/paged.h): every row of a batch is found in its sequence, values out of range
// are named and never followed, and a row's power of two is the least one that fits.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "paged.h"

using namespace s2a;

static int fail(const char* what, long long a = 0, long long b = 0) {
    std::printf("%s %lld %lld\n", what, a, b);
    return 1;
}

static int batches() {
    std::srand(5);
    for (int round = 0; round < 2000; ++round) {
        const int B = 1 + std::rand() % 9, page_log2 = 4 + std::rand() % 5, width = 1 + std::rand() % 6, pages = 1 + std::rand() % 40;
        std::vector<int> starts(B + 1), lengths(B), table(B * width);
        starts[0] = std::rand() % 3;
        for (int b = 0; b < B; ++b) {
            lengths[b] = std::rand() % ((width << page_log2) + 1);
            const int n = lengths[b] == 0 ? 0 : std::rand() % 3 == 0 ? 0 : 1 + std::rand() % (lengths[b] < 20 ? lengths[b] : 20);
            starts[b + 1] = starts[b] + n;
        }
        const int T = starts[B] + std::rand() % 4 + (starts[B] == 0);
        for (int& x : table) x = std::rand() % (pages + 8) - 4;  // some of them are not in the pool
        PagedBatch batch{table.data(), starts.data(), lengths.data(), width, B, T};
        PagedPool pool{};
        pool.pages = pages, pool.Hkv = 1 + std::rand() % 5, pool.page_log2 = page_log2;
        for (int t = 0; t < T; ++t) {
            int want = -1;
            for (int b = 0; b < B; ++b)
                if (t >= starts[b] && t < starts[b + 1]) want = b;
            const int got = find_sequence(starts.data(), B, t);
            if (got < 0 || got >= B) return fail("sequence out of range", t, got);
            Sequence s;
            if (sequence_of(batch, page_log2, 20, got, &s) != 0) return fail("a good sequence is refused", got);
            const bool in = t >= s.row0 && t < s.row0 + s.n;
            if (in != (want >= 0) || (in && got != want)) return fail("row in another sequence", t, got);
            if (!in) continue;
            const int pos = s.length - s.n + t - s.row0;
            const int page = table[got * width + (pos >> page_log2)];
            const long long row = pool_row(batch, pool, got, pos);
            if (page < 0 || page >= pages) {
                if (row != -1) return fail("a page that is not in the pool is followed", page, row);
            } else if (row != ((static_cast<long long>(page) * pool.Hkv) << page_log2) + (pos & ((1 << page_log2) - 1))) {
                return fail("row of the pool", pos, row);
            }
        }
        // one value at a time is put out of range
        const int b = std::rand() % B;
        Sequence s;
        const int length = lengths[b], end = starts[b + 1], n = end - starts[b];
        auto expect = [&](int code) { return sequence_of(batch, page_log2, 20, b, &s) == code && s.n == 0; };
        lengths[b] = n - 1;
        if (!expect(kBadLength)) return fail("length below the new tokens");
        lengths[b] = (width << page_log2) + 1;
        if (!expect(kBadLength)) return fail("length above the table");
        lengths[b] = length;
        starts[b + 1] = starts[b] - 1;
        if (!expect(kBadStarts)) return fail("falling starts");
        starts[b + 1] = T + 1;
        if (!expect(kBadStarts)) return fail("starts above T");
        starts[b + 1] = end;
        const int row0 = starts[b];
        starts[b] = -1;
        if (!expect(kBadStarts)) return fail("negative start");
        starts[b] = row0;
        if (n > 0 && sequence_of(batch, page_log2, n - 1, b, &s) != kBadNew) return fail("more new tokens than said");
        // whatever starts hold, a sequence of the batch comes back
        for (int i = 0; i < 50; ++i) {
            for (int& x : starts) x = std::rand() - RAND_MAX / 2;
            const int got = find_sequence(starts.data(), B, std::rand() % T);
            if (got < 0 || got >= B) return fail("wild starts", got);
        }
    }
    // a long table: the entry's offset passes 32 bits only with the sequence's own
    PagedBatch batch{nullptr, nullptr, nullptr, 1 << 20, 4096, 1};
    if (static_cast<long long>(batch.B - 1) * batch.width <= 0x7fffffffLL) return fail("not a long table");
    return 0;
}

static int exponents() {
    for (uint32_t bits = 0; bits < 0x7f80; ++bits) {
        const uint32_t wide = bits << 16;
        float x;
        std::memcpy(&x, &wide, 4);
        const int e = row_exponent(bits);
        if (e < kExpLeast || e > 120) return fail("exponent out of range", bits, e);
        if (std::ldexp(448.0, e) < x) return fail("does not fit", bits, e);
        if (e > kExpLeast && std::ldexp(448.0, e - 1) >= x) return fail("not the least", bits, e);
    }
    for (uint32_t bits = 0x7f80; bits < 0x8000; ++bits)
        if (row_exponent(bits) != kExpNotFinite) return fail("not marked", bits);
    return 0;
}

// Every token of a batch is in exactly one of the tiling kernel's places, whatever lengths the sequences have.
static int slots() {
    std::srand(6);
    for (int round = 0; round < 3000; ++round) {
        const int B = 1 + std::rand() % 9, span_log2 = 1 + std::rand() % 8;
        std::vector<int> starts(B + 1);
        starts[0] = std::rand() % 4 == 0 ? std::rand() % 300 : 0;
        for (int b = 0; b < B; ++b) starts[b + 1] = starts[b] + (std::rand() % 3 == 0 ? 0 : std::rand() % 700);
        const int T = starts[B] + (std::rand() % 2 ? std::rand() % 300 : 0) + (starts[B] == 0), count = slot_count(T, B, span_log2);
        std::vector<int> seen(T, 0);
        for (int slot = 0; slot < count; ++slot) {
            const int b = find_slot(starts.data(), B, span_log2, slot);
            if (b < 0 || b >= B) return fail("place in no sequence", slot, b);
            const long long at = static_cast<long long>(slot - first_slot(starts[b], b, span_log2)) << span_log2;
            if (at < 0) continue;
            for (long long i = at; i < at + (1 << span_log2) && i < starts[b + 1] - starts[b]; ++i) ++seen[starts[b] + i];
        }
        for (int t = 0; t < T; ++t)
            if (seen[t] != (t >= starts[0] && t < starts[B])) return fail("token in another number of places than one", t, seen[t]);
        for (int i = 0; i < 20; ++i) {
            for (int& x : starts) x = std::rand() - RAND_MAX / 2;
            const int got = find_slot(starts.data(), B, span_log2, std::rand() % count);
            if (got < 0 || got >= B) return fail("wild starts", got);
        }
    }
    return 0;
}

// The blocks of keys are each named once, in order, and hold every key that a token attends.
static int blocks() {
    std::srand(7);
    for (int round = 0; round < 20000; ++round) {
        const int block = round % 2 ? 16 : 128, first = std::rand() % 700, last = first + std::rand() % 260;
        const int window = std::rand() % 3 == 0 ? 0 : 1 + std::rand() % (std::rand() % 2 ? 20 : 500), sinks = std::rand() % 3 == 0 ? 0 : std::rand() % 300;
        const KeyBlocks k = key_blocks(first, last, window, sinks, block);
        std::vector<int> held(last / block + 1, 0);
        int before = -1;
        for (int i = 0; i < k.count; ++i) {
            const int x = k.at(i);
            if (x <= before || x > last / block) return fail("blocks out of order", x, before);
            before = x, held[x] = 1;
        }
        for (int j = 0; j <= last; ++j) {
            bool any = false;
            for (int p = first; p <= last; ++p) any |= attends(p, j, window, sinks);
            if (any != any_attends(first, last, j, window, sinks)) return fail("some attend", j, any);
            if (any && !held[j / block]) return fail("a key is left out", j);
            if (j % block == 0) {
                bool all = true;
                for (int p = first; p <= last; ++p)
                    for (int x = j; x < j + block; ++x) all &= attends(p, x, window, sinks);
                const bool said = all_attend(first, last, j, block, window, sinks);
                if (said && !all) return fail("not all attend", j, first);
                if (all && !said && window == 0) return fail("all attend", j, first);
            }
        }
        if (held[last / block] == 0) return fail("the last block is left out", last);
    }
    return 0;
}

// The bits of 32 keys at a time, positions, windows and sinks near 2^31 too.
static int bits() {
    std::srand(9);
    const int most = 0x7fffffff;
    for (int round = 0; round < 200000; ++round) {
        const int far = round % 4 == 0 ? most - 1100 : 0, j = far + std::rand() % 40 * 16, p = j - std::rand() % 200 + std::rand() % 400;
        if (p < 0) continue;
        const int pick = std::rand() % 4, window = pick == 0 ? 0 : pick == 1 ? most - std::rand() % 40 : 1 + std::rand() % 300;
        const int sinks = std::rand() % 3 == 0 ? 0 : std::rand() % 5 == 0 ? most : std::rand() % 700;
        const uint32_t got = attended(p, j, window, sinks);
        for (int i = 0; i < 32; ++i)
            if ((got >> i & 1) != static_cast<uint32_t>(attends(p, j + i, window, sinks))) return fail("bit of a key", p, j + i);
    }
    return 0;
}

int main() {
    if (batches() || exponents() || slots() || blocks() || bits()) return 1;
    std::printf("ok\n");
}
