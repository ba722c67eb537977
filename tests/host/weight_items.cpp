// weights_item(): the items of the tiling kernel, whole or in pieces, have each pair of a row and a key that it attends exactly once, and the pieces of an
// item are numbered without a gap, which is what the kernel that adds them up goes by.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "evict.h"

using namespace s2a;

static int pick(int low, int high) { return low + std::rand() % (high - low + 1); }

int main() {
    std::srand(7);
    long long pairs = 0, split = 0;
    for (int round = 0; round < 400; ++round) {
        const int B = pick(1, 3), page_log2 = pick(4, 8), Hkv = pick(1, 2);
        const int reps[] = {1, 2, 3, 4, 7, 8, 12, 16, 64};
        const int rep = reps[pick(0, 8)], most_length = pick(1, 4) * 300;
        std::vector<int> starts(B + 1), lengths(B);
        int longest = 1, most_new = 1;
        starts[0] = pick(0, 2);
        for (int b = 0; b < B; ++b) {
            lengths[b] = pick(0, most_length);
            const int n = lengths[b] == 0 ? 0 : pick(0, 3) == 0 ? pick(0, std::min(3, lengths[b])) : pick(1, lengths[b]);
            starts[b + 1] = starts[b] + n;
            longest = std::max(longest, lengths[b]), most_new = std::max(most_new, n);
        }
        const int width = (longest + (1 << page_log2) - 1) >> page_log2;
        WeightsTileParams p{};
        WeightsParams& a = p.a;
        a.batch = PagedBatch{nullptr, starts.data(), lengths.data(), width, B, std::max(1, starts[B])};
        a.pool.Hkv = Hkv, a.pool.page_log2 = page_log2;
        a.rep = rep, a.H = rep * Hkv, a.most_new = most_new + pick(0, 3);
        const int windows[] = {0, 1, 40, 100, 129, 300, 600}, firsts[] = {0, 4, 17, 130, 300, 700};
        a.window = windows[pick(0, 6)], a.sinks = firsts[pick(0, 5)];
        a.few_rows = pick(0, 1) * kStreamedRows;
        while (p.pack_log2 < 6 && rep % (2 << p.pack_log2) == 0) ++p.pack_log2;
        const int groups = rep >> p.pack_log2, tokens = kTile >> p.pack_log2, units = B * Hkv;
        p.blocks = ((width << page_log2) + kWeightKeys - 1) / kWeightKeys;
        p.pieces = pick(1, 16);
        p.items = p.blocks * p.pieces * units;
        p.by_units = FastDiv(units), p.by_pieces = FastDiv(p.pieces), p.by_heads = FastDiv(Hkv), p.by_groups = FastDiv(groups);
        // of each unit: [token][head group][key], by how many items
        std::vector<std::vector<unsigned char>> seen(units);
        for (int u = 0; u < units; ++u) seen[u].assign(static_cast<size_t>(starts[u / Hkv + 1] - starts[u / Hkv]) * groups * lengths[u / Hkv], 0);
        for (int block = 0; block < p.blocks; ++block)
            for (int u = 0; u < units; ++u) {
                WeightsItem whole;
                const bool any = weights_item(p, block * p.pieces * units + u, &whole);
                for (int piece = 0; piece < p.pieces; ++piece) {
                    WeightsItem w;
                    const bool there = weights_item(p, (block * p.pieces + piece) * units + u, &w);
                    if (there != (any && piece < whole.pieces)) return std::printf("piece %d of %d\n", piece, whole.pieces), 1;
                    if (!there) continue;
                    if (w.b != u / Hkv || w.hk != u % Hkv || w.key0 != whole.key0 || w.pieces != whole.pieces || w.row0 != starts[w.b]) return std::printf("another item\n"), 1;
                    split += w.pieces > 1;
                    const int n = starts[w.b + 1] - starts[w.b], length = lengths[w.b];
                    for (int r = w.r0; r < w.r1; ++r)
                        for (int t = (w.t_lo + r / groups) * tokens; t < std::min(n, (w.t_lo + r / groups + 1) * tokens); ++t)
                            for (int key = w.key0; key < std::min(length, w.key0 + kWeightKeys); ++key) ++seen[u][(static_cast<size_t>(t) * groups + r % groups) * length + key];
                }
            }
        for (int u = 0; u < units; ++u) {
            const int b = u / Hkv, n = starts[b + 1] - starts[b], length = lengths[b];
            const bool mine = n > a.few_rows / rep;
            for (int t = 0; t < n; ++t)
                for (int g = 0; g < groups; ++g)
                    for (int key = 0; key < length; ++key) {
                        const int times = seen[u][(static_cast<size_t>(t) * groups + g) * length + key];
                        const bool counts = mine && attends(length - n + t, key, a.window, a.sinks);
                        if (times > 1 || (counts && times != 1) || (!mine && times)) return std::printf("token %d of %d, key %d of %d: %d times\n", t, n, key, length, times), 1;
                        pairs += counts;
                    }
        }
    }
    if (pairs < 1000000 || split < 1000) return std::printf("too few: %lld %lld\n", pairs, split), 1;
    std::printf("ok\n");
    return 0;
}
