// Attention of many rows over the paged cache, for sm_100a: pieces of prompts.
//
// With p the position of a new token, s_j = scale * q . k_j over the keys j it attends (j <= p, with a window also j > p - window or
// j < sinks): o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), lse = m + log of that sum, in one pass with a running maximum m.
//
// A tile is 128 rows that read the same KV head: `pack` query heads (the largest power of two that divides the query heads of a KV head) of
// 128 / pack neighbouring tokens, token by token, which is one TMA box of q.  A work item is a pair of neighbouring tiles of a sequence
// and head group, against which the cache is streamed in tiles of 128 keys: the blocks of key_blocks(), which are the first
// tokens' and the window's where there is a window.  A key tile is one TMA box for each page (or 128 keys of one).
//
// One persistent block per SM, 512 threads, with the roles and the tensor-memory layout of s2a_fwd_kernel (fwd_kernel.cu), whose
// comments say what they are for:
//   warps 0-3, 4-7   softmax, two groups that take the tiles of an item in turn: one thread per score row
//   warps 8-11       O / l -> bf16 -> global memory; with a cache in 8 bits also Q, K and V to fp16
//   warp 12          work items (cluster launch control), pages and TMA loads, running ahead across items
//   warps 13, 14     tcgen05 MMAs: S = Q K_j^T of both tiles in turn / O += P V_j
// Tensor memory: O of either tile, P of either tile, then one score buffer (HD = 128) or two.
//
// 8-bit caches are multiplied in fp16, which has their values with room for a power of two.  TMA brings the codes to a ring of two raw tiles;
// warps 8-11 write them where the products read them, each row times its power of two relative to the tile's largest (6 binary places
// up: the tile's largest value is below 2^15, rows whose power is 2^-21 of the largest keep all their bits, those below 2^-30 become zeros).
// Q they turn from bf16 to fp16, each row times a power of two that brings its largest value to [2^14, 2^15).  What is the tile's, or the
// row's, then multiplies scores and weights for nothing: it goes into the constants of exp2(score * c - m).  With x a score in units of log2 and 2^e the tile's power of V the weight of
// the second product is 2^(x + e - r + 7), r a running maximum of x + e of the row: the largest term's weight is 2^7 or more, those
// down to 2^-21 of it have all of fp16's 11 bits (bf16 has 8), those below 2^-32 of it vanish.  (Largest of a tile means its largest weight
// times its largest power: rows of V that a row does not attend count for it.)  O is in units of 2^(r - m), m being
// the running maximum of x that the sum of weights goes by.  As bf16, values take five instructions instead of one and a half and the
// four warps cannot keep up: 32k tokens, 2048 new ones, 64 heads over 8 3.03 ms.
#include "paged_device.cuh"

namespace s2a {

namespace {

template <int HD, bool kE4M3>
struct PagedCfg {
    static constexpr int kThreads = 512;
    static constexpr int kBoxes = HD / 64;                  // 64-column boxes per tile
    static constexpr int kBoxBytes = kTile * 128;           // 128 rows x 128 bytes
    static constexpr int kTileBytes = kBoxes * kBoxBytes;   // one Q, K or V tile in bf16
    static constexpr int kRing = (HD == 128) ? 4 : 8;       // K and V tiles in flight: K_0 V_0 K_1 V_1 ...
    static constexpr int kRawRing = kE4M3 ? (HD == 128 ? 2 : 6) : 0;  // the same as codes
    static constexpr int kRawBytes = kTile * HD;
    static constexpr int kStatBytes = 2 * kTile * 4 + (kE4M3 ? 2 * 2 * kTile : 0);  // factors for the read-out, exponents of Q's rows
    // Items in flight: as many as s2a_fwd_kernel's for its ring, see there; with raw tiles those that the warps which turn them
    // into operands are behind with come on top.
    static constexpr int kSched = (HD == 128) ? 6 : kE4M3 ? 12 : 8;
    static_assert(kSched % 2 == 0 && kSched >= (kRing + kRawRing) / 2 + 3, "an item's slot is free when it is written again");
    static constexpr int kBarBytes = (HD == 128) ? 1536 : 4096;
    static constexpr int kSmemBytes = (2 + kRing) * kTileBytes + kRawRing * kRawBytes + kBarBytes + kStatBytes;
    static_assert(kSmemBytes <= 232448, "shared memory");
    static constexpr int kTmemCols = 512;
    static constexpr int kColO = 0, kColP = 2 * HD, kColS = 2 * HD + 2 * 64;
    static constexpr int kScoreBufs = (HD == 128) ? 1 : 2;
    static_assert(kColS + kScoreBufs * kTile <= kTmemCols, "tensor memory");
    // registers per thread after the split; the launch gives kRegsLaunch to each of the 512
    // (the softmax, whose rows are in registers, can spare some for the warps that turn codes into operands: 32k tokens in 8 bits with 184, 88
    // and 56 2150 us, with these 2095)
    static constexpr int kRegsLaunch = 128, kRegsSoftmax = kE4M3 && HD == 128 ? 176 : 184, kRegsReadOut = kE4M3 && HD == 128 ? 104 : 88, kRegsIssue = 56;
    static_assert(2 * kRegsSoftmax + kRegsReadOut + kRegsIssue <= 4 * kRegsLaunch, "register split");
};

struct PagedItem {
    int b, group;          // sequence (-1: no more items), head group
    int row[2], tokens[2];  // of either tile: first row of q and o, tokens (0: no such tile)
    int pos;               // position of the token at row[1]
    int n[2];              // key tiles that either tile's products take: the first n of the item's
    int sink_blocks, low_block;
    int j0;                // first of its key tiles among those of key_blocks()
    int piece;             // -1, or which piece of the split items it is
    uint32_t kv0;          // ring position of its first K tile
    __device__ __forceinline__ int key_tile(int j) const { return j0 + j < sink_blocks ? j0 + j : low_block + j0 + j - sink_blocks; }
    // (indexed by a variable, a copy in registers would have to go through local memory)
    __device__ __forceinline__ int row_of(int t) const { return t ? row[1] : row[0]; }
    __device__ __forceinline__ int tokens_of(int t) const { return t ? tokens[1] : tokens[0]; }
    __device__ __forceinline__ int first_pos(int t) const { return t ? pos : pos - (row[1] - row[0]); }
    // of the keys from key0 on, what none of its tokens attends
    __device__ __forceinline__ HiddenKeys hidden(int key0, int window, int sinks) const { return hidden_keys(pos - tokens[0], pos + tokens[1] - 1, key0, window, sinks); }
};

template <int HD, bool kE4M3>
struct PagedBars {
    using C = PagedCfg<HD, kE4M3>;
    // by group of softmax warps
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2], s_empty[2];
    uint64_t p_full[2], p_rest[2], p_empty[2];
    uint64_t o_full[2], o_empty[2];
    uint64_t stat_full[2], stat_empty[2];
    uint64_t kv_full[C::kRing], kv_empty[C::kRing];
    uint64_t raw_full[kE4M3 ? C::kRawRing : 1], raw_empty[kE4M3 ? C::kRawRing : 1], q_ready[2];
    uint64_t sched_full[C::kSched];
    uint64_t list_full[2][C::kSched];
    uint64_t clc, drain[2];
    alignas(16) uint8_t clc_resp[16];
    alignas(16) int8_t exps[kE4M3 ? C::kRawRing : 1][kTile];  // of the raw tiles
    int8_t tile_exp[16];  // of the K and V tiles by ring position: one is written again when its step is long over
    PagedItem item[C::kSched];
    uint8_t list_slot[2][C::kSched];
    uint32_t tmem_slot;
    int abort_flag;
};

// With 8-bit caches the tiles of an item's keys are requested and written in the order K_0 K_1 V_0 K_2 V_1 .. K_n-1 V_n-2 V_n-1: K's room is free a
// step earlier than V's, and in the order of the ring (K_0 V_0 K_1 V_1) it would be written behind V.  Tile x of 2 n: of K or V, and which.
struct TileOfItem {
    bool is_v;
    int j;
    __device__ __forceinline__ TileOfItem(int x, int n) : is_v(x > 0 && ((x & 1) == 0 || x == 2 * n - 1)), j(x == 2 * n - 1 ? n - 1 : is_v ? x / 2 - 1 : (x + 1) / 2) {}
};

// The later tile of a pair is the only one where an item has one; the groups of softmax warps take it in turn (see s2a_fwd_kernel).
__device__ __forceinline__ int group_of_tile(int item, int t) { return (item & 1) ^ t ^ 1; }
__device__ __forceinline__ int tile_of_group(int item, int group) { return (item & 1) ^ group ^ 1; }

constexpr float kLazyRescale = 8.0f;
__device__ __forceinline__ constexpr int key_of_column(int x) { return (x & ~3) | ((x & 1) << 1) | ((x >> 1) & 1); }

// The item of head group `group` whose tokens begin with token `first` of sequence b; false: the sequence has none.
__device__ __forceinline__ bool item_at(const PagedTileParams& p, int group, int b, long long first_token, PagedItem* w) {
    const PagedFwdParams& a = p.a;
    Sequence s;
    if (sequence_of(a.batch, a.pool.page_log2, a.most_new, b, &s) != 0 || s.n * a.rep <= a.few_rows || first_token < 0 || first_token >= s.n) return false;
    const int first = static_cast<int>(first_token), left = s.n - first, tile = kTile >> p.pack_log2;
    w->b = b, w->group = group;
    const bool two = !p.single && left > tile;
    w->tokens[0] = two ? tile : 0;
    w->tokens[1] = two ? (left - tile < tile ? left - tile : tile) : (left < tile ? left : tile);
    w->row[0] = s.row0 + first;
    w->row[1] = w->row[0] + w->tokens[0];
    w->pos = s.length - s.n + first + w->tokens[0];
    const KeyBlocks k = key_blocks(w->pos - w->tokens[0], w->pos + w->tokens[1] - 1, a.window, a.sinks, kTile);
    w->sink_blocks = k.sink_blocks, w->low_block = k.low_block;
    w->n[1] = k.count;
    w->n[0] = two ? k.sink_blocks + (w->pos - 1) / kTile + 1 - k.low_block : 0;
    w->j0 = 0, w->piece = -1;
    return true;
}

// Item `item` as a whole, of a batch of one sequence or of more than kRanked: the places of some head groups side by side (their items read the
// same keys), the last ones first: they have most.
__device__ __forceinline__ bool whole_item(const PagedTileParams& p, int item, PagedItem* w) {
    int group, rank;
    p.order.decode(item, &group, &rank);
    const int slot = p.slots - 1 - rank;
    const int b = find_slot(p.a.batch.starts, p.a.batch.B, p.span_log2, slot);
    return item_at(p, group, b, static_cast<long long>(slot - first_slot(S2A_LOAD(p.a.batch.starts + b), b, p.span_log2)) << p.span_log2, w);
}

// Batches of 2 .. kRanked sequences: a warp knows how many items each has (of a head group) and puts them in order, those with most keys
// first, the head groups of a place side by side.  The last items to be begun are then short ones: a launch ends about as late as
// its last item is long.  (Sequences of 400 to 4001 tokens with 1 to 701 new ones, 32 heads over 8 of 64, in their own order 129 us.)
constexpr int kRanked = kMostRanked;
struct Ranking {
    int start[kRanked / 32], count[kRanked / 32], total;  // of sequences lane and lane + 32
    __device__ __forceinline__ void set(const PagedTileParams& p) {
        const PagedFwdParams& a = p.a;
        const int lane = threadIdx.x & 31;
        int keys[kRanked / 32];
        total = 0;
#pragma unroll
        for (int u = 0; u < kRanked / 32; ++u) {
            Sequence s;
            start[u] = count[u] = keys[u] = 0;
            const int b = lane + 32 * u;
            if (b < a.batch.B && sequence_of(a.batch, a.pool.page_log2, a.most_new, b, &s) == 0 && s.n > 0 && s.n * a.rep > a.few_rows) {
                count[u] = (s.n + (1 << p.span_log2) - 1) >> p.span_log2;
                keys[u] = key_blocks(s.length - s.n, s.length - 1, a.window, a.sinks, kTile).count;
            }
            total += __reduce_add_sync(0xffffffffu, count[u]);
        }
        for (int i = 0; i < a.batch.B; ++i) {
            const int n = __shfl_sync(0xffffffffu, i < 32 ? count[0] : count[1], i & 31), k = __shfl_sync(0xffffffffu, i < 32 ? keys[0] : keys[1], i & 31);
#pragma unroll
            for (int u = 0; u < kRanked / 32; ++u)
                if (k > keys[u] || (k == keys[u] && i < lane + 32 * u)) start[u] += n;
        }
    }
    // by a whole warp
    __device__ __forceinline__ bool item(const PagedTileParams& p, int id, PagedItem* w) const {
        int group;
        const int place = p.by_groups(id, &group);
        if (place >= total) return false;
        int b = 0, x = 0;
#pragma unroll
        for (int u = 0; u < kRanked / 32; ++u) {
            const uint32_t found = __ballot_sync(0xffffffffu, place >= start[u] && place < start[u] + count[u]);
            const int from = __ffs(found) - 1, left = __shfl_sync(0xffffffffu, start[u] + count[u] - 1 - place, from & 31);
            if (found != 0) b = from + 32 * u, x = left;
        }
        return item_at(p, group, b, static_cast<long long>(x) << p.span_log2, w);
    }
};

// Key tiles of a piece of a split item (the last piece has fewer, or there are fewer pieces).
__device__ __forceinline__ int piece_tiles(const PagedTileParams& p, const PagedItem& whole) { return (whole.n[1] + p.split - 1) / p.split; }

// Item `item` as a whole, by a whole warp.
__device__ __forceinline__ bool any_item(const PagedTileParams& p, const Ranking& ranking, int item, PagedItem* w) {
    return p.ranked ? ranking.item(p, item, w) : whole_item(p, item, w);
}

// Work item `id`, by a whole warp: the items before first_split, then the pieces of the others.
__device__ __forceinline__ bool paged_item(const PagedTileParams& p, const Ranking& ranking, int id, PagedItem* w) {
    if (id < p.first_split) return any_item(p, ranking, id, w);
    const int piece = id - p.first_split;
    int part;
    if (!any_item(p, ranking, p.first_split + p.by_split(piece, &part), w)) return false;
    const int tiles = piece_tiles(p, *w), j0 = part * tiles;
    if (j0 >= w->n[1]) return false;
    w->j0 = j0, w->piece = piece;
    w->n[1] = w->n[1] - j0 < tiles ? w->n[1] - j0 : tiles;
    w->n[0] = w->n[0] - j0 < tiles ? w->n[0] - j0 : tiles;
    if (w->n[0] <= 0) w->n[0] = 0, w->tokens[0] = 0, w->row[0] = w->row[1];  // (the earlier tile attends none of the piece's keys)
    return true;
}
// What pieces leave for s2a_paged_join_kernel: of piece x and tile t O [d / 4][128 rows] by fours, then the running maximum and the sum of the rows.
template <int HD>
__device__ __forceinline__ float* piece_result(const PagedTileParams& p, int piece, int t) {
    return p.pieces + (2ll * piece + t) * (kTile * (HD + 2));
}

// kWindow: whether the call has one.  (Pages and values in front of a window are left alone, see hidden_keys(); looked for in every call, they cost
// 2048 new tokens of 32k on 64 heads over 8 in 8 bits 2170 us instead of 2134.)
template <int HD, bool kE4M3, bool kWindow>
__global__ void __launch_bounds__(PagedCfg<HD, kE4M3>::kThreads, 1) s2a_paged_fwd_kernel(const __grid_constant__ PagedTileParams p) {
    using C = PagedCfg<HD, kE4M3>;
    using Bars = PagedBars<HD, kE4M3>;
    static_assert(sizeof(Bars) <= C::kBarBytes, "barrier block");
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;                                // two query tiles
    uint8_t* sKV = sQ + 2 * C::kTileBytes;             // ring of K and V tiles
    uint8_t* sRaw = sKV + C::kRing * C::kTileBytes;    // ring of their codes
    Bars* bars = reinterpret_cast<Bars*>(sRaw + C::kRawRing * C::kRawBytes);
    float* sStat = reinterpret_cast<float*>(reinterpret_cast<uint8_t*>(bars) + C::kBarBytes);  // [group][128 rows]
    int8_t* sQExp = reinterpret_cast<int8_t*>(sStat + 2 * kTile);  // [group][item of the group, odd or even][128 rows]
    const PagedFwdParams& a = p.a;
    const int window = kWindow ? a.window : 0;

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(&bars->q_full[t], 1);
            mbar_init(&bars->q_empty[t], 1);
            mbar_init(&bars->s_full[t], 1);
            mbar_init(&bars->s_empty[t], 4);
            mbar_init(&bars->p_empty[t], 1);
            mbar_init(&bars->p_full[t], 4);
            mbar_init(&bars->p_rest[t], 4);
            mbar_init(&bars->o_full[t], 1);
            mbar_init(&bars->o_empty[t], 4);
            mbar_init(&bars->stat_full[t], 4);
            mbar_init(&bars->stat_empty[t], 4);
            mbar_init(&bars->drain[t], 1);
            mbar_init(&bars->q_ready[t], 4);
        }
        for (int x = 0; x < C::kRawRing; ++x) {
            mbar_init(&bars->raw_full[x], 1);
            mbar_init(&bars->raw_empty[x], 4);
        }
        for (int x = 0; x < C::kRing; ++x) {
            mbar_init(&bars->kv_full[x], kE4M3 ? 4 : 1);
            mbar_init(&bars->kv_empty[x], 1);
        }
        for (int x = 0; x < C::kSched; ++x) {
            mbar_init(&bars->sched_full[x], 1);
            mbar_init(&bars->list_full[0][x], 1);
            mbar_init(&bars->list_full[1][x], 1);
        }
        mbar_init(&bars->clc, 1);
        fence_barrier_init();
        tma_prefetch_desc(&p.tm_q);
        tma_prefetch_desc(&p.tm_k);
        tma_prefetch_desc(&p.tm_v);
    }
    if (warp == 13) {
        tmem_alloc(&bars->tmem_slot, C::kTmemCols);
        tmem_relinquish();
    }
    // (behind the splitting kernel of the same call there is nothing to wait for but what that one has waited for; see the end)
    if (!p.beside) wait_for_predecessor();
    // An earlier report (a wait that expired, a value out of range) leaves the status word set: nothing is done then.
    if (threadIdx.x == 0) bars->abort_flag = *reinterpret_cast<volatile int*>(a.status);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    release_successor();
    const uint32_t tmem_base = bars->tmem_slot;
    if (bars->abort_flag != 0) {
        if (warp == 13) tmem_dealloc(tmem_base, C::kTmemCols);
        if (p.beside) wait_for_predecessor();
        return;
    }
    if (blockIdx.x == 0) check_batch(a.batch, a.pool.page_log2, a.most_new, a.status, a.host_status);
    const WaitCtx ctx{&bars->abort_flag, a.status, a.host_status};

    auto next_item = [&](int k, int where, PagedItem* w) -> bool {
        if (!mbar_wait_uniform(&bars->sched_full[k % C::kSched], (k / C::kSched) & 1, ctx, where)) return false;
        *w = bars->item[k % C::kSched];
        return w->b >= 0;
    };

    if (warp >= 12) {
        setmaxnreg_dec<C::kRegsIssue>();
        if (warp == 12) {
            // ======================= work items, TMA loads ===========================================
            // The whole warp walks the loop: lane i requests the i-th page of a tile, and has looked up that of the next
            // tile before it waits for room.
            uint32_t kv = 0;              // K and V tiles requested so far
            uint32_t n_q[2] = {0, 0};     // query tiles requested so far for either group
            uint32_t n_list[2] = {0, 0};  // items in the list of either group
            uint32_t n_clc = 0;
            bool ok = true;
            int id = static_cast<int>(blockIdx.x);
            Ranking ranking;
            if (p.ranked) ranking.set(p);
            const int piece_log2 = a.pool.page_log2 < 7 ? a.pool.page_log2 : 7;  // keys of a box
            auto next_id = [&]() {
                if (lane == 0) {
                    mbar_expect_tx(&bars->clc, 16);
                    clc_try_cancel(bars->clc_resp, &bars->clc);
                }
                __syncwarp();
                if (!mbar_wait_uniform(&bars->clc, n_clc & 1, ctx, kWaitPagedFwd + 1)) {
                    if (lane == 0) {
                        mbar_wait_drain(&bars->clc, n_clc & 1);  // the answer must not land after the block has gone
                    }
                    ok = false;
                    return -1;
                }
                ++n_clc;
                const int x = clc_granted_block(bars->clc_resp);
                fence_proxy_async();  // the answer has been read before the next one is written
                __syncwarp();
                return x;
            };
            auto load_q = [&](const PagedItem& w, int t, int g) {
                const uint32_t n = g ? n_q[1]++ : n_q[0]++;
                if (!mbar_wait_uniform(&bars->q_empty[g], (n & 1) ^ 1, ctx, kWaitPagedFwd + 2)) {
                    --(g ? n_q[1] : n_q[0]);
                    ok = false;
                    return;
                }
                if (lane == 0) {
                    mbar_expect_tx(&bars->q_full[g], C::kTileBytes);
                    for (int bx = 0; bx < C::kBoxes; ++bx)
                        tma_load_3d(smem_u32(sQ + g * C::kTileBytes + bx * C::kBoxBytes), &p.tm_q, smem_u32(&bars->q_full[g]), bx * 64,
                                    w.group << p.pack_log2, w.row_of(t));
                }
                __syncwarp();
            };
            // The table's entry for the piece of key tile `tile` that is this lane's.  (Every lane has one, and it is looked at when it is used, one
            // tile later: its latency is then nobody's.)
            auto look_up = [&](const int* table, int length, int tile) {
                const int key = tile * kTile + (lane << piece_log2);
                return S2A_LOAD(table + ((key < length ? key : length - 1) >> a.pool.page_log2));
            };
            // Pool row (in head hk) of that piece, -1: none of its keys is attended.
            auto piece_row = [&](int page, int hk, const HiddenKeys& hidden, int tile) {
                const int key = tile * kTile + (lane << piece_log2);
                if (lane >= kTile >> piece_log2 || hidden.all(key, 1 << piece_log2)) return -1;
                if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.pool.pages)) {
                    report_bad_index(a.status, a.host_status, kBadPage);
                    return -1;
                }
                return ((page * a.pool.Hkv + hk) << a.pool.page_log2) + (key & ((1 << a.pool.page_log2) - 1));
            };
            auto load_kv = [&](int row, bool k_tile) {
                const int boxes = __popc(__ballot_sync(0xffffffffu, row >= 0));
                if constexpr (kE4M3) {
                    const int st = kv % C::kRawRing;
                    if (!mbar_wait_uniform(&bars->raw_empty[st], ((kv / C::kRawRing) & 1) ^ 1, ctx, kWaitPagedFwd + 3)) { ok = false; return; }
                    if (lane == 0) mbar_expect_tx(&bars->raw_full[st], static_cast<uint32_t>((boxes * (HD + 1)) << piece_log2));
                    __syncwarp();
                    if (row >= 0) {
                        const int at = lane << piece_log2;
                        tma_load_2d(smem_u32(sRaw + st * C::kRawBytes + at * HD), k_tile ? &p.tm_k : &p.tm_v, smem_u32(&bars->raw_full[st]), 0, row);
                        bulk_load_1d(&bars->exps[st][at], (k_tile ? a.pool.k_exp : a.pool.v_exp) + row, 1u << piece_log2, &bars->raw_full[st]);
                    }
                } else {
                    const int st = kv % C::kRing;
                    if (!mbar_wait_uniform(&bars->kv_empty[st], ((kv / C::kRing) & 1) ^ 1, ctx, kWaitPagedFwd + 3)) { ok = false; return; }
                    if (lane == 0) mbar_expect_tx(&bars->kv_full[st], static_cast<uint32_t>((boxes * HD * 2) << piece_log2));
                    __syncwarp();
                    if (row >= 0) {
                        const uint32_t dst = smem_u32(sKV + st * C::kTileBytes) + (lane << piece_log2) * 128, bar = smem_u32(&bars->kv_full[st]);
                        for (int bx = 0; bx < C::kBoxes; ++bx) {
                            if (k_tile) tma_load_4d_at(dst + bx * C::kBoxBytes, &p.tm_k, bar, bx * 64, 0, 0, row / 4);
                            else tma_load_2d(dst + bx * C::kBoxBytes, &p.tm_v, bar, bx * 64, row);
                        }
                    }
                }
                __syncwarp();
                ++kv;
            };
            for (int k = 0; ok; ++k) {
                PagedItem w;
                while (id >= 0 && !paged_item(p, ranking, id, &w)) id = next_id();
                if (id < 0) w.b = -1;
                const int g1 = group_of_tile(k, 1), g0 = group_of_tile(k, 0);
                w.kv0 = kv;
                if (lane == 0) {
                    bars->item[k % C::kSched] = w;
                    mbar_arrive(&bars->sched_full[k % C::kSched]);  // release: the item is visible to whoever sees the phase
                }
                auto enlist = [&](int g) {
                    const uint32_t n = g ? n_list[1]++ : n_list[0]++;
                    if (lane == 0) {
                        bars->list_slot[g][n % C::kSched] = static_cast<uint8_t>(k % C::kSched);
                        mbar_arrive(&bars->list_full[g][n % C::kSched]);
                    }
                };
                enlist(g1);
                if (id < 0 || w.n[0] > 0) enlist(g0);
                __syncwarp();
                if (id < 0) break;
                const int hk = p.by_groups_of_kv(w.group), length = w.pos + w.tokens[1];  // (keys behind the last token are nobody's)
                const int* table = a.batch.table + table_row(a.batch, w.b);
                const HiddenKeys hidden = w.hidden(0, window, a.sinks);
                int row = -1, page = look_up(table, length, w.key_tile(0));
                for (int j = 0; ok && j < w.n[1]; ++j) {
                    const int before = row;
                    row = piece_row(page, hk, hidden, w.key_tile(j));
                    page = look_up(table, length, w.key_tile(j + 1 < w.n[1] ? j + 1 : j));
                    load_kv(row, true);
                    if (j == 0 && ok) load_q(w, 1, g1);
                    if (j == 0 && ok && w.n[0] > 0) load_q(w, 0, g0);
                    // (8 bits: in the order of TileOfItem)
                    if (ok && (!kE4M3 || j > 0)) load_kv(kE4M3 ? before : row, false);
                }
                if (kE4M3 && ok) load_kv(row, false);
                if (ok) id = next_id();
            }
            // nothing may land after the block has gone
            if (lane == 0) {
                if (bars->abort_flag != 0) {
                    for (int t = 0; t < 2; ++t)
                        if (n_q[t] > 0) mbar_wait_drain(&bars->q_full[t], (n_q[t] - 1) & 1);
                    constexpr uint32_t kIn = kE4M3 ? C::kRawRing : C::kRing;
                    for (uint32_t x = (kv > kIn ? kv - kIn : 0); x < kv; ++x)
                        mbar_wait_drain(kE4M3 ? &bars->raw_full[x % kIn] : &bars->kv_full[x % kIn], (x / kIn) & 1);
                }
            }
            __syncwarp();
        } else if (warp <= 14) {
            // ======================= MMA issuers: warp 13 for S = Q K^T, warp 14 for O += P V ============
            constexpr uint32_t idesc_s = kE4M3 ? idesc_f16(128, kTile, 0, 0) : idesc_bf16(128, kTile, 0, 0);  // S = Q K^T   (both K-major)
            constexpr uint32_t idesc_o = kE4M3 ? idesc_f16(128, HD, 0, 1) : idesc_bf16(128, HD, 0, 1);        // O += P V    (V is MN-major)
            const bool is_s = warp == 13;
            const uint32_t aKV = smem_u32(sKV), dQ0 = desc_lo_k_major(smem_u32(sQ));
            uint32_t kv = 0;                    // ring position of the item's K_0
            uint32_t n_it[2] = {0, 0};          // items of either group so far
            uint32_t n_st[2] = {0, 0}, n_s = 0; // steps of either group, score products
            bool ok = true;
            for (int k = 0; ok; ++k) {
                PagedItem w;
                if (!next_item(k, kWaitPagedFwd + 10, &w)) break;
                const int n1 = w.n[1], n0 = w.n[0];
#pragma unroll 1
                for (int h = 0; ok && h < 2 * n1; ++h) {
                    const int t = (h & 1) ^ 1, j = h >> 1, n = t ? n1 : n0, g = group_of_tile(k, t);
                    if (j >= n) continue;
                    const uint32_t x = kv + 2 * j + (is_s ? 0 : 1);
                    const bool last_use = t == 0 || j >= n0;  // of this K or V tile
                    const uint32_t st = (g ? n_st[1] : n_st[0]) & 1, it = (g ? n_it[1] : n_it[0]) & 1;
                    // what tile 1 has used, tile 0 need not wait for again
                    if (t == 1 && !mbar_wait_uniform(&bars->kv_full[x % C::kRing], (x / C::kRing) & 1, ctx, kWaitPagedFwd + 5)) { ok = false; break; }
                    if (is_s) {
                        if (j == 0 && !mbar_wait_uniform(kE4M3 ? &bars->q_ready[g] : &bars->q_full[g], it, ctx, kWaitPagedFwd + 4)) { ok = false; break; }
                        const int buf = C::kScoreBufs == 1 ? 0 : g;
                        const uint32_t use = C::kScoreBufs == 1 ? n_s & 1 : st;
                        if (!mbar_wait_uniform(&bars->s_empty[buf], use ^ 1, ctx, kWaitPagedFwd + 6)) { ok = false; break; }
                        tc_fence_after();
                        const uint32_t at_g = dQ0 + g * (C::kTileBytes >> 4);
                        const uint32_t at_x = desc_lo_k_major(aKV + (x % C::kRing) * C::kTileBytes);
                        const uint32_t acc = tmem_base + C::kColS + buf * kTile;
                        if (elect_one()) {
#pragma unroll
                            for (int kk = 0; kk < HD / 16; ++kk)
                                mma_ss(acc, at_g + desc_step_k_major(kk, C::kBoxBytes), at_x + desc_step_k_major(kk, C::kBoxBytes), idesc_s, kk > 0);
                            mma_commit(&bars->s_full[g]);
                            if (last_use) mma_commit(&bars->kv_empty[x % C::kRing]);
                            if (j == n - 1) mma_commit(&bars->q_empty[g]);
                        }
                        __syncwarp();
                        ++n_s;
                    } else {
                        if (!kE4M3 && t == 1) {
                            // The rows of V that no row of the item attends hold whatever the page held before, or what the ring did: a weight
                            // of zero does not make a NaN go away.  (8-bit tiles are written without them.)
                            const HiddenKeys hidden = w.hidden(w.key_tile(j) * kTile, window, a.sinks);
                            if (hidden.any(kTile)) {
                                const uint32_t chunk = aKV + (x % C::kRing) * C::kTileBytes + (lane & 7) * 16;
                                for (int key = lane >> 3; key < kTile; key += 4)
                                    for (int bx = 0; hidden.has(key) && bx < C::kBoxes; ++bx)
                                        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(chunk + bx * C::kBoxBytes + key * 128), "r"(0) : "memory");
                                fence_proxy_async();
                                __syncwarp();
                            }
                        }
                        if (j == 0 && !mbar_wait_uniform(&bars->o_empty[g], it ^ 1, ctx, kWaitPagedFwd + 7)) { ok = false; break; }
                        const uint32_t at_x = desc_lo_mn_major(aKV + (x % C::kRing) * C::kTileBytes, C::kBoxBytes);
                        const uint32_t at_g = tmem_base + C::kColP + g * 64, acc = tmem_base + C::kColO + g * HD;
                        if (!mbar_wait_uniform(&bars->p_full[g], st, ctx, kWaitPagedFwd + 8)) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int kk = 0; kk < 6; ++kk) mma_ts(acc, at_g + kk * 8, at_x + kk * kDescStepMn, idesc_o, (j > 0) || (kk > 0));
                        }
                        __syncwarp();
                        if (!mbar_wait_uniform(&bars->p_rest[g], st, ctx, kWaitPagedFwd + 9)) { ok = false; break; }
                        tc_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int kk = 6; kk < 8; ++kk) mma_ts(acc, at_g + kk * 8, at_x + kk * kDescStepMn, idesc_o, 1);
                            mma_commit(&bars->p_empty[g]);
                            if (last_use) mma_commit(&bars->kv_empty[x % C::kRing]);
                            if (j == n - 1) mma_commit(&bars->o_full[g]);
                        }
                        __syncwarp();
                    }
                    if (g) ++n_st[1], n_it[1] += j == n - 1;
                    else ++n_st[0], n_it[0] += j == n - 1;
                }
                kv += 2 * n1;
            }
            // MMAs already issued must finish before tensor memory is released
            if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&bars->abort_flag) != 0)) {
                if (elect_one()) {
                    mma_commit(&bars->drain[is_s]);
                    mbar_wait_drain(&bars->drain[is_s], 0);
                }
            }
            __syncwarp();
        }
    } else if (warp >= 8) {
        // =========================== read-out, codes to fp16 ==========================================
        setmaxnreg_dec<C::kRegsReadOut>();
        const int quad = warp & 3;
        const int row = quad * 32 + lane;
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
        uint32_t n_o[2] = {0, 0};
        auto lds = [](uint32_t at, uint32_t (&x)[4]) {
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at));
        };
        auto sts = [](uint32_t at, uint32_t x, uint32_t y, uint32_t z, uint32_t u) {
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(u) : "memory");
        };
        auto read_out = [&](int k, const PagedItem& w) -> bool {
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
                if (w.tokens_of(t) == 0) continue;
                const int g = group_of_tile(k, t);
                const uint32_t n_done = g ? n_o[1]++ : n_o[0]++;
                if (!mbar_wait_uniform(&bars->stat_full[g], n_done & 1, ctx, kWaitPagedFwd + 12) ||
                    !mbar_wait_uniform(&bars->o_full[g], n_done & 1, ctx, kWaitPagedFwd + 13))
                    return false;
                tc_fence_after();
                const float inv_l = sStat[g * kTile + row];  // (of a piece: 1, or the unit of O)
                mbar_arrive_warp(&bars->stat_empty[g]);
                const int token = row >> p.pack_log2, head = (w.group << p.pack_log2) + (row & ((1 << p.pack_log2) - 1));
                const bool valid = token < w.tokens_of(t);  // the others are rows of another sequence, or of none
                const long long at = w.row_of(t) + token;
                uint4* dst = reinterpret_cast<uint4*>(a.o + (at * a.H + head) * HD);
                float4* partial = reinterpret_cast<float4*>(piece_result<HD>(p, w.piece, t)) + row;
#pragma unroll 1
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t r[32];
                    tmem_ld_32x32(t_row + C::kColO + g * HD + c * 32, r);
                    tmem_wait_ld();
                    if (w.piece >= 0) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            partial[(8 * c + e) * kTile] = make_float4(__uint_as_float(r[4 * e]) * inv_l, __uint_as_float(r[4 * e + 1]) * inv_l,
                                                                       __uint_as_float(r[4 * e + 2]) * inv_l, __uint_as_float(r[4 * e + 3]) * inv_l);
                        continue;
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint4 pk;
                        pk.x = pack_bf16(__uint_as_float(r[8 * e + 0]) * inv_l, __uint_as_float(r[8 * e + 1]) * inv_l);
                        pk.y = pack_bf16(__uint_as_float(r[8 * e + 2]) * inv_l, __uint_as_float(r[8 * e + 3]) * inv_l);
                        pk.z = pack_bf16(__uint_as_float(r[8 * e + 4]) * inv_l, __uint_as_float(r[8 * e + 5]) * inv_l);
                        pk.w = pack_bf16(__uint_as_float(r[8 * e + 6]) * inv_l, __uint_as_float(r[8 * e + 7]) * inv_l);
                        if (valid) dst[4 * c + e] = pk;
                    }
                }
                tc_fence_before();
                mbar_arrive_warp(&bars->o_empty[g]);
            }
            return true;
        };
        if constexpr (!kE4M3) {
            for (int k = 0;; ++k) {
                PagedItem w;
                if (!next_item(k, kWaitPagedFwd + 11, &w)) break;
                if (!read_out(k, w)) break;
            }
        } else {
            // Q of a tile, one row a thread, in place.
            uint32_t n_q[2] = {0, 0};
            auto convert_q = [&](int g) -> bool {
                const uint32_t n = g ? n_q[1]++ : n_q[0]++;
                if (!mbar_wait_uniform(&bars->q_full[g], n & 1, ctx, kWaitPagedFwd + 20)) return false;
                const uint32_t at = smem_u32(sQ + g * C::kTileBytes) + row * 128;
                uint32_t most = 0;
#pragma unroll 4
                for (int c = 0; c < HD / 8; ++c) {
                    uint32_t x[4];
                    lds(at + (c >> 3) * C::kBoxBytes + (((c ^ row) & 7) << 4), x);
#pragma unroll
                    for (int y = 0; y < 4; ++y) most = max(most, max(x[y] & 0x7fffu, x[y] >> 16 & 0x7fffu));
                }
                int up = most >= 0x7f80u || most == 0 ? 0 : 127 + 14 - static_cast<int>(most >> 7);  // (a row that is not finite stays so)
                up = up > 112 ? 112 : up;  // (2^-133, the least bf16 number, is still one of fp16 then)
                const float f = power_of_two(up);
#pragma unroll 4
                for (int c = 0; c < HD / 8; ++c) {
                    uint32_t x[4];
                    const uint32_t chunk = at + (c >> 3) * C::kBoxBytes + (((c ^ row) & 7) << 4);
                    lds(chunk, x);
#pragma unroll
                    for (int y = 0; y < 4; ++y) x[y] = pack_f16(bf16_low(x[y]) * f, bf16_high(x[y]) * f);
                    sts(chunk, x[0], x[1], x[2], x[3]);
                }
                sQExp[(2 * g + (n & 1)) * kTile + row] = static_cast<int8_t>(up);
                fence_proxy_async();
                mbar_arrive_warp(&bars->q_ready[g]);
                return true;
            };
            // The tiles of an item, and between its first ones its Q and the read-out of the item before: those tiles need no room that
            // the read-out has to make first (the ring's), and what comes behind them would have to wait for products anyway.
            // Eight lanes at a time read 128 bytes that lie in all banks and write 16-byte chunks that do: half of a row and the other half of the
            // next (or, of 64 columns, two rows).  In K's tile the rows are those of key_of_column().
            const int to_row = HD == 128 ? 2 * (lane >> 4) + ((lane >> 2) & 1) : lane >> 2;  // of a warp's first turn
            const int part = HD == 128 ? (lane & 3) | (((lane >> 2) ^ (lane >> 3)) & 1) << 2 : lane & 3;
            const int chunk0 = (2 * (part & 3)) ^ (to_row & 7);
            uint32_t kv = 0;
            bool ok = true;
            PagedItem before;
            before.b = -1;
            for (int k = 0; ok; ++k) {
                PagedItem w;
                const bool more = next_item(k, kWaitPagedFwd + 11, &w);
                const int front = kWindow ? w.hidden(0, window, a.sinks).to : 0;
                const int tiles = more ? 2 * w.n[1] : 0, pause = tiles < C::kRing - 1 ? tiles : C::kRing - 1;
                for (int x = 0; ok && x <= tiles; ++x) {
                    if (x == pause) {
                        if (more) ok = convert_q(group_of_tile(k, 1)) && (w.n[0] == 0 || convert_q(group_of_tile(k, 0)));
                        if (ok && before.b >= 0) ok = read_out(k - 1, before);
                    }
                    if (!ok || x == tiles) break;
                    const TileOfItem tile(x, w.n[1]);
                    const uint32_t at = w.kv0 + 2 * tile.j + tile.is_v;  // ring position
                    const int raw = kv % C::kRawRing, st = at % C::kRing;
                    if (!mbar_wait_uniform(&bars->raw_full[raw], (kv / C::kRawRing) & 1, ctx, kWaitPagedFwd + 18) ||
                        !mbar_wait_uniform(&bars->kv_empty[st], ((at / C::kRing) & 1) ^ 1, ctx, kWaitPagedFwd + 19)) {
                        ok = false;
                        break;
                    }
                    const bool is_v = tile.is_v;
                    // only the last tile and those that begin in front of the window can have rows that are not attended
                    const bool edge = tile.j == w.n[1] - 1 || (kWindow && w.key_tile(tile.j) * kTile < front);
                    const uint32_t src = smem_u32(sRaw + raw * C::kRawBytes), dst = smem_u32(sKV + st * C::kTileBytes);
                    // the largest exponent of the rows that are attended: four rows a lane
                    uint32_t four = *reinterpret_cast<const volatile uint32_t*>(&bars->exps[raw][4 * lane]);
                    if (edge) {
                        const HiddenKeys hidden = w.hidden(w.key_tile(tile.j) * kTile, window, a.sinks);
#pragma unroll 1  // (rarely run, and beside the softmax code costs: 2048 new of 8192 tokens on 32 heads of 64 234 us when written out, 228 so)
                        for (int y = 0; y < 4; ++y)
                            if (hidden.has(4 * lane + y)) four = (four & ~(0xffu << (8 * y))) | 0x80u << (8 * y);  // kExpNotFinite
                    }
                    int most = kExpNotFinite;
#pragma unroll
                    for (int y = 0; y < 4; ++y) most = max(most, static_cast<int>(static_cast<int8_t>(four >> (8 * y))));
                    // (of V no less than 2^-100: O's unit, 2^13 below it and divided by the sum of weights, is a number of fp32 then)
                    most = max(__reduce_max_sync(0xffffffffu, most), is_v ? -100 : kExpLeast);
                    // A warp takes 32 rows, kRows at a time, 16 codes a lane.  Lane i has the factor of the warp's row i.
                    const int e = bars->exps[raw][32 * quad + lane];
                    const float f = e == kExpNotFinite ? __uint_as_float(0x7fffffffu) : power_of_two(max(e - most + 6, -127));
                    const uint32_t factors = pack_f16(f, f);
                    constexpr int kRows = 512 / HD;
                    const int src_row = is_v ? to_row : key_of_column(to_row);
                    uint32_t from = src + (32 * quad + src_row) * HD + part * 16, to = dst + (part >> 2) * C::kBoxBytes + (32 * quad + to_row) * 128;
                    // (one short loop: written out, the code that the softmax warps run beside costs more than its branches, 2140 against 2095 us
                    // for 2048 new tokens of 32k on 64 heads over 8)
#pragma unroll 1
                    for (int i0 = 0; i0 < 32 / kRows; i0 += 2) {
                        uint32_t codes[2][4];
#pragma unroll
                        for (int i = 0; i < 2; ++i) lds(from + i * kRows * HD, codes[i]);
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t ff = __shfl_sync(0xffffffffu, factors, src_row + (i0 + i) * kRows);
                            uint32_t out[8];
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                e4m3_to_f16(codes[i][y], out[2 * y], out[2 * y + 1]);
                                out[2 * y] = f16x2_mul(out[2 * y], ff), out[2 * y + 1] = f16x2_mul(out[2 * y + 1], ff);
                            }
                            // chunks 2 part and 2 part + 1 of the row, swizzled as a TMA box would be
                            const uint32_t chunk = to + i * kRows * 128 + ((HD == 128 && i == 1 ? chunk0 ^ 4 : chunk0) << 4);
                            sts(chunk, out[0], out[1], out[2], out[3]);
                            sts(chunk ^ 16, out[4], out[5], out[6], out[7]);
                        }
                        from += 2 * kRows * HD, to += 2 * kRows * 128;
                    }
                    if (is_v && edge) {
                        const HiddenKeys hidden = w.hidden(w.key_tile(tile.j) * kTile, window, a.sinks);
                        // rows that are not attended: whatever lies there (a weight of zero does not make a NaN go away)
                        __syncwarp();
#pragma unroll 1
                        for (int key = 32 * quad + (lane >> 3); key < 32 * quad + 32; key += 4)
                            for (int bx = 0; hidden.has(key) && bx < C::kBoxes; ++bx) sts(dst + bx * C::kBoxBytes + key * 128 + (lane & 7) * 16, 0, 0, 0, 0);
                    }
                    if (threadIdx.x == 256) bars->tile_exp[at % 16] = static_cast<int8_t>(most);
                    fence_proxy_async();
                    mbar_arrive_warp(&bars->kv_full[st]);
                    mbar_arrive_warp(&bars->raw_empty[raw]);
                    ++kv;
                }
                if (!more) break;
                before = w;
            }
        }
    } else {
        // =========================== softmax =========================================================
        setmaxnreg_inc<C::kRegsSoftmax>();
        const int group = HD == 128 ? __shfl_sync(0xffffffffu, warp >> 2, 0) : warp >> 2;
        const int quad = warp & 3;             // tensor-memory lane quadrant this warp may access
        const int row = quad * 32 + lane;
        const uint32_t t_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
        const uint32_t tS = t_row + C::kColS + (C::kScoreBufs == 1 ? 0 : group * kTile), tP = t_row + C::kColP + group * 64;
        uint32_t n_s = 0, n_it = 0;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            if (!mbar_wait_uniform(&bars->list_full[group][k % C::kSched], (k / C::kSched) & 1, ctx, kWaitPagedFwd + 14)) break;
            const int slot = bars->list_slot[group][k % C::kSched];
            const PagedItem w = bars->item[slot];
            if (w.b < 0) break;
            const int tile = tile_of_group(slot, group), n = tile ? w.n[1] : w.n[0];
            const int first_pos = w.first_pos(tile), last_pos = first_pos + w.tokens_of(tile) - 1;
            const int pos = first_pos + (row >> p.pack_log2);
            float m_used = 0.f;   // running maximum in use; times c2_part it is in log2 units
            float l[2] = {0.f, 0.f};
            // A product is multiplied with c2 = c2_power * c2_part, a power of two and 1 <= c2_part < 2.  The maximum goes with the power alone, which
            // rounds nothing.
            float c2 = a.scale_log2, c2_power = a.scale_power;
            const float c2_part = a.scale_part;
            int c2_exp = 0;          // 8 bits: the exponent field of c2 for a tile of K whose power is 2^0
            float delta = 0.f;       // 8 bits: r less the maximum.  (r itself, near 2^24, would lose V's power.)
            for (int j = 0; j < n; ++j, ++n_s) {
                const int key0 = w.key_tile(j) * kTile;
                if (!mbar_wait_uniform(&bars->s_full[group], n_s & 1, ctx, kWaitPagedFwd + 15)) { ok = false; break; }
                tc_fence_after();
                if constexpr (kE4M3) {
                    // c2 = scale * 2^(K's exponent - 6 - that of the row of Q), K being 2^6 as large, held to the normal numbers: scores are multiplied with it,
                    // masked ones (-inf) and zeros too, so it must neither vanish nor become infinite.  Products are below 2^38: held from below, scores
                    // are below 2^-88.
                    if (j == 0) c2_exp = a.scale_field - 6 - sQExp[(2 * group + (n_it & 1)) * kTile + row];
                    const int e = min(max(c2_exp + bars->tile_exp[(w.kv0 + 2 * j) % 16], 1), 254);
                    c2_power = __uint_as_float(static_cast<uint32_t>(e) << 23);
                    c2 = c2_power * c2_part;
                }
                uint32_t s[4][32];
                tmem_ld_32x32(tS, s[0]);
                tmem_ld_32x32(tS + 32, s[1]);
                tmem_ld_32x32(tS + 64, s[2]);
                tmem_ld_32x32(tS + 96, s[3]);
                tmem_wait_ld();
                tc_fence_before();
                mbar_arrive_warp(&bars->s_empty[C::kScoreBufs == 1 ? 0 : group]);
                // (as bits of the columns: comparing positions for every score costs the steps that need no mask, whose code lies around it,
                // as well: 4096 new tokens with a window of 8192 on 40 heads 752 us instead of 669, 2048 of 8192 on 32 237 instead of 235)
                if (!all_attend(first_pos, last_pos, key0, kTile, window, a.sinks)) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint32_t keys = attended(pos, key0 + 32 * c, window, a.sinks);
                        const uint32_t columns = (keys & 0x99999999u) | (keys & 0x22222222u) << 1 | (keys & 0x44444444u) >> 1;  // see key_of_column()
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if ((columns >> e & 1) == 0) s[c][e] = 0xff800000u;  // -inf
                    }
                }
                float mx4[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx4[c] = fmaxf(__uint_as_float(s[c][0]), __uint_as_float(s[c][1]));
#pragma unroll
                    for (int e = 2; e < 32; e += 2) mx4[c] = fmax3(mx4[c], __uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1]));
                }
                const float m_new = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3])) * c2_power;
                // the P.V product of this tile's step before is done: P and O may be written
                if (n_s > 0 && !mbar_wait_uniform(&bars->p_empty[group], (n_s - 1) & 1, ctx, kWaitPagedFwd + 17)) { ok = false; break; }
                tc_fence_after();
                float v_exp = 0.f;  // 8 bits: the tile's of V
                if constexpr (kE4M3) {
                    // (V of this step has been written by now, or is about to be)
                    const uint32_t x = w.kv0 + 2 * j + 1;
                    if (!mbar_wait_uniform(&bars->kv_full[x % C::kRing], (x / C::kRing) & 1, ctx, kWaitPagedFwd + 21)) { ok = false; break; }
                    v_exp = static_cast<float>(bars->tile_exp[x % 16]);
                }
                if (j == 0) {
                    m_used = fmaxf(m_new, kLeast);  // (a row can have no key in the first tile of a window)
                    delta = v_exp;
                } else {
                    const float up_m = (m_new - m_used) * c2_part;
                    const bool need = up_m > kLazyRescale, need_o = kE4M3 ? up_m + v_exp - delta > kLazyRescale : need;
                    if (__any_sync(0xffffffffu, need || need_o)) {
                        const float alpha_l = need ? fast_exp2(-up_m) : 1.0f;
                        const float alpha = kE4M3 ? (need_o ? fast_exp2(delta - (up_m + v_exp)) : 1.0f) : alpha_l;
                        l[0] *= alpha_l, l[1] *= alpha_l;
#pragma unroll 1
                        for (int c = 0; c < HD / 16; ++c) {
                            uint32_t o[16];
                            const uint32_t t_o = t_row + C::kColO + group * HD + c * 16;
                            tmem_ld_32x16(t_o, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            tmem_st_32x16(t_o, o);
                        }
                        if (need) m_used = m_new;
                        if (need_o) delta = need ? v_exp : up_m + v_exp;
                        else if (need) delta -= up_m;
                    }
                }
                // Exponents of the weights are x - m + shift.  (Below 2^-45 a weight is none in fp16; the sum still wants the weights.)
                const float shift = kE4M3 ? 7.f + fmaxf(v_exp - delta, -60.f) : 0.f;
                const float tile_up = kE4M3 ? fast_exp2(-shift) : 1.f;  // of the sums of the tile's weights
                // Far from zero the product, which the fused multiply-add has in full, is off the rounded maximum by more than the weights' type takes
                // (fp16 2^16, bf16 2^128).  There fp32 holds scores that are as far apart, or equal: the power alone, with which the maximum is exact,
                // gives them weights of nothing, or 1.
                const bool far = fabsf(m_used) >= (kE4M3 ? 0x1p22f : 0x1p29f);
                const float by = far ? c2_power : c2, neg_m = fmaf(-m_used, far ? 1.f : c2_part, shift);
                const uint64_t c2x2 = f2_pack(by, by), nm = f2_pack(neg_m, neg_m);
                uint64_t sum[2];  // of a half of the tile: chains 0 and 1, chains 2 and 3 (see key_of_column in fwd_kernel.cu)
                auto add_chunk = [&](int c) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        auto weight = [&](int x) { return __uint_as_float(s[c][4 * e + x]); };
                        const uint64_t pairs = f2_add(f2_pack(weight(0), weight(1)), f2_pack(weight(2), weight(3)));
                        sum[e & 1] = (c & 1) == 0 && e < 2 ? pairs : f2_add(sum[e & 1], pairs);
                    }
                    if (c & 1) {
                        float a0, a1, b0, b1;
                        f2_unpack(sum[0], a0, a1);
                        f2_unpack(sum[1], b0, b1);
                        if constexpr (kE4M3) l[c >> 1] = fmaf((a0 + a1) + (b0 + b1), tile_up, l[c >> 1]);
                        else l[c >> 1] += (a0 + a1) + (b0 + b1);
                    }
                };
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float p0, p1, p2, p3;  // weights of the keys 4 e to 4 e + 3
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(s[c][4 * e]), __uint_as_float(s[c][4 * e + 1])), c2x2, nm), p0, p2);
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(s[c][4 * e + 2]), __uint_as_float(s[c][4 * e + 3])), c2x2, nm), p1, p3);
                        p0 = fast_exp2(p0), p1 = fast_exp2(p1), p2 = fast_exp2(p2), p3 = fast_exp2(p3);
                        s[c][4 * e] = __float_as_uint(p0), s[c][4 * e + 1] = __float_as_uint(p2);
                        s[c][4 * e + 2] = __float_as_uint(p1), s[c][4 * e + 3] = __float_as_uint(p3);
                        pk[2 * e] = kE4M3 ? pack_f16(p0, p1) : pack_bf16(p0, p1), pk[2 * e + 1] = kE4M3 ? pack_f16(p2, p3) : pack_bf16(p2, p3);
                    }
                    tmem_st_32x16(tP + c * 16, pk);
                    if (c >= 2) {
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive_warp(c == 2 ? &bars->p_full[group] : &bars->p_rest[group]);
                    }
                    if (c > 0) add_chunk(c - 1);
                    if (c == 3) add_chunk(3);
                }
            }
            if (!ok || !mbar_wait_uniform(&bars->stat_empty[group], (n_it & 1) ^ 1, ctx, kWaitPagedFwd + 16)) break;
            ++n_it;
            const float sum_l = l[0] + l[1];
            const float unit = kE4M3 ? fast_exp2(delta - 13.f) : 1.0f;  // (V is 2^6 and the weights are 2^7 as large)
            sStat[group * kTile + row] = w.piece >= 0 ? unit : unit / sum_l;
            mbar_arrive_warp(&bars->stat_full[group]);
            if (w.piece >= 0) {
                float* stats = piece_result<HD>(p, w.piece, tile) + kTile * HD;
                stats[row] = fmaxf(m_used * c2_part, kLeast), stats[kTile + row] = sum_l;
                continue;
            }
            const int token = row >> p.pack_log2, head = (w.group << p.pack_log2) + (row & ((1 << p.pack_log2) - 1));
            if (token < w.tokens_of(tile))  // natural-log sum-exp of the scaled scores
                a.lse[static_cast<long long>(head) * a.batch.T + w.row_of(tile) + token] = fmaf(m_used, c2_part, log2f(sum_l)) * 0.6931471805599453f;
        }
    }

    // ---- teardown ------------------------------------------------------------------------------
    if (p.beside) wait_for_predecessor();  // whoever waits for this kernel waits for that one too
    tc_fence_before();
    __syncthreads();
    if (warp == 13) {
        tc_fence_after();
        tmem_dealloc(tmem_base, C::kTmemCols);
    }
}

// Joins the pieces of the split items.  A thread has eight columns of a row, a block 16 columns of a tile: with a block for each tile the few
// items that are split left most of the GPU idle here (32k keys, 32 rows of 8 KV heads, both kernels: 108 us and 48).
template <int HD>
struct JoinCfg {
    static constexpr int kThreads = 256;
    static constexpr int kBlocks = kTile * (HD / 8) / kThreads;  // for each tile
};
template <int HD>
__global__ void __launch_bounds__(JoinCfg<HD>::kThreads) s2a_paged_join_kernel(const __grid_constant__ PagedTileParams p) {
    const PagedFwdParams& a = p.a;
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(a.status) != 0) return;
    PagedItem w;
    const int tile = static_cast<int>(blockIdx.x) / JoinCfg<HD>::kBlocks, x = tile >> 1, t = tile & 1;
    Ranking ranking;
    if (p.ranked) ranking.set(p);  // (every warp for itself)
    if (!any_item(p, ranking, p.first_split + x, &w)) return;
    const int tiles = piece_tiles(p, w), n = t ? w.n[1] : w.n[0], pieces = (n + tiles - 1) / tiles;
    if (pieces == 0) return;
    const int i = static_cast<int>(blockIdx.x) % JoinCfg<HD>::kBlocks * JoinCfg<HD>::kThreads + static_cast<int>(threadIdx.x);
    const int row = i % kTile, c = i / kTile;
    const int token = row >> p.pack_log2, head = (w.group << p.pack_log2) + (row & ((1 << p.pack_log2) - 1));
    if (token >= w.tokens_of(t)) return;
    float m = kLeast;
#pragma unroll 4
    for (int y = 0; y < pieces; ++y) m = fmaxf(m, __ldcg(piece_result<HD>(p, x * p.split + y, t) + kTile * HD + row));
    float l = 0.f, o[8] = {};
#pragma unroll 4
    for (int y = 0; y < pieces; ++y) {
        const float* from = piece_result<HD>(p, x * p.split + y, t);
        const float f = fast_exp2(__ldcg(from + kTile * HD + row) - m);
        l = fmaf(__ldcg(from + kTile * HD + kTile + row), f, l);
        const float4 u = __ldcg(reinterpret_cast<const float4*>(from) + 2 * c * kTile + row), v = __ldcg(reinterpret_cast<const float4*>(from) + (2 * c + 1) * kTile + row);
        o[0] = fmaf(u.x, f, o[0]), o[1] = fmaf(u.y, f, o[1]), o[2] = fmaf(u.z, f, o[2]), o[3] = fmaf(u.w, f, o[3]);
        o[4] = fmaf(v.x, f, o[4]), o[5] = fmaf(v.y, f, o[5]), o[6] = fmaf(v.z, f, o[6]), o[7] = fmaf(v.w, f, o[7]);
    }
    const float inv_l = 1.0f / l;
    const long long at = w.row_of(t) + token;
    uint4 pk;
    pk.x = pack_bf16(o[0] * inv_l, o[1] * inv_l), pk.y = pack_bf16(o[2] * inv_l, o[3] * inv_l);
    pk.z = pack_bf16(o[4] * inv_l, o[5] * inv_l), pk.w = pack_bf16(o[6] * inv_l, o[7] * inv_l);
    reinterpret_cast<uint4*>(a.o + (at * a.H + head) * HD)[c] = pk;
    if (c == 0) a.lse[static_cast<long long>(head) * a.batch.T + at] = (m + log2f(l)) * 0.6931471805599453f;
}

template <int HD, bool kE4M3, bool kWindow>
cudaError_t configure_form() {
    using C = PagedCfg<HD, kE4M3>;
    // the register split of the kernel draws on what a block is launched with
    cudaFuncAttributes attributes;
    cudaError_t e = cudaFuncGetAttributes(&attributes, s2a_paged_fwd_kernel<HD, kE4M3, kWindow>);
    if (e != cudaSuccess) return e;
    if (attributes.numRegs < C::kRegsLaunch || attributes.sharedSizeBytes != 0) return cudaErrorInvalidConfiguration;
    return cudaFuncSetAttribute(s2a_paged_fwd_kernel<HD, kE4M3, kWindow>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
}
template <int HD, bool kE4M3>
cudaError_t configure_one() {
    const cudaError_t e = configure_form<HD, kE4M3, false>();
    return e != cudaSuccess ? e : configure_form<HD, kE4M3, true>();
}

}  // namespace

cudaError_t configure_paged_fwd() {
    for (const cudaError_t e : {configure_one<64, false>(), configure_one<64, true>(), configure_one<128, false>(), configure_one<128, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

template <int HD, bool kE4M3>
static cudaError_t launch_one(const PagedTileParams& p, cudaStream_t stream) {
    const int items = p.slots * (p.a.H >> p.pack_log2), split_items = items - p.first_split;
    const unsigned grid = static_cast<unsigned>(p.first_split) + static_cast<unsigned>(split_items) * static_cast<unsigned>(p.split);
    const auto kernel = p.a.window > 0 ? s2a_paged_fwd_kernel<HD, kE4M3, true> : s2a_paged_fwd_kernel<HD, kE4M3, false>;
    const cudaError_t e = launch_kernel(kernel, grid, PagedCfg<HD, kE4M3>::kThreads, PagedCfg<HD, kE4M3>::kSmemBytes, stream, p, true);
    if (e != cudaSuccess || split_items == 0) return e;
    return launch_kernel(s2a_paged_join_kernel<HD>, 2u * JoinCfg<HD>::kBlocks * static_cast<unsigned>(split_items), JoinCfg<HD>::kThreads, 0, stream, p, true);
}

cudaError_t launch_paged_fwd(const PagedTileParams& p, bool e4m3, int d, cudaStream_t stream) {
    if (d == 64) return e4m3 ? launch_one<64, true>(p, stream) : launch_one<64, false>(p, stream);
    return e4m3 ? launch_one<128, true>(p, stream) : launch_one<128, false>(p, stream);
}

size_t paged_piece_bytes(int d) { return sizeof(float) * 2 * kTile * (d + 2); }

}  // namespace s2a
