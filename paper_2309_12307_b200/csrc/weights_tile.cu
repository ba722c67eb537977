// What attention weight cached tokens get from many rows (pieces of prompts): see weights_kernels.cu for the formula.
//
// S^T = K Q^T on tcgen05, 128 keys by 128 rows of q at a time.  A score tile has a key in each lane of tensor memory and a row of q in each column, so
// the thread that has a key adds up its columns' exponentials in registers: nothing crosses threads, and there is no second product.
// An item is two key tiles of a sequence and KV head, which stay while the row tiles that attend any of them (128 rows, as s2a_paged_fwd_kernel's: query heads
// of a KV head and neighbouring tokens, one TMA box) pass by.  Two key tiles, because a row tile is 32 KB from the L2 that would otherwise be read twice
// as often.  (Where it attends only one of them, the other's scores are made and not looked at.)
//
// The keys are the products' operand in tensor memory (8-bit codes as bf16, what they stand for exactly): read from shared memory for every product beside
// the rows they took its whole bandwidth.
//
// One persistent block per SM:
//   warps 0-15      exponentials and sums: four warps for either key tile and either half of a row tile's columns
//   warps 16-19     an item's keys to tensor memory, from shared memory, where they have come while the item before was worked on
//   warp 20         work items (cluster launch control), TMA loads of keys and of q
//   warp 21         tcgen05 MMAs
//   warp 22         the rows' log sums
// Tensor memory: the keys, then three score tiles, which the products of the two key tiles fill in turn: they are ahead of the exponentials, so that what
// a warp does between two of its tiles, and the change of keys between items, finds others at work.  (A warp that waits for a use of a score tile must
// know that the use before, three score tiles ago, is over: it has worked on the one two score tiles ago.  Score tiles of 64 rows, twice as many, took the
// products 1630 cycles a row tile, these 1130.)
//
// Bound by the exp2 unit.  2048 rows of 8192 keys on 32 heads of 128 take 150 us.  Counted in a cold launch of 155 us at 1.67 GHz it was busy 81 % of the
// clocks in which a multiprocessor had a block, 77 % of all: 474 million exponentials (of score tiles that some row attends), 16 a clock, take it 120 us by
// themselves, and the products take 58.  Between score tiles all warps of a multiprocessor's quarter wait at times.  A polynomial for some of the
// exponentials brought nothing, at any share, nor did warps that take whole score tiles in turn.
//
// Where there are few items their rows are split into pieces, whose sums a second kernel adds up in order.
#include <cuda_fp16.h>

#include <type_traits>

#include "evict.h"
#include "paged_device.cuh"

namespace s2a {

namespace {

template <int HD, bool kE4M3>
struct TileCfg {
    static constexpr int kThreads = 768;
    static constexpr int kBoxes = HD / 64;                 // 64-column boxes per row tile
    static constexpr int kBoxBytes = kTile * 128;          // 128 rows x 128 bytes
    static constexpr int kTileBytes = kBoxes * kBoxBytes;
    static constexpr int kRing = 4 * 128 / HD;             // row tiles in flight, and their log sums
    static constexpr int kKeyBytes = HD * (kE4M3 ? 1 : 2), kLine = kKeyBytes < 128 ? kKeyBytes : 128;  // of a key in the cache, and of a box of them
    static constexpr int kKeysBytes = kWeightKeys * kKeyBytes, kExpBytes = kE4M3 ? kWeightKeys : 0;
    static constexpr int kSched = 3;                       // items in flight
    static constexpr int kBarBytes = 1024, kSumBytes = 2 * kTile * 4;
    static constexpr int kSmemBytes = kKeysBytes + kRing * (kTileBytes + kTile * 4) + kSumBytes + kExpBytes + kBarBytes;
    static_assert(kSmemBytes <= 232448 && 2 * kSmemBytes > 232448, "shared memory: one block on an SM, since it takes all tensor memory");
    static constexpr int kTmemCols = 512, kKeyCols = HD / 2;  // columns of a key tile
    static constexpr int kHalf = 64, kScores = 3, kColS = 2 * kKeyCols;
    static_assert(kColS + kScores * kTile <= kTmemCols, "tensor memory");
};

template <int HD, bool kE4M3>
struct TileBars {
    using C = TileCfg<HD, kE4M3>;
    uint64_t loaded, taken;    // keys in shared memory
    uint64_t k_full[2], k_empty;  // in tensor memory
    uint64_t q_full[C::kRing], q_empty[C::kRing];
    uint64_t l_full[C::kRing], l_empty[C::kRing];
    uint64_t s_full[C::kScores], s_empty[C::kScores];
    uint64_t sched_full[C::kSched], sched_empty[C::kSched];
    uint64_t sum_full[2], sum_empty[2];
    uint64_t clc, drain;
    alignas(16) uint8_t clc_resp[16];
    WeightsItem item[C::kSched];
    uint32_t tmem_slot;
    int abort_flag;
};

// The row tiles of an item in turn: head group and first position of each.
struct RowTiles {
    int group, first_pos;
    __device__ __forceinline__ RowTiles(const WeightsTileParams& p, const WeightsItem& w, int tokens_log2)
        : first_pos(w.first + ((w.t_lo + p.by_groups(w.r0, &group)) << tokens_log2)) {}
    __device__ __forceinline__ void next(int groups, int tokens_log2) {
        if (++group == groups) group = 0, first_pos += 1 << tokens_log2;
    }
};

// The score tiles in turn: which it is, and the parity of its use.
struct ScoreTiles {
    uint32_t n = 0;  // modulo 6
    __device__ __forceinline__ uint32_t tile(int ahead) const { return (n + ahead) % 3; }
    __device__ __forceinline__ uint32_t use(int ahead) const { return (n + ahead) / 3 & 1; }
    __device__ __forceinline__ void next_row_tile() { n = n == 4 ? 0 : n + 2; }
};

// Whether any of the tokens from position first_pos to end_pos attends a key of the tile that begins with key_low.
template <bool kWindow>
__device__ __forceinline__ bool tile_attended(const WeightsParams& a, int last, int first_pos, int end_pos, int key_low) {
    return key_low <= min(end_pos, last) && (!kWindow || key_low + (kTile - 1) > first_pos - a.window || key_low < a.sinks);
}

// kWindow: whether the call has one.
template <int HD, bool kE4M3, bool kWindow>
__global__ void __launch_bounds__(TileCfg<HD, kE4M3>::kThreads, 1) s2a_weights_tile_kernel(const __grid_constant__ WeightsTileParams p) {
    using C = TileCfg<HD, kE4M3>;
    using Bars = TileBars<HD, kE4M3>;
    static_assert(sizeof(Bars) <= C::kBarBytes, "barrier block");
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sK = smem;                                                      // keys of the next item, as the cache has them
    uint8_t* sQ = sK + C::kKeysBytes;                                        // ring of row tiles
    float* sLse = reinterpret_cast<float*>(sQ + C::kRing * C::kTileBytes);   // ring of -lse / ln 2, -inf for rows that are not there
    float* sSum = sLse + C::kRing * kTile;                                   // [key tile][128]: what the second half of the columns gave
    int8_t* sExp = reinterpret_cast<int8_t*>(sSum) + C::kSumBytes;           // and their exponents
    Bars* bars = reinterpret_cast<Bars*>(sExp + C::kExpBytes);
    const WeightsParams& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kConsumers = 16 + 4 + 2;  // warps that read items

    if (threadIdx.x == 0) {
        for (int x = 0; x < 2; ++x) {
            mbar_init(&bars->k_full[x], 4);
            mbar_init(&bars->sum_full[x], 4);
            mbar_init(&bars->sum_empty[x], 4);
        }
        mbar_init(&bars->k_empty, 1);
        mbar_init(&bars->loaded, 1);
        mbar_init(&bars->taken, 4);
        for (int x = 0; x < C::kRing; ++x) {
            mbar_init(&bars->q_full[x], 1);
            mbar_init(&bars->q_empty[x], 1);
            mbar_init(&bars->l_full[x], 1);
            mbar_init(&bars->l_empty[x], 16);
        }
        for (int x = 0; x < C::kScores; ++x) mbar_init(&bars->s_full[x], 1), mbar_init(&bars->s_empty[x], 8);
        for (int x = 0; x < C::kSched; ++x) mbar_init(&bars->sched_full[x], 1), mbar_init(&bars->sched_empty[x], kConsumers);
        mbar_init(&bars->clc, 1);
        mbar_init(&bars->drain, 1);
        fence_barrier_init();
        tma_prefetch_desc(&p.tm_q);
        tma_prefetch_desc(&p.tm_k);
    }
    if (warp == 21) {
        tmem_alloc(&bars->tmem_slot, C::kTmemCols);
        tmem_relinquish();
    }
    wait_for_predecessor();
    // An earlier report (a wait that expired, a value out of range) leaves the status word set: nothing is done then.
    if (threadIdx.x == 0) bars->abort_flag = *reinterpret_cast<volatile int*>(a.status);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    release_successor();
    const uint32_t tmem_base = bars->tmem_slot;
    if (bars->abort_flag != 0) {
        if (warp == 21) tmem_dealloc(tmem_base, C::kTmemCols);
        return;
    }
    if (blockIdx.x == 0) check_batch(a.batch, a.pool.page_log2, a.most_new, a.status, a.host_status);
    const WaitCtx ctx{&bars->abort_flag, a.status, a.host_status};
    const int tokens_log2 = 7 - p.pack_log2, groups = a.rep >> p.pack_log2;

    auto next_item = [&](int k, int where, WeightsItem* w) -> bool {
        const int slot = k % C::kSched;
        if (!mbar_wait_uniform(&bars->sched_full[slot], (k / C::kSched) & 1, ctx, where)) return false;
        *w = bars->item[slot];
        mbar_arrive_warp(&bars->sched_empty[slot]);
        return w->b >= 0;
    };
    // Pool row of key `key` of the item's sequence and head, -1: no page of the pool.
    auto key_row = [&](const WeightsItem& w, int key) -> int {
        const int page = page_of(a.batch, a.pool.pages, w.b, key >> a.pool.page_log2);
        return page < 0 ? -1 : ((page * a.pool.Hkv + w.hk) << a.pool.page_log2) + (key & ((1 << a.pool.page_log2) - 1));
    };

    if (warp < 16) {
        // ======================= exponentials and sums ===========================================
        const int t = (warp >> 2) & 1, half = warp >> 3, quad = warp & 3;  // key tile, half of the columns, lanes of tensor memory
        const int in_tile = quad * 32 + lane;
        const uint32_t at = tmem_base + C::kColS + C::kHalf * half + (static_cast<uint32_t>(quad * 32) << 16);
        const uint64_t scale2 = f2_pack(a.scale_log2, a.scale_log2);
        uint32_t st = 0, q_use = 0;  // place in the ring of row tiles, and its use's parity
        ScoreTiles scores;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            WeightsItem w;
            if (!next_item(k, kWaitWeights + 30, &w)) break;
            const int key_low = w.key0 + t * kTile, key = key_low + in_tile;
            float sum = 0.f;
            // (where the sum goes, for when it is there)
            const int row = half == 0 && any_attends(w.first, w.last, key, a.window, a.sinks) ? key_row(w, key) : -1;
            RowTiles x(p, w, tokens_log2);
            for (int r = w.r0; r < w.r1; ++r, x.next(groups, tokens_log2)) {
                const int end_pos = x.first_pos + (1 << tokens_log2) - 1;
                if (!mbar_wait_uniform(&bars->l_full[st], q_use, ctx, kWaitWeights + 31)) { ok = false; break; }
                const uint32_t b = scores.tile(t), use = scores.use(t), at_b = at + b * kTile;
                scores.next_row_tile();
                if (!tile_attended<kWindow>(a, w.last, x.first_pos, end_pos, key_low)) {
                    if (!mbar_wait_uniform(&bars->s_full[b], use, ctx, kWaitWeights + 35)) { ok = false; break; }
                    mbar_arrive_warp(&bars->s_empty[b]);
                } else {
                    const float4* lse = reinterpret_cast<const float4*>(sLse + st * kTile + C::kHalf * half);
                    // Most tiles are whole: every row is there and attends every key.
                    const bool whole = end_pos <= w.last && key_low + (kTile - 1) <= x.first_pos &&
                                       (!kWindow || key_low > end_pos - a.window || key_low + kTile <= a.sinks);
                    // columns of rows that attend the key: from .. to - 1 (found before the wait: lanes must be together at what follows it)
                    int from = 0, to = C::kHalf;
                    if (!whole) {
                        int last = min(w.last - x.first_pos, kTile);
                        if (kWindow && key >= a.sinks) last = min(last, key - x.first_pos + a.window - 1);
                        from = (max(min(key - x.first_pos, kTile), 0) << p.pack_log2) - C::kHalf * half;
                        to = (last + 1) * (1 << p.pack_log2) - C::kHalf * half;
                    }
                    if (!mbar_wait_uniform(&bars->s_full[b], use, ctx, kWaitWeights + 32)) { ok = false; break; }
                    tc_fence_after();
                    // 16 columns at a time, the next ones on their way.  (With 32 the 64 registers did not fit beside the rest, and a register that a load in
                    // flight has yet to write must not be spilled.)
                    uint64_t acc[2] = {0, 0};
                    uint32_t s[2][16];
                    tmem_ld_32x16(at_b, s[0]);
                    auto columns = [&](auto is_masked) {
                        constexpr bool kMasked = decltype(is_masked)::value;
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            tmem_wait_ld();
                            if (c < 3) {
                                tmem_ld_32x16(at_b + 16 * (c + 1), s[(c + 1) & 1]);
                            } else {
                                tc_fence_before();
                                mbar_arrive_warp(&bars->s_empty[b]);
                            }
                            const uint32_t(&col)[16] = s[c & 1];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float4 l = lse[4 * c + i];
                                float e[4];
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(col[4 * i]), __uint_as_float(col[4 * i + 1])), scale2, f2_pack(l.x, l.y)), e[0], e[1]);
                                f2_unpack(f2_fma(f2_pack(__uint_as_float(col[4 * i + 2]), __uint_as_float(col[4 * i + 3])), scale2, f2_pack(l.z, l.w)), e[2], e[3]);
#pragma unroll
                                for (int y = 0; y < 4; ++y) {
                                    e[y] = fast_exp2(e[y]);
                                    if (kMasked && (16 * c + 4 * i + y < from || 16 * c + 4 * i + y >= to)) e[y] = 0.f;
                                }
                                acc[0] = f2_add(acc[0], f2_pack(e[0], e[1]));
                                acc[1] = f2_add(acc[1], f2_pack(e[2], e[3]));
                            }
                        }
                    };
                    if (whole) columns(std::false_type());
                    else columns(std::true_type());
                    float u, v, y, z;
                    f2_unpack(acc[0], u, v);
                    f2_unpack(acc[1], y, z);
                    sum += (u + v) + (y + z);  // (a tile's sum by itself: thousands of rows in one accumulator would lose more)
                }
                mbar_arrive_warp(&bars->l_empty[st]);
                if (++st == C::kRing) st = 0, q_use ^= 1;
            }
            if (!ok) break;
            // (the other half of the columns)
            if (half == 1) {
                if (!mbar_wait_uniform(&bars->sum_empty[t], (k & 1) ^ 1, ctx, kWaitWeights + 33)) break;
                sSum[t * kTile + in_tile] = sum;
                mbar_arrive_warp(&bars->sum_full[t]);
                continue;
            }
            if (!mbar_wait_uniform(&bars->sum_full[t], k & 1, ctx, kWaitWeights + 34)) break;
            sum += sSum[t * kTile + in_tile];
            mbar_arrive_warp(&bars->sum_empty[t]);
            if (p.pieces > 1) {
                p.partial[static_cast<long long>(w.id) * kWeightKeys + t * kTile + in_tile] = sum;
            } else if (row >= 0) {
                a.received[row] = (a.before && key < w.first ? __ldcg(a.before + row) : 0.f) + sum;
            }
        }
    } else if (warp < 20) {
        // ======================= keys to tensor memory ===========================================
        const int quad = warp & 3, in_tile = quad * 32 + lane;
        const uint32_t at = tmem_base + (static_cast<uint32_t>(quad * 32) << 16);
        for (int k = 0;; ++k) {
            WeightsItem w;
            if (!next_item(k, kWaitWeights + 20, &w)) break;
            if (!mbar_wait_uniform(&bars->loaded, k & 1, ctx, kWaitWeights + 21)) break;
            // until the item before has made its last product
            if (!mbar_wait_uniform(&bars->k_empty, (k & 1) ^ 1, ctx, kWaitWeights + 22)) break;
            tc_fence_after();
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
                // A lane has a key.  (What no token attends has not been loaded: its lane's scores are anything, and are not used.)
                float f = 0.f;
                if constexpr (kE4M3) {
                    const int e = sExp[t * kTile + in_tile];
                    f = e == kExpNotFinite ? __uint_as_float(0x7fffffffu) : power_of_two(e);
                }
#pragma unroll
                for (int c = 0; c < HD / 64; ++c) {  // 64 values at a time
                    uint32_t value[32];
#pragma unroll
                    for (int i = 0; i < (kE4M3 ? 4 : 8); ++i) {
                        // 16 bytes, swizzled as TMA has left them
                        const uint8_t* line = kE4M3 ? sK + (t * kTile + in_tile) * C::kLine : sK + (t * C::kBoxes + c) * C::kBoxBytes + in_tile * 128;
                        const int piece = kE4M3 ? 4 * c + i : i, moved = piece ^ (C::kLine == 128 ? in_tile & 7 : (in_tile >> 1) & 3);
                        const uint4 x = *reinterpret_cast<const uint4*>(line + 16 * moved);
                        const uint32_t word[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            if constexpr (kE4M3) {
                                uint32_t lo, hi;
                                e4m3_to_f16(word[y], lo, hi);
                                const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&lo)), v = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                                value[8 * i + 2 * y] = pack_bf16(u.x * f, u.y * f), value[8 * i + 2 * y + 1] = pack_bf16(v.x * f, v.y * f);
                            } else {
                                value[4 * i + y] = word[y];
                            }
                        }
                    }
                    tmem_st_32x32(at + t * C::kKeyCols + 32 * c, value);
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive_warp(&bars->k_full[t]);
            }
            fence_proxy_async();  // (read before TMA writes the next ones)
            mbar_arrive_warp(&bars->taken);
        }
    } else if (warp == 20) {
        // ======================= work items, TMA loads ===========================================
        uint32_t n_clc = 0, n_q = 0, n_k = 0;
        bool ok = true;
        const int box_log2 = a.pool.page_log2 < 7 ? a.pool.page_log2 : 7;  // keys of a box
        int id = static_cast<int>(blockIdx.x);
        auto next_id = [&]() {
            if (lane == 0) {
                mbar_expect_tx(&bars->clc, 16);
                clc_try_cancel(bars->clc_resp, &bars->clc);
            }
            __syncwarp();
            if (!mbar_wait_uniform(&bars->clc, n_clc & 1, ctx, kWaitWeights + 1)) {
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
        for (int k = 0; ok; ++k) {
            WeightsItem w;
            while (id >= 0 && !weights_item(p, id, &w)) id = next_id();
            if (id < 0) w.b = -1;
            if (!mbar_wait_uniform(&bars->sched_empty[k % C::kSched], ((k / C::kSched) & 1) ^ 1, ctx, kWaitWeights + 2)) break;
            if (lane == 0) {
                bars->item[k % C::kSched] = w;
                mbar_arrive(&bars->sched_full[k % C::kSched]);  // release: the item is visible to whoever sees the phase
            }
            __syncwarp();
            if (id < 0) break;
            // keys: lane i has the i-th box of them (there are 16 at most), of those that some token attends
            const int first = lane << box_log2;
            int row = -1;
            if (first < kWeightKeys && !hidden_keys(w.first, w.last, w.key0, a.window, a.sinks).all(first, 1 << box_log2)) {
                row = key_row(w, w.key0 + first);
                if (row < 0) report_bad_index(a.status, a.host_status, kBadPage);
            }
            const int boxes = __popc(__ballot_sync(0xffffffffu, row >= 0));
            if (!mbar_wait_uniform(&bars->taken, (k & 1) ^ 1, ctx, kWaitWeights + 3)) break;
            if (lane == 0) mbar_expect_tx(&bars->loaded, static_cast<uint32_t>((boxes * (C::kKeyBytes + (kE4M3 ? 1 : 0))) << box_log2));
            __syncwarp();
            ++n_k;
            if (row >= 0) {
                const uint32_t bar = smem_u32(&bars->loaded);
                if constexpr (kE4M3) {
                    tma_load_2d(smem_u32(sK + first * C::kLine), &p.tm_k, bar, 0, row);
                    bulk_load_1d(sExp + first, a.pool.k_exp + row, 1u << box_log2, &bars->loaded);
                } else {
                    for (int bx = 0; bx < C::kBoxes; ++bx)
                        tma_load_2d(smem_u32(sK + (first / kTile * C::kBoxes + bx) * C::kBoxBytes + first % kTile * 128), &p.tm_k, bar, bx * 64, row);
                }
            }
            __syncwarp();
            RowTiles x(p, w, tokens_log2);
            for (int r = w.r0; r < w.r1; ++r, ++n_q, x.next(groups, tokens_log2)) {
                const uint32_t st = n_q % C::kRing;
                if (!mbar_wait_uniform(&bars->q_empty[st], ((n_q / C::kRing) & 1) ^ 1, ctx, kWaitWeights + 4)) { ok = false; break; }
                if (lane == 0) {
                    mbar_expect_tx(&bars->q_full[st], C::kTileBytes);
                    for (int bx = 0; bx < C::kBoxes; ++bx)
                        tma_load_3d(smem_u32(sQ + st * C::kTileBytes + bx * C::kBoxBytes), &p.tm_q, smem_u32(&bars->q_full[st]), bx * 64,
                                    w.hk * a.rep + (x.group << p.pack_log2), w.row0 + x.first_pos - w.first);
                }
                __syncwarp();
            }
            if (ok) id = next_id();
        }
        // nothing may land after the block has gone
        if (lane == 0) {
            if (bars->abort_flag != 0) {
                if (n_k > 0) mbar_wait_drain(&bars->loaded, (n_k - 1) & 1);
                for (uint32_t x = (n_q > C::kRing ? n_q - C::kRing : 0); x < n_q; ++x) mbar_wait_drain(&bars->q_full[x % C::kRing], (x / C::kRing) & 1);
            }
        }
        __syncwarp();
    } else if (warp == 21) {
        // ======================= MMA issuer ======================================================
        constexpr uint32_t idesc = idesc_bf16(128, kTile, 0, 0);
        const uint32_t dQ = desc_lo_k_major(smem_u32(sQ));
        uint32_t st = 0, q_use = 0;  // as above
        ScoreTiles scores;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            WeightsItem w;
            if (!next_item(k, kWaitWeights + 10, &w)) break;
            for (int r = w.r0; ok && r < w.r1; ++r, scores.next_row_tile()) {
                if (!mbar_wait_uniform(&bars->q_full[st], q_use, ctx, kWaitWeights + 12)) { ok = false; break; }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (ok && r == w.r0 && !mbar_wait_uniform(&bars->k_full[t], k & 1, ctx, kWaitWeights + 11)) ok = false;
                    const uint32_t b = scores.tile(t);
                    if (!ok || !mbar_wait_uniform(&bars->s_empty[b], scores.use(t) ^ 1, ctx, kWaitWeights + 13)) { ok = false; continue; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t at_q = dQ + st * (C::kTileBytes >> 4), acc = tmem_base + C::kColS + b * kTile;
#pragma unroll
                        for (int kk = 0; kk < HD / 16; ++kk)
                            mma_ts(acc, tmem_base + t * C::kKeyCols + kk * 8, at_q + desc_step_k_major(kk, C::kBoxBytes), idesc, kk > 0);
                        mma_commit(&bars->s_full[b]);
                        if (t == 1) mma_commit(&bars->q_empty[st]);
                        if (t == 1 && r == w.r1 - 1) mma_commit(&bars->k_empty);
                    }
                    __syncwarp();
                }
                if (++st == C::kRing) st = 0, q_use ^= 1;
            }
        }
        // MMAs already issued must finish before tensor memory is released
        if (__any_sync(0xffffffffu, *reinterpret_cast<volatile int*>(&bars->abort_flag) != 0)) {
            if (elect_one()) {
                mma_commit(&bars->drain);
                mbar_wait_drain(&bars->drain, 0);
            }
        }
        __syncwarp();
    } else if (warp == 22) {
        // ======================= log sums ========================================================
        // -lse / ln 2 of columns 4 lane .. 4 lane + 3
        auto log_sums = [&](const WeightsItem& w, const RowTiles& x) -> float4 {
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = 4 * lane + i, pos = x.first_pos + (col >> p.pack_log2);
                const int head = w.hk * a.rep + (x.group << p.pack_log2) + (col & ((1 << p.pack_log2) - 1));
                y[i] = pos <= w.last ? __ldcg(a.lse + static_cast<long long>(head) * a.batch.T + w.row0 + pos - w.first) * -1.4426950408889634f : -__uint_as_float(0x7f800000u);
            }
            return make_float4(y[0], y[1], y[2], y[3]);
        };
        uint32_t st = 0, use = 0;
        bool ok = true;
        for (int k = 0; ok; ++k) {
            WeightsItem w;
            if (!next_item(k, kWaitWeights + 15, &w)) break;
            RowTiles x(p, w, tokens_log2);
            for (int r = w.r0; r < w.r1; ++r, x.next(groups, tokens_log2)) {
                const float4 now = log_sums(w, x);
                if (!mbar_wait_uniform(&bars->l_empty[st], use ^ 1, ctx, kWaitWeights + 16)) { ok = false; break; }
                *reinterpret_cast<float4*>(sLse + st * kTile + 4 * lane) = now;
                mbar_arrive_warp(&bars->l_full[st]);
                if (++st == C::kRing) st = 0, use ^= 1;
            }
        }
    }

    // ---- teardown ------------------------------------------------------------------------------
    tc_fence_before();
    __syncthreads();
    if (warp == 21) {
        tc_fence_after();
        tmem_dealloc(tmem_base, C::kTmemCols);
    }
}

// Adds up the pieces of each item; a thread has a key.
__global__ void __launch_bounds__(kWeightKeys) s2a_weights_join_kernel(const __grid_constant__ WeightsTileParams p) {
    const WeightsParams& a = p.a;
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(a.status) != 0) return;
    int unit;
    const int block = p.by_units(static_cast<int>(blockIdx.x), &unit), units = static_cast<int>(p.by_units.d);
    WeightsItem w;
    if (!weights_item(p, block * p.pieces * units + unit, &w)) return;
    const int key = w.key0 + static_cast<int>(threadIdx.x);
    if (!any_attends(w.first, w.last, key, a.window, a.sinks)) return;
    const int page = page_of(a.batch, a.pool.pages, w.b, key >> a.pool.page_log2);
    if (page < 0) return;
    const int row = ((page * a.pool.Hkv + w.hk) << a.pool.page_log2) + (key & ((1 << a.pool.page_log2) - 1));
    float sum = 0.f;
#pragma unroll 4
    for (int i = 0; i < w.pieces; ++i) sum += __ldcg(p.partial + (static_cast<long long>(block * p.pieces + i) * units + unit) * kWeightKeys + threadIdx.x);
    a.received[row] = (a.before && key < w.first ? __ldcg(a.before + row) : 0.f) + sum;
}

template <int HD, bool kE4M3>
cudaError_t configure_one() {
    using C = TileCfg<HD, kE4M3>;
    const cudaError_t e = cudaFuncSetAttribute(s2a_weights_tile_kernel<HD, kE4M3, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(s2a_weights_tile_kernel<HD, kE4M3, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmemBytes);
}
template <int HD, bool kE4M3>
cudaError_t launch_one(const WeightsTileParams& p, cudaStream_t stream) {
    using C = TileCfg<HD, kE4M3>;
    const auto kernel = p.a.window > 0 ? s2a_weights_tile_kernel<HD, kE4M3, true> : s2a_weights_tile_kernel<HD, kE4M3, false>;
    const cudaError_t e = launch_kernel(kernel, static_cast<unsigned>(p.items), C::kThreads, C::kSmemBytes, stream, p, true);
    if (e != cudaSuccess || p.pieces == 1) return e;
    return launch_kernel(s2a_weights_join_kernel, static_cast<unsigned>(p.items / p.pieces), kWeightKeys, 0, stream, p, true);
}

}  // namespace

cudaError_t configure_weights_tile() {
    for (const cudaError_t e : {configure_one<64, false>(), configure_one<64, true>(), configure_one<128, false>(), configure_one<128, true>()})
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

cudaError_t launch_weights_tile(const WeightsTileParams& p, bool e4m3, int d, cudaStream_t stream) {
    if (d == 64) return e4m3 ? launch_one<64, true>(p, stream) : launch_one<64, false>(p, stream);
    return e4m3 ? launch_one<128, true>(p, stream) : launch_one<128, false>(p, stream);
}

}  // namespace s2a
