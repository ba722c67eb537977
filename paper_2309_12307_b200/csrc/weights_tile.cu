// What attention weight cached tokens get from many rows (pieces of prompts): see weights_kernels.cu for the formula.
//
// S^T = K Q^T on tcgen05, 128 keys by 128 rows of q at a time.  A score tile has a key in each lane of tensor memory and a row of q in each column, so
// the thread that has a key adds up its columns' exponentials in registers: nothing crosses threads, and there is no second product.
// An item is two key tiles of a sequence and KV head, which stay in shared memory while the row tiles that attend any of them (as s2a_paged_fwd_kernel's: query heads
// of a KV head and neighbouring tokens, one TMA box) pass by.  Two tiles, because a row tile is 32 KB from the L2 that would otherwise be read twice as often.
//
// One persistent block per SM:
//   warps 0-3, 4-7  exponentials and sums, four warps for either key tile, two score buffers each
//   warp 8          work items (cluster launch control), TMA loads of q and of bf16 keys, the rows' log sums
//   warp 9          tcgen05 MMAs
//   warps 10-13     8-bit caches: codes to bf16, what they stand for exactly, once for an item, where TMA would have put them
// An item's keys are loaded while the last rows of the one before are worked on (two key buffers).
//
// Where there are few items their rows are split into pieces, whose sums a second kernel adds up in order.
#include <cuda_fp16.h>

#include "evict.h"
#include "paged_device.cuh"

namespace s2a {

namespace {

template <int HD, bool kE4M3>
struct TileCfg {
    static constexpr int kThreads = kE4M3 ? 448 : 320;
    static constexpr int kBoxes = HD / 64;                 // 64-column boxes per tile
    static constexpr int kBoxBytes = kTile * 128;          // 128 rows x 128 bytes
    static constexpr int kTileBytes = kBoxes * kBoxBytes;
    static constexpr int kRing = HD == 128 ? 3 : 6;        // row tiles in flight
    static constexpr int kStats = kRing + 1;               // their log sums
    static constexpr int kSched = 4;                       // items in flight
    static constexpr int kBarBytes = 1024;
    static constexpr int kSmemBytes = (2 * 2 + kRing) * kTileBytes + kStats * kTile * 4 + kBarBytes;
    static_assert(kSmemBytes <= 232448, "shared memory");
    static constexpr int kTmemCols = 512;                  // [key tile][buffer][128 rows]
};

template <int HD, bool kE4M3>
struct TileBars {
    using C = TileCfg<HD, kE4M3>;
    uint64_t k_full[2], k_empty[2];
    uint64_t q_full[C::kRing], q_empty[C::kRing];
    uint64_t l_full[C::kStats], l_empty[C::kStats];
    uint64_t s_full[2][2], s_empty[2][2];
    uint64_t sched_full[C::kSched], sched_empty[C::kSched];
    uint64_t clc, drain;
    alignas(16) uint8_t clc_resp[16];
    WeightsItem item[C::kSched];
    uint32_t tmem_slot;
    int abort_flag;
};

// Whether any of the tokens of row tile r attends a key of tile t.
__device__ __forceinline__ bool tile_attended(const WeightsItem& w, int first_pos, int tokens_log2, int t, int window, int sinks) {
    const int end = first_pos + (1 << tokens_log2) - 1, last = end < w.last ? end : w.last, key = w.key0 + t * kTile;
    return key <= last && (window == 0 || key + (kTile - 1) > first_pos - window || key < sinks);
}

template <int HD, bool kE4M3>
__global__ void __launch_bounds__(TileCfg<HD, kE4M3>::kThreads, 1) s2a_weights_tile_kernel(const __grid_constant__ WeightsTileParams p) {
    using C = TileCfg<HD, kE4M3>;
    using Bars = TileBars<HD, kE4M3>;
    static_assert(sizeof(Bars) <= C::kBarBytes, "barrier block");
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sK = smem;                                   // [buffer][key tile]
    uint8_t* sQ = sK + 4 * C::kTileBytes;                 // ring of row tiles
    float* sLse = reinterpret_cast<float*>(sQ + C::kRing * C::kTileBytes);  // ring of -lse / ln 2, -inf for rows that are not there
    Bars* bars = reinterpret_cast<Bars*>(reinterpret_cast<uint8_t*>(sLse) + C::kStats * kTile * 4);
    const WeightsParams& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int kConsumers = 8 + 1 + (kE4M3 ? 4 : 0);   // warps that read items

    if (threadIdx.x == 0) {
        for (int x = 0; x < 2; ++x) {
            mbar_init(&bars->k_full[x], kE4M3 ? 4 : 1);
            mbar_init(&bars->k_empty[x], 1);
            for (int y = 0; y < 2; ++y) mbar_init(&bars->s_full[x][y], 1), mbar_init(&bars->s_empty[x][y], 4);
        }
        for (int x = 0; x < C::kRing; ++x) mbar_init(&bars->q_full[x], 1), mbar_init(&bars->q_empty[x], 1);
        for (int x = 0; x < C::kStats; ++x) mbar_init(&bars->l_full[x], 1), mbar_init(&bars->l_empty[x], 8);
        for (int x = 0; x < C::kSched; ++x) mbar_init(&bars->sched_full[x], 1), mbar_init(&bars->sched_empty[x], kConsumers);
        mbar_init(&bars->clc, 1);
        mbar_init(&bars->drain, 1);
        fence_barrier_init();
        tma_prefetch_desc(&p.tm_q);
        if (!kE4M3) tma_prefetch_desc(&p.tm_k);
    }
    if (warp == 9) {
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
        if (warp == 9) tmem_dealloc(tmem_base, C::kTmemCols);
        return;
    }
    if (blockIdx.x == 0) check_batch(a.batch, a.pool.page_log2, a.most_new, a.status, a.host_status);
    const WaitCtx ctx{&bars->abort_flag, a.status, a.host_status};
    const int tokens_log2 = 7 - p.pack_log2;

    auto next_item = [&](int k, int where, WeightsItem* w) -> bool {
        if (!mbar_wait_uniform(&bars->sched_full[k % C::kSched], (k / C::kSched) & 1, ctx, where)) return false;
        *w = bars->item[k % C::kSched];
        mbar_arrive_warp(&bars->sched_empty[k % C::kSched]);
        return w->b >= 0;
    };
    // Pool row of key `key` of the item's sequence and head, -1: no page of the pool.
    auto key_row = [&](const WeightsItem& w, int key) -> int {
        const int page = page_of(a.batch, a.pool.pages, w.b, key >> a.pool.page_log2);
        return page < 0 ? -1 : ((page * a.pool.Hkv + w.hk) << a.pool.page_log2) + (key & ((1 << a.pool.page_log2) - 1));
    };

    if (warp == 8) {
        // ======================= work items, TMA loads ===========================================
        uint32_t n_clc = 0, n_q = 0, n_k = 0;
        bool ok = true;
        int id = static_cast<int>(blockIdx.x);
        const int piece_log2 = a.pool.page_log2 < 7 ? a.pool.page_log2 : 7;  // keys of a box
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
        // -lse / ln 2 of columns 4 lane .. 4 lane + 3 of row tile r
        auto log_sums = [&](const WeightsItem& w, int r) -> float4 {
            int group;
            const int token0 = (w.t_lo + p.by_groups(r, &group)) << tokens_log2, n = w.last - w.first + 1;
            float x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = 4 * lane + i, token = token0 + (col >> p.pack_log2);
                const int head = w.hk * a.rep + (group << p.pack_log2) + (col & ((1 << p.pack_log2) - 1));
                x[i] = token < n ? __ldcg(a.lse + static_cast<long long>(head) * a.batch.T + w.row0 + token) * -1.4426950408889634f : -__uint_as_float(0x7f800000u);
            }
            return make_float4(x[0], x[1], x[2], x[3]);
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
            if constexpr (!kE4M3) {
                // keys: lane i has the i-th box of either tile (there are 16 at most)
                const int buf = k & 1, at = lane << piece_log2;
                const HiddenKeys hidden = hidden_keys(w.first, w.last, w.key0, a.window, a.sinks);
                int row = -1;
                if (at < kWeightKeys && !hidden.all(at, 1 << piece_log2)) {
                    row = key_row(w, w.key0 + at);
                    if (row < 0) report_bad_index(a.status, a.host_status, kBadPage);
                }
                const int boxes = __popc(__ballot_sync(0xffffffffu, row >= 0));
                if (!mbar_wait_uniform(&bars->k_empty[buf], ((k >> 1) & 1) ^ 1, ctx, kWaitWeights + 3)) break;
                if (lane == 0) mbar_expect_tx(&bars->k_full[buf], static_cast<uint32_t>((boxes * HD * 2) << piece_log2));
                __syncwarp();
                if (row >= 0) {
                    const uint32_t dst = smem_u32(sK + (2 * buf + at / kTile) * C::kTileBytes) + (at % kTile) * 128;
                    for (int bx = 0; bx < C::kBoxes; ++bx) tma_load_2d(dst + bx * C::kBoxBytes, &p.tm_k, smem_u32(&bars->k_full[buf]), bx * 64, row);
                }
                __syncwarp();
                ++n_k;
            }
            float4 next = log_sums(w, w.r0);
            for (int r = w.r0; r < w.r1; ++r, ++n_q) {
                const float4 now = next;
                if (r + 1 < w.r1) next = log_sums(w, r + 1);
                const uint32_t st = n_q % C::kRing, sl = n_q % C::kStats;
                if (!mbar_wait_uniform(&bars->q_empty[st], ((n_q / C::kRing) & 1) ^ 1, ctx, kWaitWeights + 4)) { ok = false; break; }
                int group;
                const int token0 = (w.t_lo + p.by_groups(r, &group)) << tokens_log2;
                if (lane == 0) {
                    mbar_expect_tx(&bars->q_full[st], C::kTileBytes);
                    for (int bx = 0; bx < C::kBoxes; ++bx)
                        tma_load_3d(smem_u32(sQ + st * C::kTileBytes + bx * C::kBoxBytes), &p.tm_q, smem_u32(&bars->q_full[st]), bx * 64,
                                    w.hk * a.rep + (group << p.pack_log2), w.row0 + token0);
                }
                __syncwarp();
                if (!mbar_wait_uniform(&bars->l_empty[sl], ((n_q / C::kStats) & 1) ^ 1, ctx, kWaitWeights + 5)) { ok = false, ++n_q; break; }
                *reinterpret_cast<float4*>(sLse + sl * kTile + 4 * lane) = now;
                mbar_arrive_warp(&bars->l_full[sl]);
            }
            if (ok) id = next_id();
        }
        // nothing may land after the block has gone
        if (lane == 0) {
            if (bars->abort_flag != 0) {
                for (uint32_t x = (n_q > C::kRing ? n_q - C::kRing : 0); x < n_q; ++x) mbar_wait_drain(&bars->q_full[x % C::kRing], (x / C::kRing) & 1);
                for (uint32_t x = (n_k > 2 ? n_k - 2 : 0); x < n_k; ++x) mbar_wait_drain(&bars->k_full[x & 1], (x >> 1) & 1);
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ======================= MMA issuer ======================================================
        constexpr uint32_t idesc = idesc_bf16(128, kTile, 0, 0);
        const uint32_t dK = desc_lo_k_major(smem_u32(sK)), dQ = desc_lo_k_major(smem_u32(sQ));
        uint32_t n_q = 0, n_s[2] = {0, 0};
        bool ok = true;
        for (int k = 0; ok; ++k) {
            WeightsItem w;
            if (!next_item(k, kWaitWeights + 10, &w)) break;
            const int buf = k & 1;
            if (!mbar_wait_uniform(&bars->k_full[buf], (k >> 1) & 1, ctx, kWaitWeights + 11)) break;
            for (int r = w.r0; ok && r < w.r1; ++r, ++n_q) {
                const uint32_t st = n_q % C::kRing;
                if (!mbar_wait_uniform(&bars->q_full[st], (n_q / C::kRing) & 1, ctx, kWaitWeights + 12)) { ok = false; break; }
                int group;
                const int first_pos = w.first + ((w.t_lo + p.by_groups(r, &group)) << tokens_log2);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (!ok || !tile_attended(w, first_pos, tokens_log2, t, a.window, a.sinks)) continue;
                    const uint32_t b = n_s[t] & 1;
                    if (!mbar_wait_uniform(&bars->s_empty[t][b], ((n_s[t] >> 1) & 1) ^ 1, ctx, kWaitWeights + 13)) { ok = false; continue; }
                    tc_fence_after();
                    if (elect_one()) {
                        const uint32_t at_k = dK + (2 * buf + t) * (C::kTileBytes >> 4), at_q = dQ + st * (C::kTileBytes >> 4);
                        const uint32_t acc = tmem_base + (2 * t + b) * kTile;
#pragma unroll
                        for (int kk = 0; kk < HD / 16; ++kk)
                            mma_ss(acc, at_k + desc_step_k_major(kk, C::kBoxBytes), at_q + desc_step_k_major(kk, C::kBoxBytes), idesc, kk > 0);
                        mma_commit(&bars->s_full[t][b]);
                    }
                    __syncwarp();
                    ++n_s[t];
                }
                if (!ok) break;
                if (elect_one()) {
                    mma_commit(&bars->q_empty[st]);
                    if (r == w.r1 - 1) mma_commit(&bars->k_empty[buf]);
                }
                __syncwarp();
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
    } else if (warp >= 10) {
        // ======================= codes to bf16 ===================================================
        if constexpr (kE4M3) {
            constexpr int kLanes = HD / 16, kKeys = 32 / kLanes, kAtOnce = 4;  // lanes of a key, keys of a warp's load, loads in flight
            const int part = lane % kLanes;
            for (int k = 0;; ++k) {
                WeightsItem w;
                if (!next_item(k, kWaitWeights + 20, &w)) break;
                const int buf = k & 1;
                if (!mbar_wait_uniform(&bars->k_empty[buf], ((k >> 1) & 1) ^ 1, ctx, kWaitWeights + 21)) break;
                const HiddenKeys hidden = hidden_keys(w.first, w.last, w.key0, a.window, a.sinks);
                for (int base = (warp - 10) * 64; base < (warp - 10) * 64 + 64; base += kAtOnce * kKeys) {
                    int row[kAtOnce], e[kAtOnce];
                    uint4 code[kAtOnce];
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) {
                        const int at = base + i * kKeys + lane / kLanes;
                        row[i] = -1;
                        if (!hidden.has(at)) {
                            row[i] = key_row(w, w.key0 + at);
                            if (row[i] < 0) report_bad_index(a.status, a.host_status, kBadPage);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) {
                        if (row[i] < 0) continue;
                        code[i] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.pool.k) + static_cast<long long>(row[i]) * HD) + part);
                        e[i] = __ldcg(reinterpret_cast<const signed char*>(a.pool.k_exp) + row[i]);
                    }
#pragma unroll
                    for (int i = 0; i < kAtOnce; ++i) {
                        if (row[i] < 0) continue;
                        const int at = base + i * kKeys + lane / kLanes, in_tile = at % kTile;
                        const float f = e[i] == kExpNotFinite ? __uint_as_float(0x7fffffffu) : power_of_two(e[i]);
                        const uint32_t word[4] = {code[i].x, code[i].y, code[i].z, code[i].w};
                        uint32_t out[8];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            uint32_t lo, hi;
                            e4m3_to_f16(word[x], lo, hi);
                            const float2 u = __half22float2(*reinterpret_cast<const __half2*>(&lo)), v = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                            out[2 * x] = pack_bf16(u.x * f, u.y * f), out[2 * x + 1] = pack_bf16(v.x * f, v.y * f);
                        }
                        // 16 values: chunks 2 part and 2 part + 1 of 8, permuted in the row's 128 bytes as TMA's swizzle does
                        uint8_t* box = sK + (2 * buf + at / kTile) * C::kTileBytes + (part / 4) * C::kBoxBytes + in_tile * 128;
#pragma unroll
                        for (int x = 0; x < 2; ++x)
                            *reinterpret_cast<uint4*>(box + (((2 * part + x) & 7) ^ (in_tile & 7)) * 16) = make_uint4(out[4 * x], out[4 * x + 1], out[4 * x + 2], out[4 * x + 3]);
                    }
                }
                fence_proxy_async();
                mbar_arrive_warp(&bars->k_full[buf]);
            }
        }
    } else {
        // ======================= exponentials and sums ===========================================
        const int t = warp >> 2, quad = warp & 3;
        const int in_tile = quad * 32 + lane;
        uint32_t n_s = 0, n_q = 0;
        const uint64_t scale2 = f2_pack(a.scale_log2, a.scale_log2);
        bool ok = true;
        for (int k = 0; ok; ++k) {
            WeightsItem w;
            if (!next_item(k, kWaitWeights + 30, &w)) break;
            const int key = w.key0 + t * kTile + in_tile;
            float sum = 0.f;
            for (int r = w.r0; r < w.r1; ++r, ++n_q) {
                const uint32_t sl = n_q % C::kStats;
                int group;
                const int token0 = (w.t_lo + p.by_groups(r, &group)) << tokens_log2, first_pos = w.first + token0;
                if (!mbar_wait_uniform(&bars->l_full[sl], (n_q / C::kStats) & 1, ctx, kWaitWeights + 31)) { ok = false; break; }
                if (tile_attended(w, first_pos, tokens_log2, t, a.window, a.sinks)) {
                    const uint32_t b = n_s & 1;
                    if (!mbar_wait_uniform(&bars->s_full[t][b], (n_s >> 1) & 1, ctx, kWaitWeights + 32)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t at = tmem_base + (2 * t + b) * kTile + (static_cast<uint32_t>(quad * 32) << 16);
                    const float4* lse = reinterpret_cast<const float4*>(sLse + sl * kTile);
                    // columns of rows that attend the key: from .. to - 1
                    const int end_pos = first_pos + (1 << tokens_log2) - 1, key_low = w.key0 + t * kTile;
                    const bool whole = end_pos <= w.last && all_attend(first_pos, end_pos, key_low, kTile, a.window, a.sinks);
                    int from = 0, to = kTile;
                    if (!whole) {
                        from = key > first_pos ? min(key - first_pos, kTile) << p.pack_log2 : 0;
                        int last = min(w.last - first_pos, kTile);
                        if (a.window > 0 && key >= a.sinks) last = min(last, key - first_pos + a.window - 1);
                        to = (last + 1) * (1 << p.pack_log2);
                    }
                    uint64_t acc[2] = {0, 0};
                    uint32_t s[2][32];
                    tmem_ld_32x32(at, s[0]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        tmem_wait_ld();
                        if (c < 3) tmem_ld_32x32(at + 32 * (c + 1), s[(c + 1) & 1]);
                        if (c == 3) {
                            tc_fence_before();
                            mbar_arrive_warp(&bars->s_empty[t][b]);
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float4 l = lse[8 * c + i];
                            const uint32_t(&x)[32] = s[c & 1];
                            const uint64_t lo = f2_fma(f2_pack(__uint_as_float(x[4 * i]), __uint_as_float(x[4 * i + 1])), scale2, f2_pack(l.x, l.y));
                            const uint64_t hi = f2_fma(f2_pack(__uint_as_float(x[4 * i + 2]), __uint_as_float(x[4 * i + 3])), scale2, f2_pack(l.z, l.w));
                            float e[4];
                            f2_unpack(lo, e[0], e[1]);
                            f2_unpack(hi, e[2], e[3]);
#pragma unroll
                            for (int y = 0; y < 4; ++y) e[y] = fast_exp2(e[y]);
                            if (!whole) {
#pragma unroll
                                for (int y = 0; y < 4; ++y)
                                    if (32 * c + 4 * i + y < from || 32 * c + 4 * i + y >= to) e[y] = 0.f;
                            }
                            acc[0] = f2_add(acc[0], f2_pack(e[0], e[1]));
                            acc[1] = f2_add(acc[1], f2_pack(e[2], e[3]));
                        }
                    }
                    float u, v, x, y;
                    f2_unpack(acc[0], u, v);
                    f2_unpack(acc[1], x, y);
                    sum += (u + v) + (x + y);  // (a tile's sum by itself: thousands of rows in one accumulator would lose more)
                    ++n_s;
                }
                mbar_arrive_warp(&bars->l_empty[sl]);
            }
            if (!ok) break;
            if (p.pieces > 1) {
                p.partial[static_cast<long long>(w.id) * kWeightKeys + t * kTile + in_tile] = sum;
            } else if (any_attends(w.first, w.last, key, a.window, a.sinks)) {
                const int row = key_row(w, key);
                if (row >= 0) a.received[row] = (a.before && key < w.first ? __ldcg(a.before + row) : 0.f) + sum;
            }
        }
    }

    // ---- teardown ------------------------------------------------------------------------------
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
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
    return cudaFuncSetAttribute(s2a_weights_tile_kernel<HD, kE4M3>, cudaFuncAttributeMaxDynamicSharedMemorySize, TileCfg<HD, kE4M3>::kSmemBytes);
}
template <int HD, bool kE4M3>
cudaError_t launch_one(const WeightsTileParams& p, cudaStream_t stream) {
    using C = TileCfg<HD, kE4M3>;
    const cudaError_t e = launch_kernel(s2a_weights_tile_kernel<HD, kE4M3>, static_cast<unsigned>(p.items), C::kThreads, C::kSmemBytes, stream, p, true);
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
