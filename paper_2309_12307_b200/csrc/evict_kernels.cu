// Eviction from the paged cache: of every sequence and KV head the tokens that stay, and their way to other pages.
//
// A head of n tokens keeps m = min(n, budget): the first `sinks`, the last `recent`, and of those between the heaviest, of equal ones the earlier.
// The selecting kernel finds the weight of the lightest token that stays digit by digit (8 bits at a time of the weights as ordered whole
// numbers, a count of each digit's tokens for a pass), then goes through the tokens once more and writes down which stay, in order.  The copying
// kernel moves their rows.  Other pages, not the same ones: tokens move independently of one another, a prefix that
// other sequences share stays as it is, and each byte that stays is read and written once.
#include "evict.h"
#include "paged_device.cuh"

namespace s2a {

namespace {

constexpr int kSelectThreads = 1024;

// The length of sequence b; -1: out of range.
__device__ __forceinline__ int length_of(const EvictParams& p, int b) {
    const int n = S2A_LOAD(p.lengths + b);
    return n < 0 || n > static_cast<long long>(p.width) << p.pool.page_log2 ? -1 : n;
}

// Row of the pools of place `j` of sequence b and head hk, by a table of `width` entries; -1: no page of the pool.
__device__ __forceinline__ long long place_row(const PagedPool& pool, const int* table, int width, int b, int hk, int j) {
    const int page = S2A_LOAD(table + static_cast<long long>(b) * width + (j >> pool.page_log2));
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(pool.pages)) return -1;
    return ((static_cast<long long>(page) * pool.Hkv + hk) << pool.page_log2) + (j & ((1 << pool.page_log2) - 1));
}

__global__ void __launch_bounds__(kSelectThreads) s2a_evict_select_kernel(const __grid_constant__ EvictParams p) {
    __shared__ int s_count[256];
    __shared__ int s_digit, s_left, s_scan[2][kSelectThreads / 32];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    const int b = static_cast<int>(blockIdx.x) / p.pool.Hkv, hk = static_cast<int>(blockIdx.x) % p.pool.Hkv;
    const int n = length_of(p, b);
    if (n < 0) {
        if (threadIdx.x == 0) report_bad_index(p.status, p.host_status, kBadLength);
        return;
    }
    const int m = min(n, p.budget);
    int* kept = p.kept + static_cast<long long>(blockIdx.x) * p.budget;
    if (hk == 0 && threadIdx.x == 0) p.new_lengths[b] = m;
    for (int i = m + static_cast<int>(threadIdx.x); i < p.budget; i += kSelectThreads) kept[i] = -1;
    if (n == m) {
        for (int i = threadIdx.x; i < m; i += kSelectThreads) kept[i] = i;
        return;
    }
    // n > budget >= sinks + recent: the tokens between
    const int from = p.sinks, to = n - p.recent;
    int left = p.budget - p.sinks - p.recent;  // of them stay
    auto order_of = [&](int j) -> uint32_t {
        const long long row = place_row(p.pool, p.table, p.width, b, hk, j);
        if (row < 0) report_bad_index(p.status, p.host_status, kBadPage);
        return row < 0 ? 0u : weight_order(__float_as_uint(__ldcg(p.received + row)));
    };
    uint32_t border = 0, known = 0;  // the lightest's digits so far
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) s_count[threadIdx.x] = 0;
        __syncthreads();
        for (int j = from + static_cast<int>(threadIdx.x); j < to; j += kSelectThreads) {
            const uint32_t x = order_of(j);
            if ((x & known) == border) atomicAdd(&s_count[(x >> shift) & 255], 1);
        }
        __syncthreads();
        if (threadIdx.x < 32) {
            // lane i has digits 255 - 8 i to 248 - 8 i, the larger ones first
            int own = 0;
            for (int y = 0; y < 8; ++y) own += s_count[255 - 8 * threadIdx.x - y];
            int above = own;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int x = __shfl_up_sync(0xffffffffu, above, off);
                if (static_cast<int>(threadIdx.x) >= off) above += x;
            }
            above -= own;
            if (above < left && above + own >= left) {
                int digit = 255 - 8 * static_cast<int>(threadIdx.x);
                while (above + s_count[digit] < left) above += s_count[digit--];
                s_digit = digit, s_left = left - above;
            }
            if (left == 0 && threadIdx.x == 0) s_digit = 255, s_left = 0;
        }
        __syncthreads();
        border |= static_cast<uint32_t>(s_digit) << shift, known |= 255u << shift;
        left = s_left;
        __syncthreads();
    }
    // those above the border stay, and `left` of those on it, the first ones
    int out = 0, equal = 0;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    for (int base = 0; base < n; base += kSelectThreads) {
        const int j = base + static_cast<int>(threadIdx.x);
        const bool always = j < n && (j < from || j >= to);
        const uint32_t x = j >= from && j < to ? order_of(j) : 0u;
        const bool between = j >= from && j < to, same = between && x == border;
        const uint32_t lanes_before = (1u << lane) - 1, all_same = __ballot_sync(0xffffffffu, same);
        if (lane == 0) s_scan[0][warp] = __popc(all_same);
        __syncthreads();
        int before = equal;
        for (int i = 0; i < kSelectThreads / 32; ++i) {
            if (i < warp) before += s_scan[0][i];
            equal += s_scan[0][i];
        }
        const bool stays = always || (between && x > border) || (same && before + __popc(all_same & lanes_before) < left);
        const uint32_t all = __ballot_sync(0xffffffffu, stays);
        if (lane == 0) s_scan[1][warp] = __popc(all);
        __syncthreads();
        int at = out;
        for (int i = 0; i < kSelectThreads / 32; ++i) {
            if (i < warp) at += s_scan[1][i];
            out += s_scan[1][i];
        }
        at += __popc(all & lanes_before);
        if (stays && at < m) kept[at] = j;
    }
}

constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 64;  // kept tokens of a block

template <int kRowBytes, bool kE4M3>
__global__ void __launch_bounds__(kMoveThreads) s2a_evict_copy_kernel(const __grid_constant__ EvictParams p) {
    constexpr int kLanes = kRowBytes / 16, kAtOnce = kMoveThreads / kLanes, kTurns = 2 * kMoveRows / kAtOnce;  // rows of k and of v
    __shared__ long long s_from[kMoveRows], s_to[kMoveRows];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    int piece;
    const int unit = p.by_pieces(static_cast<int>(blockIdx.x), &piece);
    const int b = unit / p.pool.Hkv, hk = unit % p.pool.Hkv, first = piece * kMoveRows;
    if (threadIdx.x < kMoveRows) {
        const int i = first + static_cast<int>(threadIdx.x), j = i < p.budget ? S2A_LOAD(p.kept + static_cast<long long>(unit) * p.budget + i) : -1;
        long long from = -1, to = -1;
        if (j >= 0) {
            from = place_row(p.pool, p.table, p.width, b, hk, j), to = place_row(p.pool, p.to_table, p.to_width, b, hk, i);
            if (from < 0 || to < 0) report_bad_index(p.status, p.host_status, kBadPage), from = to = -1;
        }
        s_from[threadIdx.x] = from, s_to[threadIdx.x] = to;
        if (from >= 0) {
            p.received[to] = __ldcg(p.received + from);
            if constexpr (kE4M3) p.pool.k_exp[to] = __ldcg(reinterpret_cast<const signed char*>(p.pool.k_exp) + from), p.pool.v_exp[to] = __ldcg(reinterpret_cast<const signed char*>(p.pool.v_exp) + from);
        }
    }
    __syncthreads();
    const int part = static_cast<int>(threadIdx.x) % kLanes, row = static_cast<int>(threadIdx.x) / kLanes;
    uint4 x[kTurns];
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int r = i * kAtOnce + row;
        const long long from = s_from[r % kMoveRows];
        if (from >= 0) x[i] = __ldcg(reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(r < kMoveRows ? p.pool.k : p.pool.v) + from * kRowBytes) + part);
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int r = i * kAtOnce + row;
        const long long to = s_to[r % kMoveRows];
        if (to >= 0) reinterpret_cast<uint4*>(static_cast<uint8_t*>(r < kMoveRows ? p.pool.k : p.pool.v) + to * kRowBytes)[part] = x[i];
    }
}

template <int kRowBytes, bool kE4M3>
cudaError_t launch_copy(EvictParams p, int most, cudaStream_t stream) {
    const int pieces = (most + kMoveRows - 1) / kMoveRows;
    p.by_pieces = FastDiv(pieces);
    return launch_kernel(s2a_evict_copy_kernel<kRowBytes, kE4M3>, static_cast<unsigned>(p.B * p.pool.Hkv * pieces), kMoveThreads, 0, stream, p, true);
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, bool e4m3, int d, cudaStream_t stream) {
    const cudaError_t e = launch_kernel(s2a_evict_select_kernel, static_cast<unsigned>(p.B * p.pool.Hkv), kSelectThreads, 0, stream, p, true);
    if (e != cudaSuccess) return e;
    const long long longest = static_cast<long long>(p.width) << p.pool.page_log2;
    const int most = static_cast<int>(p.budget < longest ? p.budget : longest);  // tokens that a head keeps
    if (e4m3) return d == 64 ? launch_copy<64, true>(p, most, stream) : launch_copy<128, true>(p, most, stream);
    return d == 64 ? launch_copy<128, false>(p, most, stream) : launch_copy<256, false>(p, most, stream);
}

}  // namespace s2a
