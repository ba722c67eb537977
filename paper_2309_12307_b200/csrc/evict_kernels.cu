// Eviction from the paged cache: of every sequence and KV head the tokens that stay, and their way to other pages.
//
// A head of n tokens keeps m = min(n, budget): the first `sinks`, the last `recent`, and of those between the heaviest, of equal ones the earlier.
//
// The selecting kernel finds the weight of the lightest token that stays digit by digit: 11, 11 and 10 bits of the weights as ordered whole numbers (the first digit has the exponent and two bits
// more, over which weights spread; of 8 bits it would be the same for most of them, and its counter what all threads wait for).  A cluster of up to 8 blocks has a head: each
// block has a part of its tokens, whose weights it reads once and keeps in shared memory, counts their digits there, and adds up the counts of all blocks.  Then each thread counts, of the
// neighbouring tokens that are its own, those above the border and those on it; one scan over the threads, and the other blocks' totals, say where each thread's tokens go in the list
// of those that stay.  What bounds it is latency: three rounds of counting, a barrier and a scan each.  (One block a head that read the weights anew for each of four 8-bit digits, 100,000
// tokens of 8 heads: both kernels and reading back 470 us.)
//
// The copying kernel moves the rows.  Other pages, not the same ones: tokens move independently of one another, a prefix that
// other sequences share stays as it is, and each byte that stays is read and written once.  Bound by HBM.
#include "evict.h"
#include "paged_device.cuh"

namespace s2a {

namespace {

constexpr int kSelectThreads = 512;
constexpr int kDigits = 2048;              // values of a digit
constexpr int kMostBlocks = 8;             // of a cluster
constexpr int kMostKept = 48 * 1024;       // weights that a block keeps in shared memory

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

// By a whole block: the sums of x over the threads before this one (*before), and over all.  Two counts at a time.
__device__ __forceinline__ int2 scan_block(int2 x, int2 (&s_warp)[kSelectThreads / 32], int2* before) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    int2 sum = x;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, sum.x, off), v = __shfl_up_sync(0xffffffffu, sum.y, off);
        if (lane >= off) sum.x += u, sum.y += v;
    }
    __syncthreads();  // (s_warp has been read)
    if (lane == 31) s_warp[warp] = sum;
    __syncthreads();
    int2 base = make_int2(0, 0), all = make_int2(0, 0);
#pragma unroll
    for (int i = 0; i < kSelectThreads / 32; ++i) {
        const int2 w = s_warp[i];
        if (i < warp) base.x += w.x, base.y += w.y;
        all.x += w.x, all.y += w.y;
    }
    *before = make_int2(base.x + sum.x - x.x, base.y + sum.y - x.y);
    return all;
}

__global__ void __launch_bounds__(kSelectThreads) s2a_evict_select_kernel(const __grid_constant__ EvictParams p) {
    extern __shared__ __align__(16) uint32_t s_keys[];  // this block's weights, as ordered whole numbers, if there is room
    __shared__ int s_count[3][kDigits];
    __shared__ int2 s_warp[kSelectThreads / 32];
    __shared__ int s_digit, s_left;
    __shared__ int s_totals[2];
    release_successor();
    wait_for_predecessor();
    // After an earlier report nothing is written.  (The block does not leave: one of its cluster may have found nothing yet, and reads this one's shared memory.)
    const bool quiet = *reinterpret_cast<volatile int*>(p.status) != 0;
    const int rank = static_cast<int>(blockIdx.x) % p.cluster, unit = static_cast<int>(blockIdx.x) / p.cluster;
    const int b = unit / p.pool.Hkv, hk = unit % p.pool.Hkv;
    const int n = length_of(p, b);
    if (n < 0) {
        if (threadIdx.x == 0) report_bad_index(p.status, p.host_status, kBadLength);
        return;
    }
    const int m = min(n, p.budget), all_threads = p.cluster * kSelectThreads, thread = rank * kSelectThreads + static_cast<int>(threadIdx.x);
    int* kept = p.kept + static_cast<long long>(unit) * p.budget;
    if (!quiet) {
        if (hk == 0 && thread == 0) p.new_lengths[b] = m;
        for (int i = m + thread; i < p.budget; i += all_threads) kept[i] = -1;
        for (int i = thread; n == m && i < m; i += all_threads) kept[i] = i;
    }
    if (n == m) return;
    // n > budget >= sinks + recent: of the tokens from .. to - 1 `left` stay.  This block has those from low to high - 1 of all.
    const int from = p.sinks, to = n - p.recent;
    int left = p.budget - p.sinks - p.recent;
    const int part = ((n + p.cluster - 1) / p.cluster + 3) & ~3, low = min(rank * part, n), high = min(low + part, n);
    const bool keep = part <= p.room;
    // the weights of tokens j .. j + 3 (j a multiple of four, so they are neighbours in a page)
    auto four = [&](int j, uint32_t (&x)[4]) {
        const long long row = place_row(p.pool, p.table, p.width, b, hk, j);
        if (row < 0) report_bad_index(p.status, p.host_status, kBadPage);
        const float4 w = row < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcg(reinterpret_cast<const float4*>(p.received + row));
        x[0] = weight_order(__float_as_uint(w.x)), x[1] = weight_order(__float_as_uint(w.y));
        x[2] = weight_order(__float_as_uint(w.z)), x[3] = weight_order(__float_as_uint(w.w));
    };
    auto key_of = [&](int j) -> uint32_t {
        if (keep) return s_keys[j - low];
        uint32_t x[4];
        four(j & ~3, x);
        return j & 2 ? (j & 1 ? x[3] : x[2]) : (j & 1 ? x[1] : x[0]);
    };
    for (int i = threadIdx.x; i < 3 * kDigits; i += kSelectThreads) s_count[0][i] = 0;
    __syncthreads();
    // the digits: bits 21 .. 31, 10 .. 20, 0 .. 9
    for (int j = low + 4 * static_cast<int>(threadIdx.x); j < high; j += 4 * kSelectThreads) {
        uint32_t x[4];
        four(j, x);
        if (keep) *reinterpret_cast<uint4*>(s_keys + j - low) = make_uint4(x[0], x[1], x[2], x[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (j + i >= from && j + i < min(to, high)) atomicAdd(&s_count[0][x[i] >> 21], 1);
    }
    uint32_t border = 0, known = 0;  // the lightest's digits so far
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
        if (round > 0) {
            const uint32_t mask = round == 1 ? 0x7ffu : 0x3ffu;
            for (int j = low + static_cast<int>(threadIdx.x); j < high; j += kSelectThreads) {
                if (j < from || j >= to) continue;
                const uint32_t x = key_of(j);
                if ((x & known) == border) atomicAdd(&s_count[round][x >> shift & mask], 1);
            }
        }
        cluster_sync();
        // of all blocks: thread i has the digits kDigits - 1 - 4 i on downwards, the larger ones first
        static_assert(kDigits == 4 * kSelectThreads, "a thread has four digits");
        const int top = kDigits - 1 - 4 * static_cast<int>(threadIdx.x);
        int count[4] = {0, 0, 0, 0};
        for (int r = 0; r < p.cluster; ++r) {
#pragma unroll
            for (int i = 0; i < 4; ++i) count[i] += __float_as_int(load_remote(smem_u32(&s_count[round][top - i]), r));
        }
        int2 above;
        scan_block(make_int2(count[0] + count[1] + count[2] + count[3], 0), s_warp, &above);
        if (threadIdx.x == 0 && left == 0) s_digit = kDigits - 1, s_left = 0;
        if (above.x < left && above.x + count[0] + count[1] + count[2] + count[3] >= left) {
            int x = above.x, i = 0;
#pragma unroll
            for (int y = 0; y < 3; ++y)
                if (i == y && x + count[y] < left) x += count[y], ++i;
            s_digit = top - i, s_left = left - x;
        }
        __syncthreads();
        // (with nothing left to find, above all numbers)
        border |= static_cast<uint32_t>(s_digit) << shift, known |= (round == 2 ? 0x3ffu : 0x7ffu) << shift;
        left = s_left;
    }
    // Those above the border stay, and `left` of those on it, the first ones.  A thread has neighbouring tokens, an odd number of them, so that threads meet in no bank.
    const int each = ((high - low + kSelectThreads - 1) / kSelectThreads) | 1;
    const int first = min(low + each * static_cast<int>(threadIdx.x), high), end = min(first + each, high);
    auto stays = [&](int j, bool* same) -> bool {
        *same = false;
        if (j < from || j >= to) return true;
        const uint32_t x = key_of(j);
        *same = x == border;
        return x > border;
    };
    int2 mine = make_int2(0, 0), before;
    for (int j = first; j < end; ++j) {
        bool same;
        mine.x += stays(j, &same);
        mine.y += same;
    }
    const int2 all = scan_block(mine, s_warp, &before);
    if (threadIdx.x == 0) s_totals[0] = all.x, s_totals[1] = all.y;
    cluster_sync();
    for (int r = 0; r < rank; ++r) {
        before.x += __float_as_int(load_remote(smem_u32(&s_totals[0]), r));
        before.y += __float_as_int(load_remote(smem_u32(&s_totals[1]), r));
    }
    cluster_sync();  // (no block is gone before the others have read its totals)
    int at = before.x + min(before.y, left), equal = before.y;
    for (int j = first; j < end; ++j) {
        bool same;
        bool stay = stays(j, &same);
        if (same) stay = equal++ < left;
        if (stay && at < m) {
            if (!quiet) kept[at] = j;
            ++at;
        }
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

cudaError_t configure_evict() { return cudaFuncSetAttribute(s2a_evict_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostKept * 4); }

cudaError_t launch_evict(EvictParams p, int n_sm, bool e4m3, int d, cudaStream_t stream) {
    const long long longest = static_cast<long long>(p.width) << p.pool.page_log2, units = static_cast<long long>(p.B) * p.pool.Hkv;
    // Blocks of a cluster: as many as there are multiprocessors for, while each has 1024 tokens and more; more of them where their weights fit no other way.
    p.cluster = 1;
    while (p.cluster < kMostBlocks && ((units * p.cluster * 2 <= n_sm && longest > 2048ll * p.cluster) || longest > static_cast<long long>(kMostKept) * p.cluster)) p.cluster *= 2;
    const long long part = ((longest + p.cluster - 1) / p.cluster + 3) & ~3ll;
    p.room = part <= kMostKept ? static_cast<int>(part) : 0;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(units * p.cluster));
    config.blockDim = dim3(kSelectThreads);
    config.dynamicSmemBytes = static_cast<size_t>(p.room) * 4;
    config.stream = stream;
    cudaLaunchAttribute attributes[2] = {};
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = static_cast<unsigned>(p.cluster), attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.attrs = attributes, config.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&config, s2a_evict_select_kernel, p);
    if (e != cudaSuccess) return e;
    const int most = static_cast<int>(p.budget < longest ? p.budget : longest);  // tokens that a head keeps
    if (e4m3) return d == 64 ? launch_copy<64, true>(p, most, stream) : launch_copy<128, true>(p, most, stream);
    return d == 64 ? launch_copy<128, false>(p, most, stream) : launch_copy<256, false>(p, most, stream);
}

}  // namespace s2a
