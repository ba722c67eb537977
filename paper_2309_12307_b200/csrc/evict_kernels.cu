// Eviction from the paged cache: of every sequence and KV head the tokens that stay, and their way to other pages.
//
// A head of n tokens keeps m = min(n, budget): the first `sinks`, the last `recent`, and of those between the heaviest, of equal ones the earlier.
//
// The selecting kernel finds the weight of the lightest token that stays digit by digit: 11, 11 and 10 bits of the weights as ordered whole numbers (the
// first digit has the exponent and two bits more, over which weights spread; of 8 bits it would be the same for most of them, and its counter what all
// threads wait for).  A cluster of up to 8 blocks has a head: each block has a part of its tokens, whose weights it reads once and keeps in shared memory,
// counts their digits there, and adds up the counts of all blocks.  Then each warp counts, of the neighbouring tokens that are its own, those above the
// border and those on it; one scan over the warps, and the other blocks' totals, say where each warp's tokens go in the list of those that stay.  What
// bounds it is latency: three rounds of counting, a barrier and a scan each.  (One block a head that read the weights anew for each of four 8-bit digits,
// 100,000 tokens of 8 heads: both kernels and reading back 470 us; so 47.)
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
constexpr int kMostKept = 46 * 1024;       // weights that a block keeps in shared memory

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

// Four numbers of another block of the cluster, at this block's address `saddr`.
__device__ __forceinline__ int4 load_remote_four(uint32_t saddr, uint32_t rank) {
    int4 x;
    asm volatile(
        "{\n"
        ".reg .u32 a;\n"
        "mapa.shared::cluster.u32 a, %4, %5;\n"
        "ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [a];\n"
        "}\n"
        : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
        : "r"(saddr), "r"(rank)
        : "memory");
    return x;
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

// kKept: whether a block's weights fit its shared memory.
template <bool kKept>
__global__ void __launch_bounds__(kSelectThreads) s2a_evict_select_kernel(const __grid_constant__ EvictParams p) {
    extern __shared__ __align__(16) uint4 s_keys[];  // this block's weights, as ordered whole numbers
    __shared__ __align__(16) int s_count[3][kDigits];
    __shared__ __align__(16) int s_sum[3][kDigits / 2];  // of this block's part of the digits, of all blocks
    __shared__ int2 s_warp[kSelectThreads / 32];
    __shared__ int s_digit, s_left;
    __shared__ int s_totals[2];
    release_successor();
    wait_for_predecessor();
    // After an earlier report nothing is written.  (The block does not leave: one of its cluster may have found nothing yet, and reads this one's shared
    // memory.)
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
    // n > budget.  Tokens that stay in any case weigh more than all numbers, and places behind the last token less.
    const int from = p.sinks, to = n - p.recent;
    int left = m;  // of those that have the digits of the border so far, how many stay
    const int part = ((n + p.cluster - 1) / p.cluster + 3) & ~3, low = min(rank * part, n), fours = (min(low + part, n) - low + 3) / 4;
    // the weights of four tokens of this block, neighbours in a page
    auto read_four = [&](int i) -> uint4 {
        const int j = low + 4 * i;
        const long long row = place_row(p.pool, p.table, p.width, b, hk, j);
        if (row < 0) report_bad_index(p.status, p.host_status, kBadPage);
        const float4 w = row < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : __ldcg(reinterpret_cast<const float4*>(p.received + row));
        auto order = [&](float x, int j) -> uint32_t {
            return j >= n ? 0u : j < from || j >= to ? 0xffffffffu : min(weight_order(__float_as_uint(x)), 0xfffffffeu);
        };
        return make_uint4(order(w.x, j), order(w.y, j + 1), order(w.z, j + 2), order(w.w, j + 3));
    };
    auto four = [&](int i) -> uint4 {
        if constexpr (kKept) return s_keys[i];
        else return read_four(i);
    };
    for (int i = threadIdx.x; i < 3 * kDigits; i += kSelectThreads) s_count[0][i] = 0;
    for (int i = threadIdx.x; i < 3 * kDigits / 2; i += kSelectThreads) s_sum[0][i] = 0;
    __syncthreads();
    // the digits: bits 21 .. 31, 10 .. 20, 0 .. 9
    constexpr int kAtOnce = 8;  // loads of a thread in flight
    for (int base = threadIdx.x; base < fours; base += kSelectThreads * kAtOnce) {
        uint4 x[kAtOnce];
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y)
            if (base + y * kSelectThreads < fours) x[y] = read_four(base + y * kSelectThreads);
#pragma unroll
        for (int y = 0; y < kAtOnce; ++y) {
            if (base + y * kSelectThreads >= fours) break;
            if constexpr (kKept) s_keys[base + y * kSelectThreads] = x[y];
            atomicAdd(&s_count[0][x[y].x >> 21], 1);
            atomicAdd(&s_count[0][x[y].y >> 21], 1);
            atomicAdd(&s_count[0][x[y].z >> 21], 1);
            atomicAdd(&s_count[0][x[y].w >> 21], 1);
        }
    }
    uint32_t border = 0, known = 0;  // the lightest's digits so far
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
        if (round > 0) {
            const uint32_t mask = round == 1 ? 0x7ffu : 0x3ffu;
#pragma unroll 4
            for (int i = threadIdx.x; i < fours; i += kSelectThreads) {
                const uint4 x = four(i);
                if ((x.x & known) == border) atomicAdd(&s_count[round][x.x >> shift & mask], 1);
                if ((x.y & known) == border) atomicAdd(&s_count[round][x.y >> shift & mask], 1);
                if ((x.z & known) == border) atomicAdd(&s_count[round][x.z >> shift & mask], 1);
                if ((x.w & known) == border) atomicAdd(&s_count[round][x.w >> shift & mask], 1);
            }
        }
        // the counts of all blocks: each block adds up a part of the digits, and reads the others' sums.  (Of the whole cluster's counts a block reads
        // twice its own that way, not eight times.)
        int4 count;  // thread i has the digits from 4 i on
        static_assert(kDigits == 4 * kSelectThreads, "a thread has four digits");
        if (p.cluster == 1) {
            __syncthreads();
            count = *reinterpret_cast<const int4*>(&s_count[round][4 * threadIdx.x]);
        } else {
            const int own = kDigits / p.cluster;
            cluster_sync();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = i * kSelectThreads + static_cast<int>(threadIdx.x), digit = x % own;
                atomicAdd(&s_sum[round][digit], __float_as_int(load_remote(smem_u32(&s_count[round][rank * own + digit]), x / own)));
            }
            cluster_sync();
            count = load_remote_four(smem_u32(&s_sum[round][4 * threadIdx.x % own]), 4 * threadIdx.x / own);
        }
        int2 before;
        const int mine = count.x + count.y + count.z + count.w, all = scan_block(make_int2(mine, 0), s_warp, &before).x, above = all - before.x - mine;
        if (above < left && above + mine >= left) {
            int x = above, i = 3;
            const int of[4] = {count.x, count.y, count.z, count.w};
#pragma unroll
            for (int y = 3; y > 0; --y)
                if (i == y && x + of[y] < left) x += of[y], --i;
            s_digit = 4 * static_cast<int>(threadIdx.x) + i, s_left = left - x;
        }
        __syncthreads();
        border |= static_cast<uint32_t>(s_digit) << shift, known |= (round == 2 ? 0x3ffu : 0x7ffu) << shift;
        left = s_left;
    }
    // Those above the border stay, and `left` of those on it, the first ones.  A warp has neighbouring tokens, four of a lane at a time: it counts them,
    // and when it is known what is in front of them, goes through them again and writes.
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int each = (fours + kSelectThreads / 32 - 1) / (kSelectThreads / 32), first = min(each * warp, fours), end = min(first + each, fours);
    const uint32_t in_front = (1u << lane) - 1;
    auto lane_four = [&](int i) -> uint4 { return i + lane < end ? four(i + lane) : make_uint4(0, 0, 0, 0); };
    int2 mine = make_int2(0, 0), before;
#pragma unroll 4
    for (int i = first; i < end; i += 32) {
        const uint4 x = lane_four(i);
        mine.x += (x.x > border) + (x.y > border) + (x.z > border) + (x.w > border);
        mine.y += (x.x == border) + (x.y == border) + (x.z == border) + (x.w == border);
    }
    const int2 all = scan_block(mine, s_warp, &before);
    before.x = __shfl_sync(0xffffffffu, before.x, 0), before.y = __shfl_sync(0xffffffffu, before.y, 0);
    if (p.cluster > 1) {
        if (threadIdx.x == 0) s_totals[0] = all.x, s_totals[1] = all.y;
        cluster_sync();
#pragma unroll 4
        for (int r = 0; r < rank; ++r) {
            before.x += __float_as_int(load_remote(smem_u32(&s_totals[0]), r));
            before.y += __float_as_int(load_remote(smem_u32(&s_totals[1]), r));
        }
        cluster_sync();  // (no block is gone before the others have read its totals)
    }
    if (quiet) return;
    int at = before.x + min(before.y, left), room = max(left - before.y, 0);  // where the next one goes, and how many on the border still stay
    for (int i = first; i < end; i += 32) {
        const uint4 four_of = lane_four(i);
        const uint32_t x[4] = {four_of.x, four_of.y, four_of.z, four_of.w};
        // on the border: in front of this lane's, and of all lanes
        int same = 0, all_same = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const uint32_t found = __ballot_sync(0xffffffffu, x[y] == border);
            same += __popc(found & in_front), all_same += __popc(found);
        }
        bool stays[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            stays[y] = x[y] > border || (x[y] == border && same < room);
            same += x[y] == border;
        }
        int to_place = at;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const uint32_t found = __ballot_sync(0xffffffffu, stays[y]);
            to_place += __popc(found & in_front), at += __popc(found);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if (stays[y] && to_place < m) kept[to_place] = low + 4 * (i + lane) + y;
            to_place += stays[y];
        }
        room = max(room - all_same, 0);
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
            if constexpr (kE4M3) {
                p.pool.k_exp[to] = __ldcg(reinterpret_cast<const signed char*>(p.pool.k_exp) + from);
                p.pool.v_exp[to] = __ldcg(reinterpret_cast<const signed char*>(p.pool.v_exp) + from);
            }
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

cudaError_t configure_evict() { return cudaFuncSetAttribute(s2a_evict_select_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMostKept * 4); }

cudaError_t launch_evict(EvictParams p, int n_sm, bool e4m3, int d, cudaStream_t stream) {
    const long long longest = static_cast<long long>(p.width) << p.pool.page_log2, units = static_cast<long long>(p.B) * p.pool.Hkv;
    // Blocks of a cluster: as many as there are multiprocessors for, while each has 1024 tokens and more; more of them where their weights fit no other way.
    p.cluster = 1;
    while (p.cluster < kMostBlocks &&
           ((units * p.cluster * 2 <= n_sm && longest > 2048ll * p.cluster) || longest > static_cast<long long>(kMostKept) * p.cluster))
        p.cluster *= 2;
    const long long part = ((longest + p.cluster - 1) / p.cluster + 3) & ~3ll;
    const bool kept = part <= kMostKept;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(units * p.cluster));
    config.blockDim = dim3(kSelectThreads);
    config.dynamicSmemBytes = kept ? static_cast<size_t>(part) * 4 : 0;
    config.stream = stream;
    cudaLaunchAttribute attributes[2] = {};
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = static_cast<unsigned>(p.cluster), attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    config.attrs = attributes, config.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&config, kept ? s2a_evict_select_kernel<true> : s2a_evict_select_kernel<false>, p);
    if (e != cudaSuccess) return e;
    const int most = static_cast<int>(p.budget < longest ? p.budget : longest);  // tokens that a head keeps
    if (e4m3) return d == 64 ? launch_copy<64, true>(p, most, stream) : launch_copy<128, true>(p, most, stream);
    return d == 64 ? launch_copy<128, false>(p, most, stream) : launch_copy<256, false>(p, most, stream);
}

}  // namespace s2a
