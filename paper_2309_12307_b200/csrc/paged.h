// The paged cache of keys and values: its layout, where the tokens of a batch lie in it, and the parameter blocks of
// the kernels that write, read and attend it.
//
// A pool holds pages of 2^page_log2 tokens: row (page * Hkv + hk) * page_size + slot is one token of one KV head, d
// values.  So the tokens of a head lie together within a page, and a run of them is one box of a two-dimensional tensor
// map over (d, rows) or one piece of memory.
//
// The new tokens of B sequences are rows starts[b] .. starts[b+1]-1 of one tensor; sequence b has lengths[b] tokens
// in the cache, of which they are the last ones.  table[b * width + i] is the page of its tokens i * page_size on.
// All three arrays are read on the device, so a captured graph follows what they hold when it is replayed, and what
// they hold is checked there: a kernel skips what is out of range and reports it (kBadIndexCode), it never follows it.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "s2a_params.h"

namespace s2a {

// Codes in the device status word for values out of range, beside those of waits that ran out (WaitCode).
constexpr int kBadIndexCode = 1000;
enum BadIndex : int {
    kBadStarts = kBadIndexCode + 1,  // starts out of [0, T] or falling
    kBadLength = kBadIndexCode + 2,  // a length below the sequence's new tokens or above what its row of the table holds
    kBadPage = kBadIndexCode + 3,    // a page that is not in the pool
    kBadNew = kBadIndexCode + 4,     // more new tokens than the caller said a sequence has at most
};

struct PagedBatch {
    const int* table;    // [B, width]
    const int* starts;   // [B + 1]
    const int* lengths;  // [B]
    int width, B, T;
};

struct PagedPool {
    void* k;
    void* v;
    int8_t* k_exp;  // [pages, Hkv, page_size]: value = code * 2^exp, kExpNotFinite = a row that is NaN throughout
    int8_t* v_exp;
    int pages, Hkv, page_log2;
};
constexpr int kExpLeast = -126, kExpNotFinite = -128;

struct Sequence {
    int row0, n, length;  // first row, new tokens, tokens in the cache
};

// Kernels of this library can be resident before their predecessors are done (see launch_kernel), so what those may write is read from the L2.
#if defined(__CUDA_ARCH__)
#define S2A_LOAD(p) __ldcg(p)
#else
#define S2A_LOAD(p) (*(p))
#endif

// Sequence b of the batch; 0, or the code of what is wrong with it (then n = 0).  most_new: new tokens a sequence has at most.
__host__ __device__ inline int sequence_of(const PagedBatch& batch, int page_log2, int most_new, int b, Sequence* s) {
    const int row0 = S2A_LOAD(batch.starts + b), end = S2A_LOAD(batch.starts + b + 1), length = S2A_LOAD(batch.lengths + b);
    s->row0 = row0, s->n = 0, s->length = length;
    if (row0 < 0 || end < row0 || end > batch.T) return kBadStarts;
    if (length < end - row0 || length > static_cast<long long>(batch.width) << page_log2) return kBadLength;
    if (end - row0 > most_new) return kBadNew;
    s->n = end - row0;
    return 0;
}

// The last sequence that starts at or before `row`, which need not reach it.
__host__ __device__ inline int find_sequence(const int* starts, int B, int row) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (S2A_LOAD(starts + mid) <= row) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Where the entries of sequence b begin in the table: past 32 bits in a large one.
__host__ __device__ inline long long table_row(const PagedBatch& batch, int b) { return static_cast<long long>(b) * batch.width; }

// Page of the tokens i * page_size on of sequence b, or -1 where the table holds none of the pool's.
__host__ __device__ inline int page_of(const PagedBatch& batch, int pages, int b, int i) {
    const int page = S2A_LOAD(batch.table + table_row(batch, b) + i);
    return static_cast<unsigned>(page) < static_cast<unsigned>(pages) ? page : -1;
}

// Row of the pools of position `pos` of sequence b in KV head 0 (head hk: + hk << page_log2), or -1.
__host__ __device__ inline long long pool_row(const PagedBatch& batch, const PagedPool& pool, int b, int pos) {
    const int page = page_of(batch, pool.pages, b, pos >> pool.page_log2);
    if (page < 0) return -1;
    return ((static_cast<long long>(page) * pool.Hkv) << pool.page_log2) + (pos & ((1 << pool.page_log2) - 1));
}

// The power of two of a row whose largest magnitude has these bf16 bits: the least e >= kExpLeast with
// max |x| <= 448 * 2^e, 448 = 1.75 * 2^8 being the largest 8-bit float.  A power of two costs nothing (the 8-bit values
// have an exponent of their own, so none of their three bits of fraction is lost) and makes the product with 2^-e, and
// the value that a code stands for, exact: a bf16 value.
__host__ __device__ inline int row_exponent(uint32_t most_bits) {
    if (most_bits >= 0x7f80u) return kExpNotFinite;  // an infinity or a NaN
    const int e = static_cast<int>(most_bits >> 7) - 127 - 8 + ((most_bits & 0x7fu) > 0x60u ? 1 : 0);
    return e < kExpLeast ? kExpLeast : e;
}

struct CacheCopyParams {
    PagedBatch batch;
    PagedPool pool;
    __nv_bfloat16* k;  // [T, Hkv, d]: read by the writing kernel, written by the reading one
    __nv_bfloat16* v;
    int* status;
    int* host_status;
    int tokens_per_block;
    FastDiv by_rows;  // rows of a token: heads of k and of v
};

// The keys that the new tokens at positions first .. last attend, in blocks of `block` keys: with a window the blocks that hold the
// first `sinks` tokens, then those of the window, else all up to the last token.  Numbered from 0: block at(i) for i < count.
struct KeyBlocks {
    int sink_blocks, low_block, count;
    __host__ __device__ int at(int i) const { return i < sink_blocks ? i : low_block + i - sink_blocks; }
};
__host__ __device__ inline KeyBlocks key_blocks(int first, int last, int window, int sinks, int block) {
    KeyBlocks k;
    const int low = window > 0 && first - window + 1 > 0 ? first - window + 1 : 0;
    k.low_block = low / block;
    const int reach = (sinks < low ? sinks : low);
    k.sink_blocks = (reach + block - 1) / block;
    if (k.sink_blocks > k.low_block) k.sink_blocks = k.low_block;
    k.count = k.sink_blocks + last / block + 1 - k.low_block;
    return k;
}
// Whether a token at position `p` attends key j.
__host__ __device__ inline bool attends(int p, int j, int window, int sinks) { return j <= p && (window == 0 || j > p - window || j < sinks); }
// Bit i: whether it attends key j + i.  (No sum of two sizes that are near 2^31.)
__host__ __device__ inline uint32_t attended(int p, int j, int window, int sinks) {
    auto below = [](int n) { return n >= 32 ? 0xffffffffu : n > 0 ? (1u << n) - 1 : 0u; };
    const int ahead = p - j;
    const uint32_t low = window > 0 && ahead >= window ? below(ahead - window + 1) & ~below(sinks - j) : 0u;
    return below(ahead + 1) & ~low;
}
// Whether any of the tokens at positions first .. last does.
__host__ __device__ inline bool any_attends(int first, int last, int j, int window, int sinks) {
    return j <= last && (window == 0 || j > first - window || j < sinks);
}
// Whether the tokens at positions first .. last attend every key from j to j + n - 1.
__host__ __device__ inline bool all_attend(int first, int last, int j, int n, int window, int sinks) {
    return j + n - 1 <= first && (window == 0 || j > last - window || j + n <= sinks);
}
// Of the keys from `key0` on those that none of the tokens at positions first .. last attends, counted from key0: from .. to - 1, in front of their
// windows, and from `end` on.  They may hold anything, and pages that hold no other keys need not be there.
struct HiddenKeys {
    int from, to, end;
    __host__ __device__ bool has(int i) const { return i >= end || (i >= from && i < to); }
    __host__ __device__ bool any(int n) const { return end < n || (from < to && from < n && to > 0); }      // of the first n
    __host__ __device__ bool all(int i, int n) const { return i >= end || (i >= from && i + n <= to); }  // from the i-th on n of them
};
__host__ __device__ inline HiddenKeys hidden_keys(int first, int last, int key0, int window, int sinks) {
    HiddenKeys h;
    h.from = sinks - key0, h.to = window > 0 ? first - window + 1 - key0 : h.from, h.end = last + 1 - key0;
    return h;
}

// Rows (new tokens times query heads of a KV head) up to which a sequence may be worked on by the kernel that splits its keys.
constexpr int kFewRows = 64;

// What both attention kernels take.
struct PagedFwdParams {
    PagedBatch batch;
    PagedPool pool;
    const __nv_bfloat16* q;  // [T, H, d]
    __nv_bfloat16* o;        // [T, H, d]
    float* lse;              // [H, T]
    int* status;
    int* host_status;
    int H, rep, most_new;
    int window, sinks;       // window 0: none
    int few_rows;            // sequences with at most so many rows are the splitting kernel's, the others the other one's
    float scale_log2;                  // scale / ln 2 = scale_power * scale_part, a power of two (2^(scale_field - 127)) and 1 <= scale_part < 2
    float scale_power, scale_part;
    int scale_field;
};

constexpr int kMostSplit = 16;
struct alignas(64) PagedSplitParams {
    CUtensorMap tm_k, tm_v;  // (columns of a line of at most 128 bytes, rows of the pool, lines of a row), box (all, min(page_size, keys of a step), all)
    PagedFwdParams a;
    int warps;               // of a block: 1, 2 or 4
    int blocks, stages;      // blocks of four warps on an SM that the shared memory is divided among, 1 .. 3, and the stages that leaves a warp
    int split;               // blocks of a cluster, which share the keys of a unit: 1 .. kMostSplit
    int unit_rows;           // 8 or 16
    int row_blocks;          // of unit_rows rows, that a sequence and KV head has at most
    FastDiv by_split, by_row_blocks, by_heads, by_rep;
};

// Places of the tiling kernel's work items.  Sequence b has the places from first_slot() on, one for each 2^span_log2 of its tokens;
// first_slot(starts[b + 1], b + 1) leaves it enough of them whatever `starts` are, so the places are known without adding up; there are
// slot_count() of them.
__host__ __device__ inline int first_slot(int row0, int b, int span_log2) { return (row0 >> span_log2) + b; }
__host__ __device__ inline int slot_count(int T, int B, int span_log2) { return first_slot(T - 1, B, span_log2); }
__host__ __device__ inline int find_slot(const int* starts, int B, int span_log2, int slot) {
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = lo + (hi - lo) / 2;
        if (first_slot(S2A_LOAD(starts + mid), mid, span_log2) <= slot) lo = mid;
        else hi = mid;
    }
    return lo;
}

constexpr int kMostRanked = 64;  // sequences of a batch whose items are put in order
struct alignas(64) PagedTileParams {
    CUtensorMap tm_q;        // bf16 (d, H, T), box (64, pack, 128 / pack), 128-byte swizzle
    CUtensorMap tm_k, tm_v;  // V in bf16 (d, rows of the pool), box (64, min(page_size, 128)), swizzled; K the same with the two middle ones of every
                             // four rows exchanged; in 8 bits both (d, rows of the pool), box (d, min(page_size, 128)), not swizzled
    PagedFwdParams a;
    int pack_log2;           // query heads of a KV head that are rows of one tile
    int span_log2;           // tokens of a work item: two tiles, or one (`single`)
    bool single;
    bool ranked;             // the items' order follows the sequences' lengths, see Ranking
    bool beside;             // launched behind the splitting kernel of the same call
    int slots;               // of a head group: slot_count()
    BlockOrder order;        // of items that are not ranked: head groups in chunks, see plan_tiles()
    // Items from first_split on are split: `split` pieces of their keys each, which leave their results in `pieces`.
    int first_split, split;
    float* pieces;
    FastDiv by_split, by_groups, by_groups_of_kv;  // head groups, and those of a KV head: rep / pack
};

// Enqueue on `stream`; return the launch error, if any.
cudaError_t launch_cache_write(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream);
cudaError_t launch_cache_read(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream);
cudaError_t launch_paged_fwd(const PagedTileParams& p, bool e4m3, int d, cudaStream_t stream);
size_t paged_piece_bytes(int d);  // what a piece of a split item leaves
cudaError_t launch_paged_split(const PagedSplitParams& p, bool e4m3, int d, cudaStream_t stream);
int split_keys(bool e4m3, int d);  // keys of a step of a warp of the splitting kernel
int split_stages(bool e4m3, int d, int blocks);
// slots[b][n]: blocks of four warps, meant for b on an SM, that the GPU runs at a time in clusters of n, 1 .. kMostSplit (0: none)
cudaError_t configure_paged_split(int (*slots)[kMostSplit + 1]);
cudaError_t configure_paged_fwd();

}  // namespace s2a
