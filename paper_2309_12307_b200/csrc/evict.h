// What cached tokens weigh, and eviction of the lighter ones: parameter blocks and launchers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "paged.h"
#include "s2a_params.h"

namespace s2a {

// What both weighing kernels take.
struct WeightsParams {
    PagedBatch batch;
    PagedPool pool;
    const __nv_bfloat16* q;  // [T, H, d]
    const float* lse;        // [H, T]
    const float* before;     // [pages, Hkv, page_size] or nullptr
    float* received;         // the same
    int* status;
    int* host_status;
    int H, rep, most_new;
    int window, sinks;       // window 0: none
    int few_rows;            // sequences with at most so many rows are the streaming kernel's, the others the tiling one's
    float scale_log2;        // scale / ln 2 = scale_part * 2^(scale_exp - 127), 1 <= scale_part < 2
    float scale_part;
    int scale_exp;
};

// Rows (new tokens times query heads of a KV head) of a sequence up to which it is the streaming kernel's, unless it is the only one and may have more.
// Both measured (us, streaming and tiling kernel, heads of 128 in bf16; 8 bits in brackets where that differs by more than one):
//   - one sequence, 8 KV heads
//       1000 keys   16 rows 8 and 12, 64 rows 10 and 12 (12 and 12), 128 rows 14 and 12
//       8192 keys   16 rows 14 and 16, 32 rows 16 and 16, 64 rows 21 and 16 (23 and 16)
//       32k keys    16 rows 31 and 33 (27 and 35), 32 rows 33 and 33 (31 and 35), 64 rows 43 and 33 (45 and 35), 256 rows 133 and 35
//   - 8 x 4096 keys, 8 KV heads: 16 rows 31 and 33 (25 and 35), 32 rows 33 and 33 (29 and 35), 64 rows 45 and 33 (43 and 35)
//   - 4 x 4096 keys, heads of 64: 32 rows 23 and 21, 64 rows 29 and 21
constexpr int kStreamedRows = 32;
struct WeightsStreamParams {
    WeightsParams a;
    int chunk_log2;          // keys of a block
    FastDiv by_chunks, by_heads;
    int blocks;
};

constexpr int kWeightKeys = 256;  // of an item of the tiling kernel: two tiles
struct alignas(64) WeightsTileParams {
    CUtensorMap tm_q;        // bf16 (d, H, T), box (64, pack, 128 / pack), 128-byte swizzle
    CUtensorMap tm_k;        // (d, rows of the pool), box (64 values of bf16 or all of a key's codes, min(page_size, 128)), swizzled by the box's width
    WeightsParams a;
    int pack_log2;           // query heads of a KV head that are rows of one tile
    int blocks;              // of kWeightKeys keys that a sequence has at most
    int pieces;              // that the rows of an item are split into at most
    float* partial;          // [blocks][pieces][B * Hkv][kWeightKeys] where there is more than one
    FastDiv by_units, by_pieces, by_heads, by_groups;  // B * Hkv, pieces, Hkv, head groups of a KV head
    int items;               // blocks * pieces * B * Hkv
};

// What an item of the tiling kernel is: keys key0 .. key0 + 255 of a sequence and KV head, against the row tiles r0 .. r1 - 1 of those that attend any of them.
// Row tile r is head group r % groups of the tokens from (t_lo + r / groups) * (128 / pack) on.
struct WeightsItem {
    int id, b, hk;           // b = -1: no more items
    int key0, first, last;   // first key; positions of the sequence's new tokens
    int row0;                // of q, of the first new token
    int t_lo, r0, r1;
    int pieces;              // that this item's rows come in
};
__host__ __device__ inline bool weights_item(const WeightsTileParams& p, int id, WeightsItem* w) {
    int unit, piece;
    w->id = id;
    const int block = p.by_pieces(p.by_units(id, &unit), &piece);
    w->b = p.by_heads(unit, &w->hk);
    Sequence s;
    const WeightsParams& a = p.a;
    if (sequence_of(a.batch, a.pool.page_log2, a.most_new, w->b, &s) != 0 || s.n == 0 || s.n <= a.few_rows / a.rep) return false;
    w->row0 = s.row0, w->first = s.length - s.n, w->last = s.length - 1;
    const KeyBlocks k = key_blocks(w->first, w->last, a.window, a.sinks, kWeightKeys);
    if (block >= k.count) return false;
    w->key0 = k.at(block) * kWeightKeys;
    const int tokens_log2 = 7 - p.pack_log2;
    int high = w->last;  // the last position that attends any of the keys
    if (a.window > 0 && w->key0 >= a.sinks && w->key0 + (kWeightKeys - 1) <= w->last - (a.window - 1)) high = w->key0 + (kWeightKeys - 1) + (a.window - 1);
    const int low = w->key0 > w->first ? w->key0 : w->first;
    if (high < low) return false;
    w->t_lo = (low - w->first) >> tokens_log2;
    const int count = (((high - w->first) >> tokens_log2) - w->t_lo + 1) * (a.rep >> p.pack_log2), each = (count + p.pieces - 1) / p.pieces;
    w->r0 = piece * each;
    w->r1 = w->r0 + each < count ? w->r0 + each : count;
    w->pieces = (count + each - 1) / each;
    return w->r0 < w->r1;
}

struct EvictParams {
    PagedPool pool;
    float* received;
    const int* table;     // [B, width]
    const int* lengths;   // [B]
    const int* to_table;  // [B, to_width]
    int width, to_width, B;
    int budget, sinks, recent;
    int* new_lengths;     // [B]
    int* kept;            // [B, Hkv, budget]
    int cluster;          // blocks of a head in the selecting kernel
    FastDiv by_pieces;    // blocks of a head in the copying kernel
    int* status;
    int* host_status;
};

// Weights in an order of whole numbers: as they are, -0 as 0, NaN above all.
__host__ __device__ inline uint32_t weight_order(uint32_t bits) {
    if ((bits & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    if (bits == 0x80000000u) bits = 0;
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

cudaError_t launch_weights_stream(const WeightsStreamParams& p, bool e4m3, int d, cudaStream_t stream);
cudaError_t launch_weights_tile(const WeightsTileParams& p, bool e4m3, int d, cudaStream_t stream);
cudaError_t configure_weights_tile();
cudaError_t configure_evict();
cudaError_t launch_evict(EvictParams p, int n_sm, bool e4m3, int d, cudaStream_t stream);

}  // namespace s2a
