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
    float scale_log2;        // scale / ln 2
};

struct WeightsStreamParams {
    WeightsParams a;
    int chunk_log2;          // keys of a block
    FastDiv by_chunks, by_heads;
    int blocks;
};

// Tokens of a sequence that are kept, by number or by the weight of the lightest one.
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
cudaError_t launch_evict(const EvictParams& p, bool e4m3, int d, cudaStream_t stream);

}  // namespace s2a
