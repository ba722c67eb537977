// Norms of queries and keys for each head with the rotation of positions: parameter blocks and launchers.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "paged.h"
#include "s2a_params.h"

namespace s2a {

// Tensors of one kind, [T, heads, d] with `stride` values from a token to the next.
struct HeadRows {
    const __nv_bfloat16* x;
    long long stride;
    int heads;
};

struct Rotation {
    const long long* turns;  // [r / 2], of a full turn, in 2^-64, that a position turns a pair by
    const int* positions;    // [n] or nullptr (0, 1, ..): row t has positions[t % n]
    FastDiv by_positions;    // n
    int r;                   // values of a row that are rotated
    bool interleaved;        // pairs (2i, 2i + 1) instead of (i, i + r / 2)
    const void* weight[2];   // [d] of q's norm and k's, or nullptr
    bool weight_f32;         // in fp32 instead of bf16
    float eps;
};

// A block's rows: `rows` heads, one after the other, of a tile of `tokens` tokens (their heads of q, then of k, then of v).
struct RowBlocks {
    int heads[2], all;       // of a token: first one of k, of v; all of them
    int tokens, rows, count; // count: blocks of a tile
    FastDiv by_count, by_heads;
    RowBlocks() = default;
    RowBlocks(int H, int Hk, int Hv, int tokens_, int rows_) : heads{H, H + Hk}, all(H + Hk + Hv), tokens(tokens_), rows(rows_) {
        count = static_cast<int>((static_cast<long long>(tokens) * all + rows - 1) / rows);
        by_count = FastDiv(count), by_heads = FastDiv(all);
    }
    // head `h` of a token: 0 q, 1 k, 2 v, and which of them
    __host__ __device__ int kind(int h, int* head) const {
        const int kind = h < heads[0] ? 0 : h < heads[1] ? 1 : 2;
        *head = h - (kind == 0 ? 0 : heads[kind - 1]);
        return kind;
    }
};

struct RotateParams {
    HeadRows in[3];  // q, k, v (the last one where they go into the cache)
    __nv_bfloat16* out[2];
    long long out_stride[2];
    Rotation rotation;
    bool backwards;  // by the negative angles
    RowBlocks blocks;
    int T;
    // into the cache
    PagedBatch batch;
    PagedPool pool;
    int* status;
    int* host_status;
};

struct RotateBwdParams {
    HeadRows in[2], grad[2];  // q and k, gradients of what came out
    __nv_bfloat16* out[2];    // of what went in, dense
    float* weight_grad[2];    // [d]
    Rotation rotation;
    int T;
    int blocks[2];            // of the grid, that have q's rows and k's
    int tokens[2], chunks[2]; // tokens of a chunk of rows; where one token has more rows than a chunk, its parts are chunks
    FastDiv by_heads[2], by_parts[2];
    float* partial;           // [blocks[0] + blocks[1]][d]
    int* status;
};

enum class RotateTo { kTensors, kCacheBf16, kCacheE4M3 };
cudaError_t launch_rotate(const RotateParams& p, RotateTo to, bool norm, int d, cudaStream_t stream);
cudaError_t configure_rotate();
cudaError_t launch_rotate_bwd(const RotateBwdParams& p, int d, cudaStream_t stream);
int rotate_rows(int d);           // of a block at most
int rotate_bwd_blocks(int n_sm);  // of the grid, of both kinds together
int rotate_bwd_rows(int d);       // of a chunk

}  // namespace s2a
