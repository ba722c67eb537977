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

// Items are runs of `run` heads of a token: those of q, then of k (and of v).
struct HeadRuns {
    int run, first_k, first_v, count;  // `count` runs of a token, those of k from first_k on, of v from first_v on
    FastDiv by_count;
    HeadRuns() = default;
    HeadRuns(int run_, int H, int Hk, int Hv) : run(run_) {
        first_k = (H + run - 1) / run, first_v = first_k + (Hk + run - 1) / run, count = first_v + (Hv + run - 1) / run;
        by_count = FastDiv(count);
    }
    // run `i` of a token: 0 q, 1 k, 2 v, and its first head
    __host__ __device__ int kind(int i, int* head) const {
        const int kind = i < first_k ? 0 : i < first_v ? 1 : 2;
        *head = (i - (kind == 0 ? 0 : kind == 1 ? first_k : first_v)) * run;
        return kind;
    }
};

struct RotateParams {
    HeadRows in[3];  // q, k, v (the last one where they go into the cache)
    __nv_bfloat16* out[2];
    long long out_stride[2];
    Rotation rotation;
    bool backwards;  // by the negative angles
    HeadRuns runs;
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
    int run[2];               // heads of an item, of either kind
    int blocks[2];            // of the grid, that have q's rows and k's
    FastDiv by_runs[2];
    float* partial;           // [blocks[0] + blocks[1]][d]
    int* status;
};

enum class RotateTo { kTensors, kCacheBf16, kCacheE4M3 };
cudaError_t launch_rotate(const RotateParams& p, RotateTo to, bool norm, int d, cudaStream_t stream);
cudaError_t launch_rotate_bwd(const RotateBwdParams& p, int d, cudaStream_t stream);
int rotate_bwd_blocks(int n_sm);  // of the grid, of both kinds together

}  // namespace s2a
