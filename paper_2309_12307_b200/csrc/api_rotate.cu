// Host side of the rotation's part of include/s2a.h: argument validation and kernel launches.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/s2a.h"
#include "host_paged.h"
#include "host_state.h"
#include "rotate.h"

namespace s2a {
namespace {

constexpr long long kIntMax = 0x7fffffffLL;
constexpr long long kMostStride = 1 << 28;  // (64 tokens of it, in eights, and the place of a head in a token, fit an int)

// `x` [T, heads, d] with `stride` values from a token to the next
int check_rows(const void* x, long long stride, int T, int heads, int d) {
    if (!x || !aligned16(x) || heads <= 0) return S2A_ERR_INVALID_ARG;
    const long long dense = static_cast<long long>(heads) * d;
    if (T == 1) return dense > kMostStride ? S2A_ERR_UNSUPPORTED : S2A_OK;
    if (stride % 8 != 0 || stride < dense) return S2A_ERR_INVALID_ARG;
    return stride > kMostStride ? S2A_ERR_UNSUPPORTED : S2A_OK;
}

int check_rotation(const s2a_rotation* ro, int d, bool counted) {
    if (!ro || ro->r < 0 || ro->r > d || (ro->r > 0 && !ro->turns)) return S2A_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(ro->turns) & 7u) != 0 || (reinterpret_cast<uintptr_t>(ro->positions) & 3u) != 0) return S2A_ERR_INVALID_ARG;
    if ((ro->positions || counted) && ro->n_positions <= 0) return S2A_ERR_INVALID_ARG;
    if (ro->interleaved != 0 && ro->interleaved != 1) return S2A_ERR_INVALID_ARG;
    if (ro->norm != 0 && ro->norm != 1) return S2A_ERR_INVALID_ARG;
    if (ro->norm) {
        if (ro->weight_type != S2A_WEIGHT_BF16 && ro->weight_type != S2A_WEIGHT_F32) return S2A_ERR_INVALID_ARG;
        if (!aligned16(ro->q_weight) || !aligned16(ro->k_weight) || !(ro->eps >= 0.f) || !isfinite(ro->eps)) return S2A_ERR_INVALID_ARG;
    } else if (ro->q_weight || ro->k_weight) {
        return S2A_ERR_INVALID_ARG;
    }
    return ro->r % 16 != 0 ? S2A_ERR_UNSUPPORTED : S2A_OK;
}

int check_sizes(int T, int H, int Hkv, int d) {
    if (T <= 0 || H <= 0 || Hkv <= 0 || d <= 0) return S2A_ERR_INVALID_ARG;
    if (d != 64 && d != 128) return S2A_ERR_UNSUPPORTED;
    return static_cast<long long>(T) * (static_cast<long long>(H) + 2 * static_cast<long long>(Hkv)) > kIntMax ? S2A_ERR_UNSUPPORTED : S2A_OK;
}

Rotation rotation_of(const s2a_rotation* ro) {
    Rotation r;
    memset(&r, 0, sizeof r);
    r.turns = ro->turns, r.positions = ro->positions, r.by_positions = FastDiv(ro->n_positions), r.r = ro->r, r.interleaved = ro->interleaved != 0;
    if (ro->norm) r.weight[0] = ro->q_weight, r.weight[1] = ro->k_weight, r.weight_f32 = ro->weight_type == S2A_WEIGHT_F32, r.eps = ro->eps;
    return r;
}

HeadRows rows_of(const void* x, long long stride, int heads) {
    HeadRows r;
    r.x = static_cast<const __nv_bfloat16*>(x), r.stride = stride, r.heads = heads;
    return r;
}

// The blocks of a launch: of few tokens the heads are spread over more blocks, two for each multiprocessor.
RowBlocks blocks_of(int T, int H, int Hk, int Hv, int d, int n_sm) {
    const int all = H + Hk + Hv, most = rotate_rows(d);
    int rows = most;
    while (rows > most / 4 && static_cast<long long>(T) * all < static_cast<long long>(rows) * 2 * n_sm) rows /= 2;
    // a tile has as many tokens as fill its blocks, up to 16
    int tokens = std::max(1, rows / all), best = tokens;
    auto full = [&](int n) { return static_cast<double>(n) * all / ((static_cast<long long>(n) * all + rows - 1) / rows * rows); };
    for (; tokens <= 16 && tokens <= T; ++tokens)
        if (full(tokens) > full(best) + 0.02) best = tokens;
    return RowBlocks(H, Hk, Hv, best, rows);
}

// One kernel for the forward pass, and for gradients that go through no norm.
int rotate_impl(const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, long long q_out_stride, void* k_out, long long k_out_stride,
                const s2a_rotation* rotation, bool backwards, int T, int H, int Hkv, int d, void* stream) {
    DeviceState* ds = nullptr;
    int rc = prepare_device(&ds);
    if (rc != S2A_OK || (rc = standing_status(ds)) != S2A_OK) return rc;
    RotateParams p;
    memset(&p, 0, sizeof p);
    p.in[0] = rows_of(q, q_stride, H), p.in[1] = rows_of(k, k_stride, Hkv);
    p.out[0] = static_cast<__nv_bfloat16*>(q_out), p.out[1] = static_cast<__nv_bfloat16*>(k_out);
    p.out_stride[0] = q_out_stride, p.out_stride[1] = k_out_stride;
    p.rotation = rotation_of(rotation), p.backwards = backwards, p.T = T;
    p.blocks = blocks_of(T, H, Hkv, 0, d, ds->n_sm);
    p.status = ds->status_ptr, p.host_status = ds->host_word_dev;
    const cudaError_t e = launch_rotate(p, RotateTo::kTensors, rotation->norm != 0 && !backwards, d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

// The blocks of the backward's grid that have q's rows and k's: in proportion to what their chunks cost, at least one each, no more than there are chunks.
// (A chunk of k's few heads has more tokens, so more sines and cosines: with 16 of them it takes 1.25 times as long as with 2.)
void bwd_blocks(RotateBwdParams* p, int n_sm, int d) {
    const int all = rotate_bwd_blocks(n_sm);
    double cost[2];
    for (int x = 0; x < 2; ++x) {
        const int heads = p->in[x].heads, rows = rotate_bwd_rows(d), parts = (heads + rows - 1) / rows;
        p->tokens[x] = std::min(4096 / d, std::max(1, rows / heads));  // (two chunks' sines and cosines in 32 KB)
        p->chunks[x] = (p->T + p->tokens[x] - 1) / p->tokens[x] * parts;
        p->by_heads[x] = FastDiv(heads), p->by_parts[x] = FastDiv(parts);
        cost[x] = p->chunks[x] * (1 + p->tokens[x] * d / (64.0 * 128));
    }
    const int of_q = std::min(all - 1, std::max(1, static_cast<int>(all * cost[0] / (cost[0] + cost[1]))));
    p->blocks[0] = std::min(of_q, p->chunks[0]), p->blocks[1] = std::min(all - of_q, p->chunks[1]);
}

size_t bwd_bytes(int n_sm, int d) { return static_cast<size_t>(rotate_bwd_blocks(n_sm)) * d * sizeof(float); }

}  // namespace
}  // namespace s2a

using namespace s2a;

#pragma GCC visibility push(default)
extern "C" {

int s2a_rotate(const void* q, long long q_stride, const void* k, long long k_stride, void* q_out, long long q_out_stride, void* k_out,
               long long k_out_stride, const s2a_rotation* rotation, int T, int H, int Hkv, int d, void* stream) {
    int rc = check_sizes(T, H, Hkv, d);
    if (rc != S2A_OK) return rc;
    if ((rc = check_rows(q, q_stride, T, H, d)) != S2A_OK || (rc = check_rows(k, k_stride, T, Hkv, d)) != S2A_OK) return rc;
    if ((rc = check_rows(q_out, q_out_stride, T, H, d)) != S2A_OK || (rc = check_rows(k_out, k_out_stride, T, Hkv, d)) != S2A_OK) return rc;
    if ((rc = check_rotation(rotation, d, true)) != S2A_OK) return rc;
    return rotate_impl(q, q_stride, k, k_stride, q_out, q_out_stride, k_out, k_out_stride, rotation, false, T, H, Hkv, d, stream);
}

int s2a_rotate_bwd(const void* q, long long q_stride, const void* k, long long k_stride, const void* dq_out, long long dq_out_stride, const void* dk_out,
                   long long dk_out_stride, void* dq, void* dk, float* dq_weight, float* dk_weight, const s2a_rotation* rotation, int T, int H, int Hkv,
                   int d, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_sizes(T, H, Hkv, d);
    if (rc != S2A_OK) return rc;
    const long long q_dense = static_cast<long long>(H) * d, k_dense = static_cast<long long>(Hkv) * d;
    if ((rc = check_rows(dq_out, dq_out_stride, T, H, d)) != S2A_OK || (rc = check_rows(dk_out, dk_out_stride, T, Hkv, d)) != S2A_OK) return rc;
    if ((rc = check_rows(dq, q_dense, T, H, d)) != S2A_OK || (rc = check_rows(dk, k_dense, T, Hkv, d)) != S2A_OK) return rc;
    if ((rc = check_rotation(rotation, d, true)) != S2A_OK) return rc;
    if (!rotation->norm) {
        if (dq_weight || dk_weight) return S2A_ERR_INVALID_ARG;
        return rotate_impl(dq_out, dq_out_stride, dk_out, dk_out_stride, dq, q_dense, dk, k_dense, rotation, true, T, H, Hkv, d, stream);
    }
    if ((rc = check_rows(q, q_stride, T, H, d)) != S2A_OK || (rc = check_rows(k, k_stride, T, Hkv, d)) != S2A_OK) return rc;
    if (!aligned16(dq_weight) || !aligned16(dk_weight) || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return S2A_ERR_INVALID_ARG;
    DeviceState* ds = nullptr;
    if ((rc = prepare_device(&ds)) != S2A_OK) return rc;
    if (ds->rotate_error != cudaSuccess) return cuda_fail(ds->rotate_error);
    if (workspace_bytes < bwd_bytes(ds->n_sm, d)) return S2A_ERR_INVALID_ARG;
    if ((rc = standing_status(ds)) != S2A_OK) return rc;
    RotateBwdParams p;
    memset(&p, 0, sizeof p);
    p.in[0] = rows_of(q, q_stride, H), p.in[1] = rows_of(k, k_stride, Hkv);
    p.grad[0] = rows_of(dq_out, dq_out_stride, H), p.grad[1] = rows_of(dk_out, dk_out_stride, Hkv);
    p.out[0] = static_cast<__nv_bfloat16*>(dq), p.out[1] = static_cast<__nv_bfloat16*>(dk);
    p.weight_grad[0] = dq_weight, p.weight_grad[1] = dk_weight;
    p.rotation = rotation_of(rotation), p.T = T;
    bwd_blocks(&p, ds->n_sm, d);
    p.partial = static_cast<float*>(workspace), p.status = ds->status_ptr;
    const cudaError_t e = launch_rotate_bwd(p, d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

size_t s2a_rotate_bwd_workspace_bytes(int d) {
    DeviceState* ds = nullptr;
    return (d == 64 || d == 128) && prepare_device(&ds) == S2A_OK ? bwd_bytes(ds->n_sm, d) : 0;
}

int s2a_rotate_write(const void* q, long long q_stride, const void* k, long long k_stride, const void* v, long long v_stride, void* q_out,
                     const s2a_rotation* rotation, const s2a_cache* cache, const s2a_batch* batch, int H, void* stream) {
    int rc = check_cache(cache);
    if (rc != S2A_OK || (rc = check_batch(batch, cache)) != S2A_OK) return rc;
    const int T = batch->T, Hkv = cache->Hkv, d = cache->d;
    if ((rc = check_sizes(T, H, Hkv, d)) != S2A_OK) return rc;
    if ((rc = check_rows(q, q_stride, T, H, d)) != S2A_OK || (rc = check_rows(k, k_stride, T, Hkv, d)) != S2A_OK) return rc;
    if ((rc = check_rows(v, v_stride, T, Hkv, d)) != S2A_OK || (rc = check_rows(q_out, static_cast<long long>(H) * d, T, H, d)) != S2A_OK) return rc;
    if ((rc = check_rotation(rotation, d, false)) != S2A_OK) return rc;
    DeviceState* ds = nullptr;
    if ((rc = prepare_device(&ds)) != S2A_OK || (rc = standing_status(ds)) != S2A_OK) return rc;
    RotateParams p;
    memset(&p, 0, sizeof p);
    p.in[0] = rows_of(q, q_stride, H), p.in[1] = rows_of(k, k_stride, Hkv), p.in[2] = rows_of(v, v_stride, Hkv);
    p.out[0] = static_cast<__nv_bfloat16*>(q_out), p.out_stride[0] = static_cast<long long>(H) * d;
    p.rotation = rotation_of(rotation), p.T = T;
    p.blocks = blocks_of(T, H, Hkv, Hkv, d, ds->n_sm);
    p.batch = batch_of(batch), p.pool = pool_of(cache);
    p.status = ds->status_ptr, p.host_status = ds->host_word_dev;
    const RotateTo to = cache->type == S2A_CACHE_E4M3 ? RotateTo::kCacheE4M3 : RotateTo::kCacheBf16;
    const cudaError_t e = launch_rotate(p, to, rotation->norm != 0, d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

}  // extern "C"
#pragma GCC visibility pop
