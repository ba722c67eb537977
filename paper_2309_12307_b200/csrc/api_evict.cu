// Host side of the weights of cached tokens and of eviction (include/s2a.h): argument validation and kernel launches.
#include <float.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/s2a.h"
#include "evict.h"
#include "host_paged.h"
#include "host_state.h"

namespace s2a {
namespace {

constexpr long long kIntMax = 0x7fffffffLL;

// The device, set up for these kernels.
int prepare_evict(DeviceState** ds) {
    const int rc = prepare_device(ds);
    return rc != S2A_OK || (*ds)->evict_error == cudaSuccess ? rc : cuda_fail((*ds)->evict_error);
}

// Blocks of `keys` keys that the new tokens of a sequence together attend at most.
long long most_chunks(const WeightsParams& a, long long longest, int keys) {
    const long long all = (longest + keys - 1) / keys;
    if (a.window == 0) return all;
    return std::min(all, (static_cast<long long>(a.sinks) + keys - 1) / keys + (static_cast<long long>(a.window) + a.most_new + keys - 1) / keys + 1);
}

// Keys of a block of the streaming kernel: as many as leave eight blocks for a multiprocessor, so that each reads its rows of q for many keys.
bool plan_stream(WeightsStreamParams* p, int n_sm, long long longest) {
    const long long units = static_cast<long long>(p->a.batch.B) * p->a.pool.Hkv;
    int log2 = 10;
    while (log2 > 6 && units * most_chunks(p->a, longest, 1 << log2) < 8ll * n_sm) --log2;
    const long long chunks = most_chunks(p->a, longest, 1 << log2);
    if (units * chunks > kIntMax) return false;
    p->chunk_log2 = log2, p->by_chunks = FastDiv(static_cast<int>(chunks)), p->by_heads = FastDiv(p->a.pool.Hkv), p->blocks = static_cast<int>(units * chunks);
    return true;
}

// The items of the tiling kernel and the pieces their rows come in.  Without a window the first key blocks have all rows and the last ones few, and the
// longest item must not be longer than the others together: a piece has about a quarter of a multiprocessor's share of all row tiles, eight at least (an item's
// start and the second launch cost about as much as three).  Measured, whole and in pieces, us, one prompt at once on 32 heads over 8 of 128: 512 tokens
// 31 and 23, 1024 51 and 25, 2048 92 and 41, 4096 176 and 98; 512 new of 16,384 96 and 94.
bool plan_tile(WeightsTileParams* p, int n_sm, long long longest) {
    const WeightsParams& a = p->a;
    p->pack_log2 = 0;
    while (p->pack_log2 < 6 && a.rep % (2 << p->pack_log2) == 0) ++p->pack_log2;
    const int groups = a.rep >> p->pack_log2, tokens = kTile >> p->pack_log2;
    const long long units = static_cast<long long>(a.batch.B) * a.pool.Hkv, blocks = most_chunks(a, longest, kWeightKeys);
    long long attending = a.most_new;  // tokens that attend a key
    if (a.window > 0) attending = std::min(attending, static_cast<long long>(a.window) + kWeightKeys);
    const long long most_tiles = (attending + tokens - 1) / tokens * groups;
    const double likely = static_cast<double>(a.batch.T) / a.batch.B / a.most_new;  // of most_new, that an average sequence has
    const double all = 0.75 * static_cast<double>(units) * static_cast<double>(blocks) * static_cast<double>(most_tiles) * std::min(1.0, likely);
    const double each = std::max(8.0, all / (4.0 * n_sm));
    p->pieces = static_cast<int>(std::min<double>(16.0, std::max(1.0, ceil(static_cast<double>(most_tiles) / each))));
    if (units * blocks > kIntMax / 16) return false;
    p->blocks = static_cast<int>(blocks), p->items = static_cast<int>(units * blocks) * p->pieces;
    p->by_units = FastDiv(static_cast<int>(units)), p->by_pieces = FastDiv(p->pieces), p->by_heads = FastDiv(a.pool.Hkv), p->by_groups = FastDiv(groups);
    return true;
}

void set_pieces(WeightsTileParams* p, int pieces) {
    p->items = p->items / p->pieces * pieces, p->pieces = pieces, p->by_pieces = FastDiv(pieces);
}

size_t tile_bytes(const WeightsTileParams& p) { return p.pieces > 1 ? static_cast<size_t>(p.items) * kWeightKeys * sizeof(float) : 0; }

int weights_tmaps(WeightsTileParams* p, const s2a_cache* c, const void* q, int H, int T) {
    const cuuint64_t d = static_cast<cuuint64_t>(c->d);
    const cuuint64_t q_dims[3] = {d, static_cast<cuuint64_t>(H), static_cast<cuuint64_t>(T)}, q_strides[2] = {2 * d, 2 * d * H};
    const cuuint32_t q_box[3] = {64, 1u << p->pack_log2, static_cast<cuuint32_t>(kTile) >> p->pack_log2};
    const int rc = encode_tmap(&p->tm_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_SWIZZLE_128B, q, 3, q_dims, q_strides, q_box);
    if (rc != S2A_OK) return rc;
    const bool codes = c->type == S2A_CACHE_E4M3;
    const cuuint64_t dims[2] = {d, static_cast<cuuint64_t>(c->pages) * c->Hkv * c->page_size}, stride = codes ? d : 2 * d;
    const cuuint32_t box[2] = {codes ? static_cast<cuuint32_t>(d) : 64, static_cast<cuuint32_t>(std::min(c->page_size, kTile))};
    return encode_tmap(&p->tm_k, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                       codes && d == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, c->k, 2, dims, &stride, box);
}

// What a call's sizes say; its pointers and the scale are still missing.
WeightsParams weights_params(const s2a_cache* cache, const s2a_batch* batch, int H, int max_new, int window, int sinks) {
    WeightsParams a;
    memset(&a, 0, sizeof a);
    const int longest = batch->width * cache->page_size;  // no sequence has more tokens
    a.batch = batch_of(batch), a.pool = pool_of(cache);
    a.H = H, a.rep = H / cache->Hkv, a.most_new = max_new;
    a.window = window >= longest ? 0 : window, a.sinks = sinks > longest ? longest : sinks;
    // (kStreamedRows has the measurements.)  A single sequence has as many new tokens as it is said to have at most, but for loose values
    a.few_rows = batch->B == 1 && static_cast<long long>(max_new) * a.rep > kStreamedRows ? 0 : kStreamedRows;
    return a;
}

}  // namespace
}  // namespace s2a

using namespace s2a;

#pragma GCC visibility push(default)
extern "C" {

int s2a_paged_weights(const void* q, const float* lse, const s2a_cache* cache, const s2a_batch* batch, const float* before, float* received, int H,
                      int max_new, float scale, int window, int sinks, void* workspace, size_t workspace_bytes, void* stream) {
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return S2A_ERR_INVALID_ARG;
    if (!q || !lse || !received || !aligned16(q) || !aligned16(lse) || !aligned16(before) || !aligned16(received)) return S2A_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != S2A_OK || (rc = check_batch(batch, cache)) != S2A_OK) return rc;
    if (!(scale > 0.f) || !isfinite(scale)) return S2A_ERR_INVALID_ARG;
    if ((rc = check_heads(cache, batch, H, max_new, window, sinks)) != S2A_OK) return rc;
    DeviceState* ds = nullptr;
    if ((rc = prepare_evict(&ds)) != S2A_OK || (rc = standing_status(ds)) != S2A_OK) return rc;
    WeightsParams a = weights_params(cache, batch, H, max_new, window, sinks);
    a.q = static_cast<const __nv_bfloat16*>(q), a.lse = lse, a.before = before, a.received = received;
    a.status = ds->status_ptr, a.host_status = ds->host_word_dev;
    a.scale_log2 = std::min(scale * 1.4426950408889634f, FLT_MAX);
    const float half_part = frexpf(a.scale_log2, &a.scale_exp);  // 0.5 <= half_part < 1
    a.scale_part = 2 * half_part, a.scale_exp += 126;
    const bool e4m3 = cache->type == S2A_CACHE_E4M3, few = a.rep <= a.few_rows, many = static_cast<long long>(max_new) * a.rep > a.few_rows;
    const long long longest = static_cast<long long>(batch->width) * cache->page_size;
    // everything that can be refused comes before the first launch
    WeightsStreamParams ps;
    memset(&ps, 0, sizeof ps);
    ps.a = a;
    if (few && !plan_stream(&ps, ds->n_sm, longest)) return S2A_ERR_UNSUPPORTED;
    WeightsTileParams pt;
    memset(&pt, 0, sizeof pt);
    pt.a = a;
    if (many) {
        if (!plan_tile(&pt, ds->n_sm, longest)) return S2A_ERR_UNSUPPORTED;
        if (!workspace || tile_bytes(pt) > workspace_bytes) set_pieces(&pt, 1);
        pt.partial = static_cast<float*>(workspace);
        if ((rc = weights_tmaps(&pt, cache, q, H, batch->T)) != S2A_OK) return rc;
    }
    cudaError_t e = cudaSuccess;
    if (few) e = launch_weights_stream(ps, e4m3, cache->d, static_cast<cudaStream_t>(stream));
    if (many && e == cudaSuccess) e = launch_weights_tile(pt, e4m3, cache->d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

size_t s2a_paged_weights_workspace_bytes(const s2a_cache* cache, const s2a_batch* batch, int H, int max_new, int window, int sinks) {
    DeviceState* ds = nullptr;
    if (check_cache(cache) != S2A_OK || check_batch(batch, cache) != S2A_OK || check_heads(cache, batch, H, max_new, window, sinks) != S2A_OK) return 0;
    WeightsTileParams p;
    memset(&p, 0, sizeof p);
    p.a = weights_params(cache, batch, H, max_new, window, sinks);
    if (static_cast<long long>(max_new) * p.a.rep <= p.a.few_rows || prepare_evict(&ds) != S2A_OK) return 0;
    return plan_tile(&p, ds->n_sm, static_cast<long long>(batch->width) * cache->page_size) ? tile_bytes(p) : 0;
}

int s2a_cache_evict(const s2a_cache* cache, float* received, const int* table, int width, const int* lengths, const int* to_table, int to_width, int B,
                    int budget, int sinks, int recent, int* new_lengths, int* kept, void* stream) {
    int rc = check_cache(cache);
    if (rc != S2A_OK) return rc;
    if (!received || !aligned16(received) || !table || !lengths || !to_table || !new_lengths || !kept) return S2A_ERR_INVALID_ARG;
    if (B <= 0 || width <= 0 || to_width <= 0 || budget <= 0 || sinks < 0 || recent < 0) return S2A_ERR_INVALID_ARG;
    if (static_cast<long long>(sinks) + recent > budget) return S2A_ERR_INVALID_ARG;
    // (every head's block reads its sequence's length; one of them writes the new one)
    if (new_lengths < lengths + B && lengths < new_lengths + B) return S2A_ERR_INVALID_ARG;
    const long long longest = static_cast<long long>(width) * cache->page_size, room = static_cast<long long>(to_width) * cache->page_size;
    if (longest > kIntMax / 2 || room > kIntMax / 2 || budget > kIntMax / 2) return S2A_ERR_UNSUPPORTED;  // (places, and steps beyond them, are ints)
    if (room < std::min<long long>(budget, longest)) return S2A_ERR_INVALID_ARG;
    if (static_cast<long long>(B) * cache->Hkv > kIntMax / 16 / ((std::min<long long>(budget, longest) + 15) / 16)) return S2A_ERR_UNSUPPORTED;
    DeviceState* ds = nullptr;
    if ((rc = prepare_evict(&ds)) != S2A_OK || (rc = standing_status(ds)) != S2A_OK) return rc;
    EvictParams p;
    memset(&p, 0, sizeof p);
    p.pool = pool_of(cache), p.received = received, p.table = table, p.lengths = lengths, p.to_table = to_table;
    p.width = width, p.to_width = to_width, p.B = B, p.budget = budget, p.sinks = sinks, p.recent = recent;
    p.new_lengths = new_lengths, p.kept = kept, p.status = ds->status_ptr, p.host_status = ds->host_word_dev;
    const cudaError_t e = launch_evict(p, ds->n_sm, cache->type == S2A_CACHE_E4M3, cache->d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

}  // extern "C"
#pragma GCC visibility pop
