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

}  // namespace
}  // namespace s2a

using namespace s2a;

#pragma GCC visibility push(default)
extern "C" {

int s2a_paged_weights(const void* q, const float* lse, const s2a_cache* cache, const s2a_batch* batch, const float* before, float* received, int H,
                      int max_new, float scale, int window, int sinks, void* stream) {
    if (!q || !lse || !received || !aligned16(q) || !aligned16(lse) || !aligned16(before) || !aligned16(received)) return S2A_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != S2A_OK || (rc = check_batch(batch, cache)) != S2A_OK) return rc;
    if (!(scale > 0.f) || !isfinite(scale)) return S2A_ERR_INVALID_ARG;
    if ((rc = check_heads(cache, batch, H, max_new, window, sinks)) != S2A_OK) return rc;
    DeviceState* ds = nullptr;
    if ((rc = prepare_device(&ds)) != S2A_OK || (rc = standing_status(ds)) != S2A_OK) return rc;
    WeightsStreamParams p;
    memset(&p, 0, sizeof p);
    const int longest = batch->width * cache->page_size;  // no sequence has more tokens
    p.a.batch = batch_of(batch), p.a.pool = pool_of(cache);
    p.a.q = static_cast<const __nv_bfloat16*>(q), p.a.lse = lse, p.a.before = before, p.a.received = received;
    p.a.status = ds->status_ptr, p.a.host_status = ds->host_word_dev;
    p.a.H = H, p.a.rep = H / cache->Hkv, p.a.most_new = max_new;
    p.a.window = window >= longest ? 0 : window, p.a.sinks = sinks > longest ? longest : sinks;
    p.a.few_rows = 0x7fffffff;
    p.a.scale_log2 = std::min(scale * 1.4426950408889634f, FLT_MAX);
    if (!plan_stream(&p, ds->n_sm, longest)) return S2A_ERR_UNSUPPORTED;
    const cudaError_t e = launch_weights_stream(p, cache->type == S2A_CACHE_E4M3, cache->d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
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
    if (longest > kIntMax / 2 || room > kIntMax / 2) return S2A_ERR_UNSUPPORTED;
    if (room < std::min<long long>(budget, longest)) return S2A_ERR_INVALID_ARG;
    if (static_cast<long long>(B) * cache->Hkv > kIntMax / ((std::min<long long>(budget, longest) + 15) / 16)) return S2A_ERR_UNSUPPORTED;
    DeviceState* ds = nullptr;
    if ((rc = prepare_device(&ds)) != S2A_OK || (rc = standing_status(ds)) != S2A_OK) return rc;
    EvictParams p;
    memset(&p, 0, sizeof p);
    p.pool = pool_of(cache), p.received = received, p.table = table, p.lengths = lengths, p.to_table = to_table;
    p.width = width, p.to_width = to_width, p.B = B, p.budget = budget, p.sinks = sinks, p.recent = recent;
    p.new_lengths = new_lengths, p.kept = kept, p.status = ds->status_ptr, p.host_status = ds->host_word_dev;
    const cudaError_t e = launch_evict(p, cache->type == S2A_CACHE_E4M3, cache->d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

}  // extern "C"
#pragma GCC visibility pop
