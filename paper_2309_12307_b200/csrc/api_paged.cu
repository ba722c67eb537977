// Host side of the paged cache's part of include/s2a.h: argument validation and kernel launches.
#include <float.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "../../include/s2a.h"
#include "host_paged.h"
#include "host_state.h"
#include "paged.h"
#include "s2a_params.h"

namespace s2a {

namespace {
constexpr long long kIntMax = 0x7fffffffLL;
}  // namespace

int check_cache(const s2a_cache* c) {
    if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return S2A_ERR_INVALID_ARG;
    if (c->type != S2A_CACHE_BF16 && c->type != S2A_CACHE_E4M3) return S2A_ERR_INVALID_ARG;
    if (c->type == S2A_CACHE_E4M3 && (!c->k_exp || !c->v_exp || !aligned16(c->k_exp) || !aligned16(c->v_exp))) return S2A_ERR_INVALID_ARG;
    if (c->pages <= 0 || c->Hkv <= 0 || c->page_size <= 0 || c->d <= 0) return S2A_ERR_INVALID_ARG;
    if (c->d != 64 && c->d != 128) return S2A_ERR_UNSUPPORTED;
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)) != 0) return S2A_ERR_UNSUPPORTED;
    if (static_cast<long long>(c->pages) * c->Hkv > kIntMax / c->page_size) return S2A_ERR_UNSUPPORTED;
    return S2A_OK;
}

int check_batch(const s2a_batch* b, const s2a_cache* c) {
    if (!b || !b->table || !b->starts || !b->lengths) return S2A_ERR_INVALID_ARG;
    if (b->B <= 0 || b->T <= 0 || b->width <= 0) return S2A_ERR_INVALID_ARG;
    if (static_cast<long long>(b->T) * 2 * c->Hkv > kIntMax || static_cast<long long>(b->width) * c->page_size > kIntMax / 2) return S2A_ERR_UNSUPPORTED;
    return S2A_OK;
}

int check_heads(const s2a_cache* cache, const s2a_batch* batch, int H, int max_new, int window, int sinks) {
    if (H <= 0 || H % cache->Hkv != 0 || max_new <= 0 || max_new > batch->T || window < 0 || sinks < 0) return S2A_ERR_INVALID_ARG;
    return static_cast<long long>(batch->T) * H > kIntMax ? S2A_ERR_UNSUPPORTED : S2A_OK;
}

PagedBatch batch_of(const s2a_batch* b) {
    PagedBatch r;
    r.table = b->table, r.starts = b->starts, r.lengths = b->lengths, r.width = b->width, r.B = b->B, r.T = b->T;
    return r;
}

PagedPool pool_of(const s2a_cache* c) {
    PagedPool r;
    r.k = c->k, r.v = c->v, r.k_exp = reinterpret_cast<int8_t*>(c->k_exp), r.v_exp = reinterpret_cast<int8_t*>(c->v_exp);
    r.pages = c->pages, r.Hkv = c->Hkv, r.page_log2 = 0;
    while ((1 << r.page_log2) < c->page_size) ++r.page_log2;
    return r;
}

namespace {

// The rows of a pool, as lines of 128 bytes (or of a row, where that is less); a box is `keys` rows, or a page where that is less, one line after
// the other.  See swizzled() for how a line's box lies in shared memory.
int cache_tmap(CUtensorMap* tm, const s2a_cache* c, const void* pool, int keys) {
    const bool codes = c->type == S2A_CACHE_E4M3;
    const cuuint32_t size = codes ? 1 : 2, row_bytes = static_cast<cuuint32_t>(c->d) * size, line = row_bytes < 128 ? row_bytes : 128;
    const cuuint64_t dims[3] = {line / size, static_cast<cuuint64_t>(c->pages) * c->Hkv * c->page_size, row_bytes / line};
    const cuuint64_t strides[2] = {row_bytes, line};
    const cuuint32_t box[3] = {line / size, static_cast<cuuint32_t>(c->page_size < keys ? c->page_size : keys), row_bytes / line};
    return encode_tmap(tm, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, line < 128 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                       pool, 3, dims, strides, box);
}

// The tensor maps of the tiling kernel, see PagedTileParams.
int tile_tmaps(PagedTileParams* p, const s2a_cache* c, const void* q, int H, int T) {
    const cuuint64_t d = static_cast<cuuint64_t>(c->d), rows = static_cast<cuuint64_t>(c->pages) * c->Hkv * c->page_size;
    const cuuint32_t keys = static_cast<cuuint32_t>(c->page_size < kTile ? c->page_size : kTile);
    const cuuint64_t q_dims[3] = {d, static_cast<cuuint64_t>(H), static_cast<cuuint64_t>(T)}, q_strides[2] = {2 * d, 2 * d * H};
    const cuuint32_t q_box[3] = {64, 1u << p->pack_log2, static_cast<cuuint32_t>(kTile) >> p->pack_log2};
    int rc = encode_tmap(&p->tm_q, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_SWIZZLE_128B, q, 3, q_dims, q_strides, q_box);
    if (rc != S2A_OK) return rc;
    const cuuint64_t dims[2] = {d, rows};
    if (c->type == S2A_CACHE_E4M3) {
        const cuuint32_t box[2] = {static_cast<cuuint32_t>(d), keys};
        rc = encode_tmap(&p->tm_k, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_NONE, c->k, 2, dims, &d, box);
        return rc != S2A_OK ? rc : encode_tmap(&p->tm_v, CU_TENSOR_MAP_DATA_TYPE_UINT8, CU_TENSOR_MAP_SWIZZLE_NONE, c->v, 2, dims, &d, box);
    }
    const cuuint64_t row_bytes = 2 * d;
    const cuuint32_t box[2] = {64, keys};
    const cuuint64_t k_dims[4] = {d, 2, 2, rows / 4}, k_strides[3] = {2 * row_bytes, row_bytes, 4 * row_bytes};
    const cuuint32_t k_box[4] = {64, 2, 2, keys / 4};
    rc = encode_tmap(&p->tm_k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_SWIZZLE_128B, c->k, 4, k_dims, k_strides, k_box);
    return rc != S2A_OK ? rc : encode_tmap(&p->tm_v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, CU_TENSOR_MAP_SWIZZLE_128B, c->v, 2, dims, &row_bytes, box);
}

// Bytes of a token's k and v of a head.
int key_bytes(const s2a_cache* c) { return c->type == S2A_CACHE_E4M3 ? 2 * c->d + 2 : 4 * c->d; }

// Keys that `tokens` tokens of a sequence together attend at most, of `longest`.
long long reach_of(const PagedFwdParams& a, long long longest, int tokens) {
    const long long most = static_cast<long long>(a.window) + a.sinks + tokens;
    return a.window > 0 && most < longest ? most : longest;
}

// How the keys of the units (8 or 16 rows of a sequence and KV head) are dealt out: blocks of `warps` warps, `split` of them in a cluster
// for each unit, whatever should be done first by this estimate, in microseconds.
//   - All units' bytes at the memory's rate.  A batch's sequences differ in length: the average is taken as 0.7 of the longest.
//   - What a piece takes: a block of four warps needs 13 ns (8 bits: 10) for a key of 128 columns when it is alone on its multiprocessor, 1.23
//     times that beside another one and 1.6 times beside two.  Blocks of a batch end about half of the longest piece's time apart.  Of a
//     single sequence all pieces are alike and run in waves.
//   - 8 us for every block that a place on the GPU sees: the launch, the addresses, the first loads' latency, joining the results.
// Measured (us, by blocks in a cluster, of four warps): 16 x up to 8192 tokens of 32 heads of 128 1 190, 2 170, 3 171, 4 181; 8 x up to 32k of 8 heads
// in 8 bits 4 117, 6 94, 8 96, 10 88, 12 99; 16 x up to 32k of 8 heads in 8 bits 4 136, 6 114, 8 126; 4 x 8192 of 40 heads 2 112, 3 126, 4 104, 6 115;
// one of 100,000 of 32 heads in 8 bits 4 255, 6 198, 7 172, 8 153, 9 171, 10 155, 12 201, in bf16 4 356, 6 267, 7 243, 8 263, 10 256; 64 x up to 1024 of 32
// heads, one block of two warps 89, of four 92.
void choose_pieces(PagedSplitParams* p, const DeviceState* ds, long long reach, int key_bytes, bool e4m3, int d) {
    const long long units = static_cast<long long>(p->a.batch.B) * p->a.pool.Hkv * p->row_blocks;
    const double rate = 6.5e6, block_start = 8.0;  // bytes in a microsecond, microseconds
    const double key_time = (e4m3 ? 0.010 : 0.013) * d / 128, beside[4] = {0, 1.0, 1.23, 1.6};
    double best = 0;
    p->warps = 4, p->split = 1, p->blocks = 3;
    for (int warps = 4; warps >= 1; warps /= 2)
        for (int split = 1; split <= kMostSplit; ++split) {
            const long long blocks = units * split;
            auto slots = [&](int on_sm) { return static_cast<long long>(ds->cluster_slots[on_sm][split]) * (4 / warps); };
            if (slots(3) <= 0 || (split > 1 && reach <= static_cast<long long>(split - 1) * warps * split_keys(e4m3, d))) continue;
            auto on_sm = [&](long long n) { return n <= slots(1) ? 1 : n <= slots(2) ? 2 : 3; };  // blocks beside one another when n run
            const double piece = static_cast<double>((reach + split - 1) / split), alone = piece * key_time * 4 / warps;
            double t;
            if (p->a.batch.B > 1) {
                const double waves = static_cast<double>(blocks) / slots(3);
                t = 0.7 * units * reach * key_bytes / rate + 0.5 * alone + block_start * (waves < 1 ? 1 : waves);
            } else {
                auto wave = [&](long long n) {
                    const double bytes = n * piece * key_bytes / rate, work = alone * beside[on_sm(n)];
                    return n == 0 ? 0 : (bytes > work ? bytes : work) + block_start;
                };
                t = static_cast<double>(blocks / slots(3)) * wave(slots(3)) + wave(blocks % slots(3));
            }
            if (best == 0 || t < best) best = t, p->warps = warps, p->split = split, p->blocks = on_sm(blocks);
        }
    p->stages = split_stages(e4m3, d, p->blocks);  // where fewer blocks run at a time, each has more in flight
}

// The items of the tiling kernel: how many rows and tokens one has, in which order they come and into how many pieces of its keys each is split,
// whatever should be done first.  Counted in steps of 128 keys of a pair, 1.8 us and more: a single tile's takes four fifths of it (1024 new
// tokens of 8192 on 32 heads: as 128 pairs 128 us, as 256 single tiles 201), so single tiles are for what the GPU works on at a time.  The
// start and end of an item or piece take two steps, a second launch five and a tenth for every piece, and what pieces leave goes to the L2 and
// back at 6.5 MB a microsecond.  A batch's sequences are taken to have the same number of new tokens.  Measured, one sequence, without
// this splitting and with it: 1024 new tokens of 16,384 on 40 heads (160 pairs, in three) 422 us and 324; 257 of 23,219 on 16 heads over 8 in
// 8 bits as 40 single tiles in three 131, as 24 pairs in six 90.
// (Splitting the items of the last, partial wave alone brings nothing: with fewer multiprocessors busy those run at a higher
// clock.  2048 new tokens of 8192 on 32 heads 246 us without and 263 with it, of 32k on 64 over 8 2.09 and 2.06 ms.)
bool plan_tiles(PagedTileParams* p, int n_sm, long long longest, int d, int key_bytes) {
    const PagedFwdParams& a = p->a;
    p->pack_log2 = 0;
    while (p->pack_log2 < 6 && a.rep % (2 << p->pack_log2) == 0) ++p->pack_log2;
    const long long groups = a.H >> p->pack_log2;
    p->ranked = a.batch.B > 1 && a.batch.B <= kMostRanked;
    double best = 0;
    int best_split = 1;
    for (const bool single : {false, true}) {
        const int span_log2 = 7 - p->pack_log2 + (single ? 0 : 1), slots = slot_count(a.batch.T, a.batch.B, span_log2);
        const int likely = std::min(slots, a.batch.B * (((a.batch.T + a.batch.B - 1) / a.batch.B + (1 << span_log2) - 1) >> span_log2));
        const long long items = slots * groups, busy = likely * groups;
        const int tiles = static_cast<int>((reach_of(a, longest, 1 << span_log2) + kTile - 1) / kTile);
        if (single && items > n_sm) break;
        for (int split = 1; split <= kMostSplit && split <= tiles; ++split) {
            if (split > 1 && (a.batch.B > kMostRanked || items * split > 4 * n_sm)) break;
            double t = static_cast<double>((busy * split + n_sm - 1) / n_sm) * ((tiles + split - 1) / split + 2) * (single ? 0.8 : 1.0);
            if (split > 1) t += 5 + 0.1 * split + 2.0 * busy * split * paged_piece_bytes(d) / 6.5e6 / 1.8;
            if (best != 0 && t > (split > 1 ? 0.95 : 1.0) * best) continue;
            best = t, best_split = split;
            p->single = single, p->span_log2 = span_log2, p->slots = slots;
        }
    }
    const long long items = p->slots * groups;
    if (items * kMostSplit > 0x7fffffffLL) return false;
    p->split = best_split, p->first_split = best_split > 1 ? 0 : static_cast<int>(items);
    // The last items to begin should be short ones, so the head groups are taken in chunks that together have an item for every multiprocessor, all
    // chunks alike, as far as the keys of a chunk leave half of the L2.  (One sequence, a group at a time and so: 8192 tokens on 32 heads of 64
    // 415 us and 373, of 128 454 and 422; 2048 of 8192 204 and 200.  Without a look at the L2, 2048 of 65,536 1755 and 1890.)
    const double group_bytes = static_cast<double>(reach_of(a, longest, a.batch.T)) * key_bytes / (a.rep >> p->pack_log2);
    const int room = static_cast<int>(std::min<double>(static_cast<double>(groups), std::max(1.0, 64e6 / group_bytes)));
    int chunk = std::min(room, (n_sm + p->slots - 1) / p->slots);
    for (const int least = chunk; groups % chunk != 0;) {
        if (chunk < least || ++chunk > room) chunk = std::min(chunk, least) - 1;
    }
    p->order = BlockOrder(static_cast<int>(groups), p->slots, chunk);
    p->by_groups = FastDiv(static_cast<int>(groups)), p->by_groups_of_kv = FastDiv(a.rep >> p->pack_log2);
    return true;
}

// Up to how many rows (new tokens times query heads of a KV head) a sequence is the splitting kernel's.  Each 16 rows of a sequence
// read its keys again there, and make legacy tensor products of them; the tiling kernel does all 128 rows of a tile at once, but starts and
// joins more slowly.  Up to 16 rows are the former's and more than 64 never.  Between them the tiling kernel takes batches with many keys to
// read: `visits`, of a key by 16 rows of an average sequence.  Measured, in us, splitting and tiling kernel, heads of 128:
//   - one sequence, 8 KV heads: 32 rows, 1000 15 and 21, 8000 26 and 24 (8 bits 26 and 28), 16,000 40 and 31, 32k 63 and 48, 100,000 160 and 87 (8 bits 157 and
//     111); 64 rows, 1000 16 and 21, 4000 25 and 21; 32 KV heads, 8192, in 8 bits: 20 rows 49 and 52, 40 rows 64 and 52
//   - several, 8 KV heads: 32 rows, 2 x 2000 20 and 23, 4 x 4000 31 and 33 (8 bits 34 and 38), 2 x 8000 in 8 bits 55 and 37, 16 x 2000 77 and 37; 64 rows, 4 x 1000
//     26 and 22, 4 x 4000 70 and 36
//   - heads of 64: 4 x 1000, 24 rows 13 and 22, 32 x 4000 104 and 97, 2 x 32,000, 20 rows 70 and 57; in 8 bits, one of 24,700, 40 KV heads, 22 rows 88 and 121
//   - 6 x 16,700, 1 to 20 rows, 10 on average, in 8 bits 146 and 187.
// With both kernels a call takes 5 to 8 us longer, so where no sequence has more than 64 rows the tiling kernel takes them all.
int few_rows(long long most_rows, long long all_rows, long long reach, int B, int Hkv, int d, bool e4m3) {
    if (most_rows <= 16) return 16;
    if (B == 1 && most_rows > kFewRows) return 0;
    const double rows = static_cast<double>(all_rows) / B < kFewRows ? static_cast<double>(all_rows) / B : kFewRows;
    const double visits = static_cast<double>(B) * Hkv * ceil(rows / 16) * reach * d / 128;
    if (rows <= (e4m3 && d == 64 ? 32 : 16) || visits < 1 << 18) return kFewRows;
    return most_rows <= kFewRows ? 0 : 16;
}

// What a call's sizes say; its pointers and the scale are still missing.
PagedFwdParams fwd_params(const s2a_cache* cache, const s2a_batch* batch, int H, int max_new, int window, int sinks) {
    PagedFwdParams p;
    memset(&p, 0, sizeof p);
    p.batch = batch_of(batch), p.pool = pool_of(cache);
    const int longest = batch->width * cache->page_size;  // no sequence has more tokens
    p.H = H, p.rep = H / cache->Hkv, p.most_new = max_new;
    p.window = window >= longest ? 0 : window, p.sinks = sinks > longest ? longest : sinks;
    p.few_rows = few_rows(static_cast<long long>(max_new) * p.rep, static_cast<long long>(batch->T) * p.rep, reach_of(p, longest, max_new), batch->B, cache->Hkv, cache->d, cache->type == S2A_CACHE_E4M3);
    return p;
}

int copy_impl(void* k, void* v, const s2a_cache* cache, const s2a_batch* batch, void* stream, bool write) {
    if (!k || !v || !aligned16(k) || !aligned16(v)) return S2A_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != S2A_OK) return rc;
    if ((rc = check_batch(batch, cache)) != S2A_OK) return rc;
    DeviceState* ds = nullptr;
    if ((rc = prepare_device(&ds)) != S2A_OK) return rc;
    if ((rc = standing_status(ds)) != S2A_OK) return rc;
    CacheCopyParams p;
    memset(&p, 0, sizeof p);
    p.batch = batch_of(batch), p.pool = pool_of(cache);
    p.k = static_cast<__nv_bfloat16*>(k), p.v = static_cast<__nv_bfloat16*>(v);
    p.status = ds->status_ptr, p.host_status = ds->host_word_dev;
    const auto launch = write ? launch_cache_write : launch_cache_read;
    const cudaError_t e = launch(p, cache->type == S2A_CACHE_E4M3, cache->d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

}  // namespace
}  // namespace s2a

using namespace s2a;

#pragma GCC visibility push(default)
extern "C" {

int s2a_cache_write(const void* k, const void* v, const s2a_cache* cache, const s2a_batch* batch, void* stream) {
    return copy_impl(const_cast<void*>(k), const_cast<void*>(v), cache, batch, stream, true);
}

int s2a_cache_read(const s2a_cache* cache, const s2a_batch* batch, void* k, void* v, void* stream) {
    return copy_impl(k, v, cache, batch, stream, false);
}

int s2a_paged_fwd(const void* q, const s2a_cache* cache, const s2a_batch* batch, void* o, float* lse, int H, int max_new, float scale,
                  int window, int sinks, void* workspace, size_t workspace_bytes, void* stream) {
    if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return S2A_ERR_INVALID_ARG;
    if (!q || !o || !lse || !aligned16(q) || !aligned16(o) || !aligned16(lse)) return S2A_ERR_INVALID_ARG;
    int rc = check_cache(cache);
    if (rc != S2A_OK) return rc;
    if ((rc = check_batch(batch, cache)) != S2A_OK) return rc;
    if (!(scale > 0.f) || !isfinite(scale)) return S2A_ERR_INVALID_ARG;
    if ((rc = check_heads(cache, batch, H, max_new, window, sinks)) != S2A_OK) return rc;
    DeviceState* ds = nullptr;
    if ((rc = prepare_paged(&ds)) != S2A_OK) return rc;
    if ((rc = standing_status(ds)) != S2A_OK) return rc;
    const bool e4m3 = cache->type == S2A_CACHE_E4M3;
    const int longest = batch->width * cache->page_size;  // no sequence has more tokens
    const long long most_rows = static_cast<long long>(max_new) * (H / cache->Hkv);
    PagedFwdParams p = fwd_params(cache, batch, H, max_new, window, sinks);
    p.q = static_cast<const __nv_bfloat16*>(q), p.o = static_cast<__nv_bfloat16*>(o), p.lse = lse;
    p.status = ds->status_ptr, p.host_status = ds->host_word_dev;
    p.scale_log2 = std::min(scale * 1.4426950408889634f, FLT_MAX);  // (a score of zero times infinity would be NaN)
    const float half_part = frexpf(p.scale_log2, &p.scale_field);  // 0.5 <= half_part < 1
    p.scale_part = 2 * half_part, p.scale_field += 126, p.scale_power = ldexpf(1.f, p.scale_field - 127);
    // everything that can be refused comes before the first launch
    const bool few = p.few_rows > 0, many = most_rows > p.few_rows;
    PagedSplitParams ps;
    memset(&ps, 0, sizeof ps);
    if (few) {
        ps.a = p;
        if ((rc = cache_tmap(&ps.tm_k, cache, cache->k, split_keys(e4m3, cache->d))) != S2A_OK) return rc;
        if ((rc = cache_tmap(&ps.tm_v, cache, cache->v, split_keys(e4m3, cache->d))) != S2A_OK) return rc;
        ps.unit_rows = most_rows <= 8 ? 8 : 16;
        ps.row_blocks = static_cast<int>((most_rows < p.few_rows ? most_rows : p.few_rows) + ps.unit_rows - 1) / ps.unit_rows;
        choose_pieces(&ps, ds, reach_of(p, longest, max_new), key_bytes(cache), e4m3, cache->d);
        if (static_cast<long long>(batch->B) * cache->Hkv * ps.row_blocks * ps.split > kIntMax) return S2A_ERR_UNSUPPORTED;
        ps.by_split = FastDiv(ps.split), ps.by_row_blocks = FastDiv(ps.row_blocks), ps.by_heads = FastDiv(cache->Hkv), ps.by_rep = FastDiv(p.rep);
    }
    PagedTileParams pt;
    memset(&pt, 0, sizeof pt);
    if (many) {
        pt.a = p;
        if (!plan_tiles(&pt, ds->n_sm, longest, cache->d, key_bytes(cache))) return S2A_ERR_UNSUPPORTED;
        pt.beside = few;
        const size_t items = static_cast<size_t>(pt.slots) * (H >> pt.pack_log2);
        if (!workspace || (items - pt.first_split) * pt.split * paged_piece_bytes(cache->d) > workspace_bytes) pt.first_split = static_cast<int>(items), pt.split = 1;
        pt.pieces = static_cast<float*>(workspace);
        pt.by_split = FastDiv(pt.split);
        if ((rc = tile_tmaps(&pt, cache, q, H, batch->T)) != S2A_OK) return rc;
    }
    cudaError_t e = cudaSuccess;
    if (few) e = launch_paged_split(ps, e4m3, cache->d, static_cast<cudaStream_t>(stream));
    if (many && e == cudaSuccess) e = launch_paged_fwd(pt, e4m3, cache->d, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? S2A_OK : cuda_fail(e);
}

size_t s2a_paged_workspace_bytes(const s2a_cache* cache, const s2a_batch* batch, int H, int max_new, int window, int sinks) {
    DeviceState* ds = nullptr;
    if (check_cache(cache) != S2A_OK || check_batch(batch, cache) != S2A_OK || check_heads(cache, batch, H, max_new, window, sinks) != S2A_OK) return 0;
    PagedTileParams p;
    memset(&p, 0, sizeof p);
    p.a = fwd_params(cache, batch, H, max_new, window, sinks);
    if (static_cast<long long>(max_new) * p.a.rep <= p.a.few_rows || prepare_paged(&ds) != S2A_OK) return 0;
    if (!plan_tiles(&p, ds->n_sm, static_cast<long long>(batch->width) * cache->page_size, cache->d, key_bytes(cache))) return 0;
    return (static_cast<size_t>(p.slots) * (H >> p.pack_log2) - p.first_split) * p.split * paged_piece_bytes(cache->d);
}

}  // extern "C"
#pragma GCC visibility pop
