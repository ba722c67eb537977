// Attention of few rows over the paged cache: sequences with one new token, or a handful.
//
// A row is a new token and a query head; the rows of a sequence and KV head (new tokens times query heads of a KV head) read the
// same keys.  With few of them, at most 64, the work is reading the cache: 2 d multiply-adds for each row and key against 4 d
// bytes of bf16 for the key.  So the keys are split: a unit, 8 or 16 rows of one sequence and KV head, is worked on by a cluster of blocks, each
// with a share of the keys, its warps taking 16 or 32 keys in turn.  A warp has a ring of its own that TMA fills, a
// running maximum and sum for its rows and the weighted sum of v in registers.  What the warps and then the blocks have is
// joined through shared memory and the cluster's: no second launch, no workspace, no atomics.
//
// Products of a warp, with the keys and the columns of V as the 16 rows of an mma.sync product and the rows of the unit as its 8 columns
// (twice where there are more than 8): S^T = K Q^T, O^T += V^T P^T.  Which columns of a head go into which product does not matter as
// long as K and Q agree, so a thread takes what lies together in shared memory.
//
// Cached 8-bit floats become fp16, which has them all (one conversion for two values; as bf16 they take five instructions).  Q, in bf16, goes
// to fp16, each row with a power of two that brings its largest value near fp16's: nothing is lost of values within 2^-29 of it, and no row
// reaches another (with one power for the unit 8 x 32k tokens of 8 heads take the same 87.5 us).  The row's power of two and K's multiply the scores.
// V's goes into the exponents of the weights: with x a score in units of log2 and 2^e V's power the weight of the second product is
// 2^(x + e - r + 7), r a running maximum of x + e.  So the largest term has a weight of 2^7 or more, those down to 2^-21 of it have all of
// fp16's 11 bits (bf16 has 8), and O is in units of 2^(r - 7); the sum of weights takes an exponential of its own.
#include "paged_device.cuh"

namespace s2a {

namespace {

template <int HD, bool kE4M3>
struct SplitCfg {
    static constexpr int kMostWarps = 4;
    static constexpr int kRowBytes = HD * (kE4M3 ? 1 : 2);        // a key's row
    static constexpr int kKeys = kRowBytes == 256 ? 16 : 32;      // keys of a warp's step
    static constexpr int kLine = kRowBytes < 128 ? kRowBytes : 128;  // bytes of a row in one box
    static constexpr int kBoxes = kRowBytes / kLine;
    static constexpr int kTile = kKeys * kRowBytes;               // K or V of a step
    static constexpr int kStageBytes = 2 * kTile;
    static constexpr int kExpBytes = kE4M3 ? 2 * kKeys : 0;       // exponents of K and V
    // A warp's ring: 16 KB where three blocks of four warps are on an SM, 24 KB for two, 48 KB for one, so that what is in flight there is the
    // same 192 KB (a token over 100,000 of 32 heads in 8 bits, 256 blocks: 16 KB 193 us, 24 KB 154).
    static constexpr int ring_bytes(int blocks) { return blocks == 3 ? 16384 : blocks == 2 ? 24576 : 49152; }
    static constexpr int stages(int blocks) { return ring_bytes(blocks) / kStageBytes; }
    static constexpr int smem_bytes(int blocks, int warps) {  // rings, exponents, barriers, the abort flag
        return warps * (ring_bytes(blocks) + stages(blocks) * (kExpBytes + 8)) + 16;
    }
    static constexpr int kPartFloats = 16 * HD + 4 * 16;          // a warp's result: O, m, l, and the joined m, l
    static_assert(kPartFloats * 4 <= ring_bytes(3), "the ring holds a result");
    static_assert(ring_bytes(3) % kStageBytes == 0 && ring_bytes(2) % kStageBytes == 0, "whole stages");
    static_assert(kTile % 1024 == 0, "swizzle atoms");
};

// 16 bytes of shared memory, as loaded by TMA with a swizzle over the tile's lines
template <int kLine>
__device__ __forceinline__ uint32_t swizzled(uint32_t tile, int row, int byte) {
    const uint32_t at = static_cast<uint32_t>(row * kLine + byte);
    return tile + (kLine == 128 ? at ^ ((at >> 3) & 0x70u) : at ^ ((at >> 3) & 0x30u));
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a));
    return r;
}
__device__ __forceinline__ int lds_s8(uint32_t a) {
    int r;
    asm volatile("ld.shared.s8 %0, [%1];" : "=r"(r) : "r"(a));
    return r;
}
// x * 2^e, x > 0 and |e| <= 250, no larger than fp32's largest number: scores of zero are multiplied with it too.  (In two steps towards the result: a
// step of the other sign could lose bits that the result has.)
__device__ __forceinline__ float score_factor(float x, int e) {
    const int half = e >> 1;
    return fminf(x * power_of_two(half) * power_of_two(e - half), 3.40282347e38f);
}
// 2^e times `by`, likewise; NaN for kExpNotFinite.
__device__ __forceinline__ float key_factor(int e, float by) {
    return e == kExpNotFinite ? __uint_as_float(0x7fffffffu) : fminf(power_of_two(e) * by, 3.40282347e38f);
}

constexpr float kLazy = 8.0f;        // a running maximum (of log2) that is exceeded by less stays

// kWindow: whether the call has one.  (Pages in front of a window are not asked for; where every call looks, one token over 100,000 of 32 heads in
// 8 bits takes 159 us instead of 155, 8 x up to 32k of 8 heads 88.2 instead of 87.7.)
template <int HD, bool kE4M3, int kRowTiles, bool kWindow>
__global__ void __launch_bounds__(32 * SplitCfg<HD, kE4M3>::kMostWarps, 3) s2a_paged_split_kernel(const __grid_constant__ PagedSplitParams p) {
    using C = SplitCfg<HD, kE4M3>;
    constexpr int kRows = 8 * kRowTiles;     // of a unit
    extern __shared__ __align__(1024) uint8_t smem[];
    const PagedFwdParams& a = p.a;
    const int window = kWindow ? a.window : 0;
    const int warps = p.warps, threads = 32 * warps;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int stages = p.stages, ring_bytes = stages * C::kStageBytes;
    uint8_t* ring = smem + warp * ring_bytes;
    uint8_t* exps = smem + warps * ring_bytes + warp * (stages * C::kExpBytes);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + warps * stages * (C::kStageBytes + C::kExpBytes)) + warp * stages;
    volatile int& abort_flag = *reinterpret_cast<volatile int*>(smem + warps * stages * (C::kStageBytes + C::kExpBytes + 8));

    if (lane == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(&full[s], 1);
        fence_barrier_init();
        tma_prefetch_desc(&p.tm_k);
        tma_prefetch_desc(&p.tm_v);
    }
    if (threadIdx.x == 0) abort_flag = 0;
    __syncthreads();
    wait_for_predecessor();
    release_successor();  // (not before: the tiling kernel of the same call relies on what this one has waited for)
    const int standing = *reinterpret_cast<volatile int*>(a.status);
    if (blockIdx.x == 0) check_batch(a.batch, a.pool.page_log2, a.most_new, a.status, a.host_status);
    const WaitCtx ctx{&abort_flag, a.status, a.host_status};

    int part, row_block, hk;
    const int unit = p.by_split(static_cast<int>(blockIdx.x), &part);
    const int b = p.by_heads(p.by_row_blocks(unit, &row_block), &hk);
    Sequence s;
    if (sequence_of(a.batch, a.pool.page_log2, a.most_new, b, &s) != 0) return;  // (the same for all blocks of the cluster)
    const int all_rows = s.n * a.rep, r0 = row_block * kRows;
    if (r0 >= all_rows || all_rows > a.few_rows) return;
    const int rows = all_rows - r0 < kRows ? all_rows - r0 : kRows;
    const int first_pos = s.length - s.n + p.by_rep(r0), last_pos = s.length - s.n + p.by_rep(r0 + rows - 1);
    const KeyBlocks blocks = key_blocks(first_pos, last_pos, window, a.sinks, C::kKeys);
    const int share = (blocks.count + p.split - 1) / p.split;
    const int i0 = part * share + warp, i1 = (part + 1) * share < blocks.count ? (part + 1) * share : blocks.count;
    int steps = i0 < i1 ? (i1 - i0 + warps - 1) / warps : 0;
    // an earlier report: nothing is read or written, but every block of a cluster goes on to the end with the others
    if (__any_sync(0xffffffffu, standing != 0)) {
        steps = 0;
        if (lane == 0) abort_flag = standing;
    }

    // ---- loads of this warp: lane 0 (and 1, where a step spans two pages) requests, and has looked up the page of the next step before
    constexpr int kKeysLog2 = C::kKeys == 16 ? 4 : 5;
    const int piece_log2 = a.pool.page_log2 < kKeysLog2 ? a.pool.page_log2 : kKeysLog2;
    // Looked up in every lane and looked at when it is used: otherwise its latency is a part of every step (one token over 100,000 in 8 bits 172 us
    // instead of 154).
    int next_page = 0, next_key = 0;  // entry of the table, and the key that it is for
    auto look_up = [&](int c) {
        next_key = blocks.at(i0 + c * warps) * C::kKeys + (lane << piece_log2);
        const int at = (next_key < last_pos ? next_key : last_pos) >> a.pool.page_log2;
        next_page = S2A_LOAD(a.batch.table + table_row(a.batch, b) + at);
    };
    auto request = [&](int c, int st) {
        int row = -1;  // of the pool: what this lane requests
        if (lane < C::kKeys >> piece_log2 && !hidden_keys(first_pos, last_pos, 0, window, a.sinks).all(next_key, 1 << piece_log2)) {
            if (static_cast<unsigned>(next_page) < static_cast<unsigned>(a.pool.pages))
                row = ((next_page * a.pool.Hkv + hk) << a.pool.page_log2) + (next_key & ((1 << a.pool.page_log2) - 1));
            else
                report_bad_index(a.status, a.host_status, kBadPage);
        }
        const int boxes = __popc(__ballot_sync(0xffffffffu, row >= 0));
        if (lane == 0) mbar_expect_tx(&full[st], static_cast<uint32_t>(boxes * (2 * C::kRowBytes + (kE4M3 ? 2 : 0))) << piece_log2);
        __syncwarp();
        if (row >= 0) {
            const uint32_t bar = smem_u32(&full[st]), dst = smem_u32(ring + st * C::kStageBytes) + ((lane << piece_log2) * C::kLine);
            tma_load_3d(dst, &p.tm_k, bar, 0, row, 0);
            tma_load_3d(dst + C::kTile, &p.tm_v, bar, 0, row, 0);
            if constexpr (kE4M3) {
                uint8_t* e = exps + st * C::kExpBytes + (lane << piece_log2);
                bulk_load_1d(e, a.pool.k_exp + row, 1u << piece_log2, &full[st]);
                bulk_load_1d(e + C::kKeys, a.pool.v_exp + row, 1u << piece_log2, &full[st]);
            }
        }
        look_up(c + 1);
        __syncwarp();
    };
    look_up(0);
    for (int c = 0; c < stages && c < steps; ++c) request(c, c);

    // ---- Q: row g of every eight, of every 64 columns (of all, in 8 bits) the quarter t, as pairs in the order of K's words
    constexpr int kPer = kE4M3 ? HD / 4 : 16;  // columns that lie together
    uint32_t q[kRowTiles][HD / 8];
    int pos[kRowTiles][2];  // positions of the rows 2 t and 2 t + 1 of every eight
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r) {
        auto row_of = [&](int x, int* hh) {  // rows past the end follow the last one
            const int row = 8 * r + x < rows ? 8 * r + x : rows - 1;
            return p.by_rep(r0 + row, hh);
        };
        int hh;
        pos[r][0] = s.length - s.n + row_of(2 * t, &hh), pos[r][1] = s.length - s.n + row_of(2 * t + 1, &hh);
        const int i = row_of(g, &hh);
        const __nv_bfloat16* src = a.q + (static_cast<long long>(s.row0 + i) * a.H + hk * a.rep + hh) * HD + kPer * t;
#pragma unroll
        for (int c = 0; c < HD / 32; ++c) {
            const uint4 w = __ldcg(reinterpret_cast<const uint4*>(src + 8 * c + (c * 8 / kPer) * (64 - kPer) * (kE4M3 ? 0 : 1)));
            q[r][4 * c] = w.x, q[r][4 * c + 1] = w.y, q[r][4 * c + 2] = w.z, q[r][4 * c + 3] = w.w;
        }
    }
    // 8 bits: a product c, at most 2^30, is a score after a multiplication with its key's power of two, 2^(exponent - off_key), and then one with its
    // row's and the scale, 2^(off_key - up) * scale.  With off_key = 23 the first leaves at most 2^127 and loses nothing that the second would bring above
    // 2^-23, whatever the rows beside this one are.  (It is less where a row or the scale is so large that its factor would be out of range: queries from
    // about 2^122 on.)
    float row_scale[kRowTiles][2];
    float key_scale = 1.f;
    if constexpr (kE4M3) {
        int up[kRowTiles], least_up = 112;  // exponent of row 8 r + g
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
            uint32_t most = 0;
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) most = max(most, max(q[r][c] & 0x7fffu, q[r][c] >> 16 & 0x7fffu));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1)), most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // the largest goes to [2^14, 2^15), or as near as 2^112 brings it, with which 2^-133, the least bf16 number, is one of fp16
            up[r] = most == 0 ? 112 : most >= 0x7f80u ? 0 : min(127 + 14 - static_cast<int>(most >> 7), 112);  // (a row that is not finite stays so)
            const float f = power_of_two(up[r]);
#pragma unroll
            for (int c = 0; c < HD / 8; ++c) q[r][c] = pack_f16(bf16_low(q[r][c]) * f, bf16_high(q[r][c]) * f);
            least_up = min(least_up, up[r]);
        }
        const int off_key = min(23, static_cast<int>(__reduce_min_sync(0xffffffffu, least_up)) + 126 + 127 - a.scale_field);
        key_scale = power_of_two(-off_key);
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
            for (int h = 0; h < 2; ++h) row_scale[r][h] = score_factor(a.scale_log2, off_key - __shfl_sync(0xffffffffu, up[r], 4 * (2 * t + h)));
    }

    float o[kRowTiles][HD / 16][4] = {};
    float m[kRowTiles][2], l[kRowTiles][2];  // running maximum in use and this thread's part of the sum, rows 2 t and 2 t + 1
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r) m[r][0] = m[r][1] = kLeast, l[r][0] = l[r][1] = 0.f;
    float delta[kRowTiles][2] = {};  // 8 bits: r - m, see above.  (Not r: near 2^24 the power of V would be lost in it.)
    bool ok = true;
    int c = 0, st = 0, phase = 0;  // step, its stage, and which use of the stage it is (odd or even)
    for (; c < steps; ++c) {
        if (!mbar_wait_uniform(&full[st], phase, ctx, kWaitPagedSplit + 1)) { ok = false; break; }
        const uint32_t sK = smem_u32(ring + st * C::kStageBytes), sV = sK + C::kTile, sE = smem_u32(exps + st * C::kExpBytes);
        const int key0 = blocks.at(i0 + c * warps) * C::kKeys;
        const bool masked = !all_attend(first_pos, last_pos, key0, C::kKeys, window, a.sinks);
        constexpr int kTiles = C::kKeys / 16;
        float sc[kTiles][kRowTiles][4];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r) sc[u][r][0] = sc[u][r][1] = sc[u][r][2] = sc[u][r][3] = 0.f;
            const int key = 16 * u + g;
            auto product = [&](int k, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
                for (int r = 0; r < kRowTiles; ++r) mma_16x8x16<kE4M3>(sc[u][r], a0, a1, a2, a3, q[r][2 * k], q[r][2 * k + 1]);
            };
            if constexpr (kE4M3) {
#pragma unroll
                for (int x = 0; x < HD / 64; ++x) {
                    const uint4 w = lds128(swizzled<C::kLine>(sK, key, HD / 4 * t + 16 * x)), z = lds128(swizzled<C::kLine>(sK, key + 8, HD / 4 * t + 16 * x));
                    const uint32_t ww[4] = {w.x, w.y, w.z, w.w}, zz[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        uint32_t w0, w1, z0, z1;
                        e4m3_to_f16(ww[y], w0, w1);
                        e4m3_to_f16(zz[y], z0, z1);
                        product(4 * x + y, w0, z0, w1, z1);
                    }
                }
            } else {
#pragma unroll
                for (int x = 0; x < 2 * C::kBoxes; ++x) {
                    const uint32_t box = sK + (x >> 1) * C::kKeys * C::kLine;
                    const uint4 w = lds128(swizzled<C::kLine>(box, key, 32 * t + 16 * (x & 1))), z = lds128(swizzled<C::kLine>(box, key + 8, 32 * t + 16 * (x & 1)));
                    product(2 * x, w.x, z.x, w.y, z.y);
                    product(2 * x + 1, w.z, z.z, w.w, z.w);
                }
            }
        }
        // Exponents of the step's keys (8 bits): lane i has those of key i, as what a score is multiplied with and as it is.
        float k_scale = a.scale_log2, v_exp = 0.f;
        bool grows = false;
        if constexpr (kE4M3) {
            k_scale = key_factor(lds_s8(sE + lane), key_scale);
            const int e = lds_s8(sE + C::kKeys + lane);
            v_exp = e == kExpNotFinite ? __uint_as_float(0x7fffffffu) : static_cast<float>(e);
        }
        float v_exps[kTiles][2];
        // scores in units of log2: keys 16 u + g + 8 (x >> 1), rows 8 r + 2 t + (x & 1)
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            float scale[2] = {k_scale, k_scale};
            if constexpr (kE4M3) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    scale[x] = __shfl_sync(0xffffffffu, k_scale, 16 * u + 8 * x + g);
                    v_exps[u][x] = __shfl_sync(0xffffffffu, v_exp, 16 * u + 8 * x + g);
                }
            }
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    sc[u][r][x] *= scale[x >> 1];
                    if constexpr (kE4M3) sc[u][r][x] *= row_scale[r][x & 1];
                    if (masked && !attends(pos[r][x & 1], key0 + 16 * u + 8 * (x >> 1) + g, window, a.sinks)) sc[u][r][x] = -INFINITY;
                    const float over = sc[u][r][x] - m[r][x & 1];
                    grows |= over > kLazy;
                    if constexpr (kE4M3) grows |= over + v_exps[u][x >> 1] > delta[r][x & 1] + kLazy;
                }
        }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r) {
                float down[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float top = m[r][h];
#pragma unroll
                    for (int u = 0; u < kTiles; ++u) top = fmax3(top, sc[u][r][h], sc[u][r][h + 2]);
#pragma unroll
                    for (int off = 4; off < 32; off *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                    const float up = top - m[r][h];
                    down[h] = fast_exp2(-up);
                    m[r][h] = top;
                    l[r][h] *= down[h];
                    if constexpr (kE4M3) {
                        const float before = delta[r][h] - up;  // (of a row without a key so far -3e38, and all there is of it is zeros)
                        top = before;
#pragma unroll
                        for (int u = 0; u < kTiles; ++u) top = fmax3(top, (sc[u][r][h] - m[r][h]) + v_exps[u][0], (sc[u][r][h + 2] - m[r][h]) + v_exps[u][1]);
#pragma unroll
                        for (int off = 4; off < 32; off *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                        down[h] = fast_exp2(before - top);
                        delta[r][h] = top;
                    }
                }
#pragma unroll
                for (int x = 0; x < HD / 16; ++x) o[r][x][0] *= down[0], o[r][x][1] *= down[1], o[r][x][2] *= down[0], o[r][x][3] *= down[1];
            }
        }
        uint32_t w[kTiles][kRowTiles][2];  // weights of rows 8 r + g, keys 16 u + 2 t.. and 16 u + 8 + 2 t.. as pairs
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
#pragma unroll
            for (int r = 0; r < kRowTiles; ++r) {
                float e[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float over = sc[u][r][x] - m[r][x & 1];
                    e[x] = fast_exp2(over);
                    l[r][x & 1] += e[x];
                    // (a key that is not attended can have any exponent, also that of a row that is not finite)
                    if constexpr (kE4M3) e[x] = masked && sc[u][r][x] == -INFINITY ? 0.f : fast_exp2(over + v_exps[u][x >> 1] - (delta[r][x & 1] - 7.f));
                }
                w[u][r][0] = transpose_8x8(kE4M3 ? pack_f16(e[0], e[1]) : pack_bf16(e[0], e[1]));
                w[u][r][1] = transpose_8x8(kE4M3 ? pack_f16(e[2], e[3]) : pack_bf16(e[2], e[3]));
            }
        }
        // O^T += V^T P^T, 16 keys at a time.  A thread loads 8 (or 16) columns from column 8 g (16 g) on of the keys 2 t, 2 t + 1, 2 t + 8 and
        // 2 t + 9; two neighbouring columns are rows g and g + 8 of a product.
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            constexpr int kLoad = kE4M3 && HD == 64 ? 8 : 16;  // bytes
#pragma unroll
            for (int bx = 0; bx < C::kBoxes; ++bx) {
                uint32_t v[4][4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int key = 16 * u + 2 * t + (x & 1) + 8 * (x >> 1);
                    const uint32_t from = swizzled<C::kLine>(sV + bx * C::kKeys * C::kLine, key, kLoad * g);
                    if constexpr (kLoad == 16) {
                        const uint4 y = lds128(from);
                        v[x][0] = y.x, v[x][1] = y.y, v[x][2] = y.z, v[x][3] = y.w;
                    } else {
                        const uint2 y = lds64(from);
                        v[x][0] = y.x, v[x][1] = y.y, v[x][2] = v[x][3] = 0u;
                    }
                    // what no row attends may be anything (past the end of the sequence whatever the page held before, in front of a
                    // window another sequence's, or what the ring held), and a weight of zero does not make a NaN go away
                    if (masked && !any_attends(first_pos, last_pos, key0 + key, window, a.sinks)) v[x][0] = v[x][1] = v[x][2] = v[x][3] = 0u;
                }
                auto product = [&](int x, uint32_t p0, uint32_t p1, uint32_t p2, uint32_t p3) {  // a pair of columns of the four keys
                    const uint32_t a0 = __byte_perm(p0, p1, 0x5410), a1 = __byte_perm(p0, p1, 0x7632), a2 = __byte_perm(p2, p3, 0x5410), a3 = __byte_perm(p2, p3, 0x7632);
#pragma unroll
                    for (int r = 0; r < kRowTiles; ++r) mma_16x8x16<kE4M3>(o[r][x], a0, a1, a2, a3, w[u][r][0], w[u][r][1]);
                };
#pragma unroll
                for (int y = 0; y < kLoad / 4; ++y) {
                    if constexpr (kE4M3) {
                        uint32_t lo[4], hi[4];
#pragma unroll
                        for (int x = 0; x < 4; ++x) e4m3_to_f16(v[x][y], lo[x], hi[x]);
                        product(2 * y, lo[0], lo[1], lo[2], lo[3]);
                        product(2 * y + 1, hi[0], hi[1], hi[2], hi[3]);
                    } else {
                        product(4 * bx + y, v[0][y], v[1][y], v[2][y], v[3][y]);
                    }
                }
            }
        }
        __syncwarp();
        if (c + stages < steps) request(c + stages, st);
        if (++st == stages) st = 0, phase ^= 1;
    }
    if (lane == 0) {
        // of a warp that gave up, loads in flight land before the memory is used for something else
        for (int x = c; !ok && x < steps && x < c + stages; ++x) {
            mbar_wait_drain(&full[st], phase);
            if (++st == stages) st = 0, phase ^= 1;
        }
    }
    __syncwarp();

    // ---- this warp's result into its ring: O of the rows, then m and l
    float* mine = reinterpret_cast<float*>(ring);
    constexpr int kM = kRows * HD, kL = kM + kRows, kJoined = kL + kRows;
    constexpr int kCols = kE4M3 ? HD / 8 : 8;  // columns of a thread that lie together
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = 8 * r + 2 * t + h;
            // unit^2 is O's, beside the sum of weights (which fp32's numbers reach, where exp2 does not)
            const float unit = kE4M3 ? fast_exp2(0.5f * (delta[r][h] - 7.f)) : 1.f;
#pragma unroll
            for (int off = 4; off < 32; off *= 2) l[r][h] += __shfl_xor_sync(0xffffffffu, l[r][h], off);
            if (g == 0) mine[kM + row] = m[r][h], mine[kL + row] = l[r][h];
#pragma unroll
            for (int x = 0; x < HD / 16; ++x) {
                float2* to = reinterpret_cast<float2*>(mine + row * HD + 2 * x / kCols * (8 * kCols) + kCols * g + 2 * x % kCols);
                *to = make_float2(o[r][x][h] * unit * unit, o[r][x][h + 2] * unit * unit);
            }
        }
    __syncthreads();

    auto finish = [&](int e, float value, float top, float sum) {
        const int row = e / HD, col = e % HD;
        int hh;
        const int i = p.by_rep(r0 + row, &hh), h = hk * a.rep + hh;
        const long long to = static_cast<long long>(s.row0 + i);
        if (abort_flag != 0) return;
        a.o[(to * a.H + h) * HD + col] = __float2bfloat16(value / sum);
        if (col == 0) a.lse[static_cast<long long>(h) * a.batch.T + to] = (top + log2f(sum)) * 0.6931471805599453f;
    };
    // ---- the warps' results joined, into the first ring
    const int ring_floats = ring_bytes / 4;
    float* first = reinterpret_cast<float*>(smem);
    for (int e = threadIdx.x; e < rows * HD; e += threads) {
        const int row = e / HD;
        float top = kLeast, sum = 0.f, value = 0.f;
#pragma unroll
        for (int w = 0; w < C::kMostWarps; ++w)
            if (w < warps) top = fmaxf(top, first[w * ring_floats + kM + row]);
#pragma unroll
        for (int w = 0; w < C::kMostWarps; ++w) {
            if (w >= warps) break;
            const float f = fast_exp2(first[w * ring_floats + kM + row] - top);
            sum += f * first[w * ring_floats + kL + row];
            value += f * first[w * ring_floats + e];
        }
        if (p.split == 1) {
            finish(e, value, top, sum);
        } else {
            first[e] = value;  // only this thread reads and writes this place
            // (m and l of the first warp are still read for other columns: the joined ones go behind them)
            if (e % HD == 0) first[kJoined + row] = top, first[kJoined + kRows + row] = sum;
        }
    }
    if (p.split == 1) return;
    cluster_sync();
    // ---- the blocks' results joined, a share of the elements in each block
    const uint32_t at = smem_u32(first);
    for (int e = part * threads + static_cast<int>(threadIdx.x); e < rows * HD; e += p.split * threads) {
        const int row = e / HD;
        float tops[kMostSplit], top = kLeast, sum = 0.f, value = 0.f;
#pragma unroll
        for (int x = 0; x < kMostSplit; ++x) {
            tops[x] = x < p.split ? load_remote(at + (kJoined + row) * 4, x) : kLeast;
            top = fmaxf(top, tops[x]);
        }
#pragma unroll
        for (int x = 0; x < kMostSplit; ++x)
            if (x < p.split) {
                const float f = fast_exp2(tops[x] - top);
                sum += f * load_remote(at + (kJoined + kRows + row) * 4, x);
                value += f * load_remote(at + e * 4, x);
            }
        finish(e, value, top, sum);
    }
    cluster_sync();  // nobody leaves while its results are read
}

template <int HD, bool kE4M3, int kRowTiles, bool kWindow>
cudaError_t configure_form() {
    auto kernel = s2a_paged_split_kernel<HD, kE4M3, kRowTiles, kWindow>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               SplitCfg<HD, kE4M3>::smem_bytes(1, SplitCfg<HD, kE4M3>::kMostWarps));
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}
template <int HD, bool kE4M3, int kRowTiles>
cudaError_t configure_one() {
    const cudaError_t e = configure_form<HD, kE4M3, kRowTiles, false>();
    return e != cudaSuccess ? e : configure_form<HD, kE4M3, kRowTiles, true>();
}

template <int HD, bool kE4M3>
struct SplitLaunch {
    cudaLaunchConfig_t config = {};
    cudaLaunchAttribute attribute[2] = {};
    SplitLaunch(const PagedSplitParams& p, unsigned grid, cudaStream_t stream) {
        config.gridDim = dim3(grid);
        config.blockDim = dim3(32u * static_cast<unsigned>(p.warps));
        config.dynamicSmemBytes = SplitCfg<HD, kE4M3>::smem_bytes(p.blocks, p.warps);
        config.stream = stream;
        attribute[0].id = cudaLaunchAttributeClusterDimension;
        attribute[0].val.clusterDim.x = static_cast<unsigned>(p.split), attribute[0].val.clusterDim.y = attribute[0].val.clusterDim.z = 1;
        attribute[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attribute[1].val.programmaticStreamSerializationAllowed = 1;
        config.attrs = attribute;
        config.numAttrs = 2;
    }
};

template <int HD, bool kE4M3, int kRowTiles>
cudaError_t launch_one(const PagedSplitParams& p, cudaStream_t stream) {
    const unsigned units = static_cast<unsigned>(p.row_blocks) * static_cast<unsigned>(p.a.batch.B) * static_cast<unsigned>(p.a.pool.Hkv);
    const SplitLaunch<HD, kE4M3> launch(p, units * static_cast<unsigned>(p.split), stream);
    return cudaLaunchKernelEx(&launch.config, p.a.window > 0 ? s2a_paged_split_kernel<HD, kE4M3, kRowTiles, true> : s2a_paged_split_kernel<HD, kE4M3, kRowTiles, false>, p);
}

}  // namespace

int split_stages(bool e4m3, int d, int blocks) {
    return d == 64 ? (e4m3 ? SplitCfg<64, true>::stages(blocks) : SplitCfg<64, false>::stages(blocks))
                   : (e4m3 ? SplitCfg<128, true>::stages(blocks) : SplitCfg<128, false>::stages(blocks));
}

int split_keys(bool e4m3, int d) {
    return d == 64 ? (e4m3 ? SplitCfg<64, true>::kKeys : SplitCfg<64, false>::kKeys) : (e4m3 ? SplitCfg<128, true>::kKeys : SplitCfg<128, false>::kKeys);
}

cudaError_t configure_paged_split(int (*slots)[kMostSplit + 1]) {
    for (const cudaError_t e : {configure_one<64, false, 1>(), configure_one<64, false, 2>(), configure_one<64, true, 1>(), configure_one<64, true, 2>(),
                                configure_one<128, false, 1>(), configure_one<128, false, 2>(), configure_one<128, true, 1>(), configure_one<128, true, 2>()})
        if (e != cudaSuccess) return e;
    // (what limits the blocks on an SM is shared memory, of which all forms take the same)
    for (int blocks = 1; blocks <= 3; ++blocks)
        for (int split = 1; split <= kMostSplit; ++split) {
            PagedSplitParams p = {};
            p.warps = 4, p.split = split, p.blocks = blocks;
            SplitLaunch<128, true> launch(p, static_cast<unsigned>(split), nullptr);
            int clusters = 0;
            if (cudaOccupancyMaxActiveClusters(&clusters, s2a_paged_split_kernel<128, true, 1, false>, &launch.config) != cudaSuccess) {
                cudaGetLastError();  // clusters of this size are not to be had
                clusters = 0;
            }
            slots[blocks][split] = clusters * split;
        }
    return cudaSuccess;
}

cudaError_t launch_paged_split(const PagedSplitParams& p, bool e4m3, int d, cudaStream_t stream) {
    auto launch = p.unit_rows == 8 ? (d == 64 ? (e4m3 ? launch_one<64, true, 1> : launch_one<64, false, 1>) : (e4m3 ? launch_one<128, true, 1> : launch_one<128, false, 1>))
                                   : (d == 64 ? (e4m3 ? launch_one<64, true, 2> : launch_one<64, false, 2>) : (e4m3 ? launch_one<128, true, 2> : launch_one<128, false, 2>));
    return launch(p, stream);
}

}  // namespace s2a
