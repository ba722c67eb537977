// Attention of few rows over the paged cache: sequences with one new token, or a handful.
//
// A row is a new token and a query head; the rows of a sequence and KV head (new tokens times query heads of a KV head) read the
// same keys.  With at most 64 of them the work is reading the cache: 4 d multiply-adds for each row and key against 4 d
// bytes of bf16.  So the keys are split: a unit, 16 rows of one sequence and KV head, is worked on by a cluster of blocks, each
// with a share of the keys, its four warps taking 16 or 32 keys in turn.  A warp has a ring of its own that TMA fills, a
// running maximum and sum for its rows and the weighted sum of v in registers.  What the warps and then the blocks have is
// joined through shared memory and the cluster's: no second launch, no workspace, no atomics.
//
// Products of a warp: S = Q K^T and O += P V, 16 rows at a time (mma.sync: the tensor work is a tenth of the time).  Which columns
// of a head go into which product does not matter as long as Q and K agree, so a thread takes what lies together in
// shared memory; the two keys of a pair of P are next to each other in the accumulator of S, as P's operand needs them.
//
// Cached 8-bit floats become bf16 in registers by moving bits (e4m3_spread).  K's power of two multiplies the scores, V's the
// weights before they are rounded: both exactly.
#include "paged_device.cuh"

namespace s2a {

namespace {

template <int HD, bool kE4M3>
struct SplitCfg {
    static constexpr int kWarps = 4, kThreads = 32 * kWarps;
    static constexpr int kRowBytes = HD * (kE4M3 ? 1 : 2);        // a key's row
    static constexpr int kKeys = kRowBytes == 256 ? 16 : 32;      // keys of a warp's step
    static constexpr int kLine = kRowBytes < 128 ? kRowBytes : 128;  // bytes of a row in one box
    static constexpr int kBoxes = kRowBytes / kLine;
    static constexpr int kTile = kKeys * kRowBytes;               // K or V of a step
    static constexpr int kStageBytes = 2 * kTile;
    static constexpr int kStages = 24576 / kStageBytes;           // 24 KB in flight for each warp, two blocks on an SM
    static constexpr int kExpBytes = kE4M3 ? 2 * kKeys : 0;       // exponents of K and V
    static constexpr int kSmemBytes = kWarps * kStages * (kStageBytes + kExpBytes) + kWarps * kStages * 8 + 16;  // and the abort flag
    static constexpr int kPartFloats = 16 * HD + 32;              // a warp's result: O, m, l
    static_assert(kPartFloats * 4 <= kStages * kStageBytes, "the ring holds a result");
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
__device__ __forceinline__ float exponent_factor(int e) {
    return e == kExpNotFinite ? __uint_as_float(0x7fffffffu) : __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

constexpr float kLeast = -3.0e38f;  // stands for "no key yet": finite, so that differences are numbers

template <int HD, bool kE4M3>
__global__ void __launch_bounds__(SplitCfg<HD, kE4M3>::kThreads, 2) s2a_paged_split_kernel(const __grid_constant__ PagedSplitParams p) {
    using C = SplitCfg<HD, kE4M3>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const PagedFwdParams& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    uint8_t* ring = smem + warp * (C::kStages * C::kStageBytes);
    uint8_t* exps = smem + C::kWarps * C::kStages * C::kStageBytes + warp * (C::kStages * C::kExpBytes);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + C::kWarps * C::kStages * (C::kStageBytes + C::kExpBytes)) + warp * C::kStages;
    volatile int& abort_flag = *reinterpret_cast<volatile int*>(smem + C::kSmemBytes - 16);

    if (lane == 0) {
        for (int s = 0; s < C::kStages; ++s) mbar_init(&full[s], 1);
        fence_barrier_init();
        tma_prefetch_desc(&p.tm_k);
        tma_prefetch_desc(&p.tm_v);
    }
    release_successor();
    wait_for_predecessor();
    // an earlier report: nothing is read or written, but every block of a cluster goes on to the end with the others
    if (threadIdx.x == 0) abort_flag = *reinterpret_cast<volatile int*>(a.status);
    __syncthreads();
    if (blockIdx.x == 0) check_batch(a.batch, a.pool.page_log2, a.most_new, a.status, a.host_status);
    const WaitCtx ctx{&abort_flag, a.status, a.host_status};

    int part, row_block, hk;
    const int unit = p.by_split(static_cast<int>(blockIdx.x), &part);
    const int b = p.by_heads(p.by_row_blocks(unit, &row_block), &hk);
    Sequence s;
    if (sequence_of(a.batch, a.pool.page_log2, a.most_new, b, &s) != 0) return;  // (the same for all blocks of the cluster)
    const int all_rows = s.n * a.rep, r0 = row_block * 16;
    if (r0 >= all_rows || all_rows > a.few_rows) return;
    const int rows = all_rows - r0 < 16 ? all_rows - r0 : 16;
    const int first_pos = s.length - s.n + p.by_rep(r0), last_pos = s.length - s.n + p.by_rep(r0 + rows - 1);
    const KeyBlocks blocks = key_blocks(first_pos, last_pos, a.window, a.sinks, C::kKeys);
    const int share = (blocks.count + p.split - 1) / p.split;
    const int i0 = part * share + warp, i1 = (part + 1) * share < blocks.count ? (part + 1) * share : blocks.count;
    int steps = i0 < i1 ? (i1 - i0 + C::kWarps - 1) / C::kWarps : 0;
    if (__any_sync(0xffffffffu, *ctx.abort_flag != 0)) steps = 0;

    // ---- loads of this warp: pages of its next 32 steps are in its lanes; lane 0 (and 1, where a step spans two pages) requests
    const int piece_log2 = a.pool.page_log2 < (C::kKeys == 16 ? 4 : 5) ? a.pool.page_log2 : (C::kKeys == 16 ? 4 : 5);
    const int pieces = C::kKeys >> piece_log2;
    int page[2] = {-1, -1};
    auto look_up = [&](int from) {
        const int x = from + lane;
        page[0] = page[1] = -1;
        if (x < steps) {
            const int key = blocks.at(i0 + x * C::kWarps) * C::kKeys;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = key + (i << piece_log2);
                if (i < pieces && k < s.length) {
                    page[i] = page_of(a.batch, a.pool.pages, b, k >> a.pool.page_log2);
                    if (page[i] < 0) report_bad_index(a.status, a.host_status, kBadPage);
                }
            }
        }
    };
    auto request = [&](int c) {
        if ((c & 31) == 0) look_up(c);
        const int st = c % C::kStages;
        const int key = blocks.at(i0 + c * C::kWarps) * C::kKeys;
        const int p0 = __shfl_sync(0xffffffffu, page[0], c & 31), p1 = __shfl_sync(0xffffffffu, page[1], c & 31);
        const int mine = lane == 0 ? p0 : lane == 1 ? p1 : -1;
        const uint32_t bytes = static_cast<uint32_t>((2 * C::kRowBytes + (kE4M3 ? 2 : 0)) << piece_log2);
        if (lane == 0) mbar_expect_tx(&full[st], bytes * ((p0 >= 0) + (p1 >= 0)));
        __syncwarp();
        if (mine >= 0) {
            const int slot = (key + (lane << piece_log2)) & ((1 << a.pool.page_log2) - 1);
            const int row = ((mine * a.pool.Hkv + hk) << a.pool.page_log2) + slot;
            const uint32_t bar = smem_u32(&full[st]), dst = smem_u32(ring + st * C::kStageBytes) + ((lane << piece_log2) * C::kLine);
#pragma unroll
            for (int x = 0; x < C::kBoxes; ++x) {
                tma_load_2d(dst + x * C::kKeys * C::kLine, &p.tm_k, bar, x * (C::kLine / (kE4M3 ? 1 : 2)), row);
                tma_load_2d(dst + C::kTile + x * C::kKeys * C::kLine, &p.tm_v, bar, x * (C::kLine / (kE4M3 ? 1 : 2)), row);
            }
            if constexpr (kE4M3) {
                uint8_t* e = exps + st * C::kExpBytes + (lane << piece_log2);
                bulk_load_1d(e, a.pool.k_exp + row, 1u << piece_log2, &full[st]);
                bulk_load_1d(e + C::kKeys, a.pool.v_exp + row, 1u << piece_log2, &full[st]);
            }
        }
        __syncwarp();
    };
    for (int c = 0; c < C::kStages && c < steps; ++c) request(c);

    // ---- the rows of Q that this thread's products take: rows g and g + 8; of every line of a key's row the 32 bytes from 32 t on
    // (16 from 16 t on where a line has 64), as pairs in the order in which K's come out of their words
    constexpr int kSteps = HD / 16;          // products of a score tile
    uint32_t q[2][2 * kSteps];
    int pos[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int r = r0 + (g + 8 * half < rows ? g + 8 * half : rows - 1);  // rows past the end follow the last one
        int hh;
        const int i = p.by_rep(r, &hh);
        pos[half] = s.length - s.n + i;
        const __nv_bfloat16* src = a.q + (static_cast<long long>(s.row0 + i) * a.H + hk * a.rep + hh) * HD;
        if constexpr (kE4M3) {
            constexpr int kPer = HD / 4;  // values of a thread
#pragma unroll
            for (int c = 0; c < kPer / 8; ++c) {
                const uint4 x = *reinterpret_cast<const uint4*>(src + kPer * t + 8 * c);
                q[half][4 * c] = __byte_perm(x.x, x.y, 0x5410), q[half][4 * c + 1] = __byte_perm(x.x, x.y, 0x7632);
                q[half][4 * c + 2] = __byte_perm(x.z, x.w, 0x5410), q[half][4 * c + 3] = __byte_perm(x.z, x.w, 0x7632);
            }
        } else {
#pragma unroll
            for (int x = 0; x < C::kBoxes; ++x)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint4 w = *reinterpret_cast<const uint4*>(src + 64 * x + 16 * t + 8 * c);
                    uint32_t* to = &q[half][8 * x + 4 * c];
                    to[0] = w.x, to[1] = w.y, to[2] = w.z, to[3] = w.w;
                }
        }
    }

    float o[HD / 8][4];
#pragma unroll
    for (int x = 0; x < HD / 8; ++x) o[x][0] = o[x][1] = o[x][2] = o[x][3] = 0.f;
    float m[2] = {kLeast, kLeast}, l[2] = {0.f, 0.f};
    bool ok = true;
    int c = 0;
    for (; c < steps; ++c) {
        const int st = c % C::kStages;
        if (!mbar_wait_uniform(&full[st], (c / C::kStages) & 1, ctx, kWaitPagedSplit + 1)) { ok = false; break; }
        const uint32_t sK = smem_u32(ring + st * C::kStageBytes), sV = sK + C::kTile, sE = smem_u32(exps + st * C::kExpBytes);
        const int key0 = blocks.at(i0 + c * C::kWarps) * C::kKeys;
        const bool masked = !all_attend(first_pos, last_pos, key0, C::kKeys, a.window, a.sinks);
        constexpr int kTiles = C::kKeys / 8;
        float sc[kTiles][4];
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            sc[u][0] = sc[u][1] = sc[u][2] = sc[u][3] = 0.f;
            const int key = 8 * u + g;
            if constexpr (kE4M3) {
#pragma unroll
                for (int x = 0; x < HD / 64; ++x) {
                    const uint4 w4 = lds128(swizzled<C::kLine>(sK, key, HD / 4 * t + 16 * x));
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        uint32_t lo, hi;
                        e4m3_spread(w[y], lo, hi);
                        const int k = 4 * x + y;
                        mma_16x8x16(sc[u], q[0][2 * k], q[1][2 * k], q[0][2 * k + 1], q[1][2 * k + 1], bf16x2_mul(lo, kTwoTo120), bf16x2_mul(hi, kTwoTo120));
                    }
                }
            } else {
#pragma unroll
                for (int x = 0; x < 2 * C::kBoxes; ++x) {
                    const uint4 w = lds128(swizzled<C::kLine>(sK + (x >> 1) * C::kKeys * C::kLine, key, 32 * t + 16 * (x & 1)));
                    mma_16x8x16(sc[u], q[0][4 * x], q[1][4 * x], q[0][4 * x + 1], q[1][4 * x + 1], w.x, w.y);
                    mma_16x8x16(sc[u], q[0][4 * x + 2], q[1][4 * x + 2], q[0][4 * x + 3], q[1][4 * x + 3], w.z, w.w);
                }
            }
        }
        // scores in units of log2, keys 8 u + 2 t + (x & 1), rows g + 8 (x >> 1)
        float v_factor[kTiles][2];
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            float factor[2] = {a.scale_log2, a.scale_log2};
            if constexpr (kE4M3) {
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    factor[x] *= exponent_factor(lds_s8(sE + 8 * u + 2 * t + x));
                    v_factor[u][x] = exponent_factor(lds_s8(sE + C::kKeys + 8 * u + 2 * t + x));
                }
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                sc[u][x] *= factor[x & 1];
                if (masked && !attends(pos[x >> 1], key0 + 8 * u + 2 * t + (x & 1), a.window, a.sinks)) sc[u][x] = -INFINITY;
                top[x >> 1] = fmaxf(top[x >> 1], sc[u][x]);
            }
        }
        uint32_t changed = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 1));
            top[h] = fmaxf(top[h], __shfl_xor_sync(0xffffffffu, top[h], 2));
            changed |= top[h] != m[h];
        }
        if (__any_sync(0xffffffffu, changed)) {
            const float down[2] = {fast_exp2(m[0] - top[0]), fast_exp2(m[1] - top[1])};
            l[0] *= down[0], l[1] *= down[1];
#pragma unroll
            for (int x = 0; x < HD / 8; ++x) o[x][0] *= down[0], o[x][1] *= down[0], o[x][2] *= down[1], o[x][3] *= down[1];
            m[0] = top[0], m[1] = top[1];
        }
        uint32_t w[kTiles][2];  // weights of rows g and g + 8 as pairs of keys
#pragma unroll
        for (int u = 0; u < kTiles; ++u) {
            float e[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                e[x] = fast_exp2(sc[u][x] - m[x >> 1]);
                l[x >> 1] += e[x];
                if constexpr (kE4M3) e[x] = masked && sc[u][x] == -INFINITY ? 0.f : e[x] * v_factor[u][x & 1];
            }
            w[u][0] = pack_bf16(e[0], e[1]), w[u][1] = pack_bf16(e[2], e[3]);
        }
        // O += P V, 16 keys at a time: a thread loads 8 (or 16) columns from column 8 g (16 g) on of the keys 2 t, 2 t + 1 of either tile
#pragma unroll
        for (int u = 0; u < kTiles; u += 2) {
            const int keys[4] = {8 * u + 2 * t, 8 * u + 2 * t + 1, 8 * u + 8 + 2 * t, 8 * u + 9 + 2 * t};
            if constexpr (kE4M3) {
                constexpr int kWords = HD / 32;
                uint32_t v[4][kWords];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if constexpr (HD == 128) {
                        const uint4 r = lds128(swizzled<C::kLine>(sV, keys[x], 16 * g));
                        v[x][0] = r.x, v[x][1] = r.y, v[x][2] = r.z, v[x][3] = r.w;
                    } else {
                        const uint2 r = lds64(swizzled<C::kLine>(sV, keys[x], 8 * g));
                        v[x][0] = r.x, v[x][1] = r.y;
                    }
                }
#pragma unroll
                for (int y = 0; y < kWords; ++y) {
                    uint32_t lo[4], hi[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        e4m3_spread(v[x][y], lo[x], hi[x]);
                        lo[x] = bf16x2_mul(lo[x], kTwoTo120), hi[x] = bf16x2_mul(hi[x], kTwoTo120);
                    }
                    mma_16x8x16(o[4 * y], w[u][0], w[u][1], w[u + 1][0], w[u + 1][1], __byte_perm(lo[0], lo[1], 0x5410), __byte_perm(lo[2], lo[3], 0x5410));
                    mma_16x8x16(o[4 * y + 1], w[u][0], w[u][1], w[u + 1][0], w[u + 1][1], __byte_perm(hi[0], hi[1], 0x5410), __byte_perm(hi[2], hi[3], 0x5410));
                    mma_16x8x16(o[4 * y + 2], w[u][0], w[u][1], w[u + 1][0], w[u + 1][1], __byte_perm(lo[0], lo[1], 0x7632), __byte_perm(lo[2], lo[3], 0x7632));
                    mma_16x8x16(o[4 * y + 3], w[u][0], w[u][1], w[u + 1][0], w[u + 1][1], __byte_perm(hi[0], hi[1], 0x7632), __byte_perm(hi[2], hi[3], 0x7632));
                }
            } else {
#pragma unroll
                for (int bx = 0; bx < C::kBoxes; ++bx) {
                    uint32_t v[4][4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint4 r = lds128(swizzled<C::kLine>(sV + bx * C::kKeys * C::kLine, keys[x], 16 * g));
                        v[x][0] = r.x, v[x][1] = r.y, v[x][2] = r.z, v[x][3] = r.w;
                        // what no row attends may be anything (positions past the end of the sequence hold whatever the page held
                        // before), and a weight of zero does not make a NaN go away
                        if (masked && !any_attends(first_pos, last_pos, key0 + keys[x], a.window, a.sinks))
                            v[x][0] = v[x][1] = v[x][2] = v[x][3] = 0u;
                    }
#pragma unroll
                    for (int y = 0; y < 4; ++y) {
                        mma_16x8x16(o[8 * bx + 2 * y], w[u][0], w[u][1], w[u + 1][0], w[u + 1][1], __byte_perm(v[0][y], v[1][y], 0x5410),
                                    __byte_perm(v[2][y], v[3][y], 0x5410));
                        mma_16x8x16(o[8 * bx + 2 * y + 1], w[u][0], w[u][1], w[u + 1][0], w[u + 1][1], __byte_perm(v[0][y], v[1][y], 0x7632),
                                    __byte_perm(v[2][y], v[3][y], 0x7632));
                    }
                }
            }
        }
        __syncwarp();
        if (c + C::kStages < steps) request(c + C::kStages);
    }
    if (!ok && lane == 0)  // loads in flight land before the memory is used for something else
        for (int x = c; x < steps && x < c + C::kStages; ++x) mbar_wait_drain(&full[x % C::kStages], (x / C::kStages) & 1);
    __syncwarp();

    // ---- this warp's result into its ring: [16][HD] of O, then m and l of the 16 rows
    float* mine = reinterpret_cast<float*>(ring);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
        l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
        if (t == 0) mine[16 * HD + g + 8 * h] = m[h], mine[16 * HD + 16 + g + 8 * h] = l[h];
    }
    // product x of a group of kCols has the columns kCols * (2 t) + x and kCols * (2 t + 1) + x of the group's 8 * kCols
    constexpr int kCols = kE4M3 ? HD / 8 : 8;
#pragma unroll
    for (int x = 0; x < HD / 8; ++x) {
        const int col = x / kCols * (8 * kCols) + kCols * 2 * t + x % kCols;
        mine[g * HD + col] = o[x][0], mine[g * HD + col + kCols] = o[x][1];
        mine[(g + 8) * HD + col] = o[x][2], mine[(g + 8) * HD + col + kCols] = o[x][3];
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
    // ---- the four warps' results joined, into the first ring
    constexpr int kRing = C::kStages * C::kStageBytes / 4;  // floats of a ring
    float* first = reinterpret_cast<float*>(smem);
    for (int e = threadIdx.x; e < rows * HD; e += C::kThreads) {
        const int row = e / HD;
        float top = kLeast, sum = 0.f, value = 0.f;
#pragma unroll
        for (int w = 0; w < C::kWarps; ++w) top = fmaxf(top, first[w * kRing + 16 * HD + row]);
#pragma unroll
        for (int w = 0; w < C::kWarps; ++w) {
            const float f = fast_exp2(first[w * kRing + 16 * HD + row] - top);
            sum += f * first[w * kRing + 16 * HD + 16 + row];
            value += f * first[w * kRing + e];
        }
        if (p.split == 1) {
            finish(e, value, top, sum);
        } else {
            first[e] = value;  // only this thread reads and writes this place
            // (m and l of the first warp are still read for other columns: the joined ones go behind them)
            if (e % HD == 0) first[16 * HD + 32 + row] = top, first[16 * HD + 48 + row] = sum;
        }
    }
    if (p.split == 1) return;
    cluster_sync();
    // ---- the blocks' results joined, a share of the elements in each block
    const uint32_t at = smem_u32(first);
    for (int e = part * C::kThreads + static_cast<int>(threadIdx.x); e < rows * HD; e += p.split * C::kThreads) {
        const int row = e / HD;
        float tops[16], top = kLeast, sum = 0.f, value = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
            tops[x] = x < p.split ? load_remote(at + (16 * HD + 32 + row) * 4, x) : kLeast;
            top = fmaxf(top, tops[x]);
        }
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (x < p.split) {
                const float f = fast_exp2(tops[x] - top);
                sum += f * load_remote(at + (16 * HD + 48 + row) * 4, x);
                value += f * load_remote(at + e * 4, x);
            }
        finish(e, value, top, sum);
    }
    cluster_sync();  // nobody leaves while its results are read
}

template <int HD, bool kE4M3>
cudaError_t configure_one() {
    auto kernel = s2a_paged_split_kernel<HD, kE4M3>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SplitCfg<HD, kE4M3>::kSmemBytes);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
}

template <int HD, bool kE4M3>
cudaError_t launch_one(const PagedSplitParams& p, cudaStream_t stream) {
    using C = SplitCfg<HD, kE4M3>;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(static_cast<unsigned>(p.split) * static_cast<unsigned>(p.row_blocks) * static_cast<unsigned>(p.a.batch.B) * static_cast<unsigned>(p.a.pool.Hkv));
    config.blockDim = dim3(C::kThreads);
    config.dynamicSmemBytes = C::kSmemBytes;
    config.stream = stream;
    cudaLaunchAttribute attribute[2] = {};
    attribute[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute[0].val.programmaticStreamSerializationAllowed = 1;
    attribute[1].id = cudaLaunchAttributeClusterDimension;
    attribute[1].val.clusterDim.x = static_cast<unsigned>(p.split), attribute[1].val.clusterDim.y = attribute[1].val.clusterDim.z = 1;
    config.attrs = attribute;
    config.numAttrs = 2;
    return cudaLaunchKernelEx(&config, s2a_paged_split_kernel<HD, kE4M3>, p);
}

}  // namespace

int split_keys(bool e4m3, int d) {
    return d == 64 ? (e4m3 ? SplitCfg<64, true>::kKeys : SplitCfg<64, false>::kKeys) : (e4m3 ? SplitCfg<128, true>::kKeys : SplitCfg<128, false>::kKeys);
}

cudaError_t configure_paged_split() {
    cudaError_t e = configure_one<64, false>();
    if (e == cudaSuccess) e = configure_one<64, true>();
    if (e == cudaSuccess) e = configure_one<128, false>();
    if (e == cudaSuccess) e = configure_one<128, true>();
    return e;
}

cudaError_t launch_paged_split(const PagedSplitParams& p, bool e4m3, int d, cudaStream_t stream) {
    if (d == 64) return e4m3 ? launch_one<64, true>(p, stream) : launch_one<64, false>(p, stream);
    return e4m3 ? launch_one<128, true>(p, stream) : launch_one<128, false>(p, stream);
}

}  // namespace s2a
