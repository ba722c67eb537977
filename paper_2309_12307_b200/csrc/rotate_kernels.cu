// Norms of queries and keys for each head, and the rotation of positions in the same pass; forward, backward, and into the paged cache.
//
// A row is the d values of one head of a token.  With a norm y = w * x * s, s = 1 / sqrt(mean x^2 + eps), else y = x; then pair i of the
// first r values, (u, v) -> (u cos a - v sin a, u sin a + v cos a), a = position * frequency i.  Backwards the gradients of the
// pairs turn by -a, g; then the weight gets sum g * x * s, and x, with n = x * s, s (w g - n mean(w g * n)).  All of it in fp32, rounded to
// bf16 once.
//
// Angles: a frequency is a whole number of 2^-64 turns, so its product with a position, modulo 2^64, is the angle's fraction of a turn
// at any position, of which 32 bits count; 24 of them go to sincospif, the others into the first two terms of the sums of angles.  A row is d / 16 lanes,
// a lane has both values of eight pairs (two pieces of 16 bytes, d / 8 or r / 2 values apart), so that only the sums of a norm cross lanes.  A block's
// tokens have their sines and cosines in shared memory, each made once: a lane that made its own for the 8 heads it had of a token spent as long on them,
// and had no registers left for loads in flight (32768 tokens of 32 + 32 heads of 128 329 us, so 160 to 173).
//
// Bound by HBM: each value is read and written once (the backward of a norm reads two).
#include <cuda_fp16.h>

#include <algorithm>

#include "paged_device.cuh"
#include "rotate.h"

namespace s2a {

namespace {

constexpr int kRotateThreads = 256;
constexpr int kRowsOfLane = 4;  // whose loads a lane has in flight

template <int HD>
struct RowLanes {
    static constexpr int kLanes = HD / 16;
    static constexpr int kGroups = kRotateThreads / kLanes;  // rows of a block at a time
    static constexpr int kTable = HD;                        // sines and cosines of a token
};

// Where a lane's two pieces of 8 values are in a row, and whether they are rotated.
struct Pieces {
    int at[2];
    bool turned;
    __device__ __forceinline__ Pieces(int part, int r) {
        turned = part < r / 16;
        at[0] = turned ? 8 * part : 16 * part;
        at[1] = turned ? 8 * part + r / 2 : 16 * part + 8;
    }
};

__device__ __forceinline__ void unpack_row(const uint4 (&w)[2], float (&x)[16]) {
    const uint32_t v[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) x[2 * i] = bf16_low(v[i]), x[2 * i + 1] = bf16_high(v[i]);
}
__device__ __forceinline__ void pack_row(const float (&x)[16], uint4 (&w)[2]) {
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
    w[0] = make_uint4(v[0], v[1], v[2], v[3]), w[1] = make_uint4(v[4], v[5], v[6], v[7]);
}

__device__ __forceinline__ void load_row(const __nv_bfloat16* row, const Pieces& pieces, uint4 (&w)[2]) {
#pragma unroll
    for (int y = 0; y < 2; ++y) w[y] = __ldcg(reinterpret_cast<const uint4*>(row + pieces.at[y]));
}
__device__ __forceinline__ void store_row(__nv_bfloat16* row, const Pieces& pieces, const uint4 (&w)[2]) {
#pragma unroll
    for (int y = 0; y < 2; ++y) *reinterpret_cast<uint4*>(row + pieces.at[y]) = w[y];
}

__device__ __forceinline__ int position_of(const Rotation& ro, int t) {
    int rest;
    ro.by_positions(t, &rest);
    return ro.positions ? S2A_LOAD(ro.positions + rest) : rest;
}

// Cosines and sines of a token's pairs in shared memory: [4][lanes of a row][4], a lane's pairs 2 j and 2 j + 1 as four numbers, so that lanes that read
// theirs meet in no bank.  Pair i < 8 of a lane is values i and 8 + i of its 16, or 2 i and 2 i + 1 where they are interleaved.
template <int HD>
__device__ __forceinline__ void make_angle(float* table, const Rotation& ro, int pair, int position, bool backwards) {
    int part, i;
    if (!ro.interleaved) part = pair / 8, i = pair % 8;
    else part = (pair < ro.r / 4 ? pair : pair - ro.r / 4) / 4, i = pair % 4 + (pair < ro.r / 4 ? 0 : 4);
    const unsigned long long turn = static_cast<unsigned long long>(static_cast<long long>(position)) * static_cast<unsigned long long>(S2A_LOAD(ro.turns + pair));
    const int fraction = static_cast<int>(turn >> 32);
    float s, c;
    sincospif(static_cast<float>(fraction & ~255) * 0x1p-31f, &s, &c);
    const float rest = static_cast<float>(fraction & 255) * (3.14159265358979f * 0x1p-31f);
    float2 x = make_float2(fmaf(-rest, s, c), fmaf(rest, c, s));
    if (backwards) x.y = -x.y;
    *reinterpret_cast<float2*>(table + (i / 2 * RowLanes<HD>::kLanes + part) * 4 + i % 2 * 2) = x;
}
template <int HD>
__device__ __forceinline__ void turn_row(float (&x)[16], const float* table, const Pieces& pieces, int part, bool interleaved) {
    if (!pieces.turned) return;
    auto pair = [](float& u, float& v, float c, float s) {
        const float a = u, b = v;
        u = a * c - b * s, v = a * s + b * c;
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 y = *reinterpret_cast<const float4*>(table + (j * RowLanes<HD>::kLanes + part) * 4);
        if (interleaved) {
            pair(x[4 * j], x[4 * j + 1], y.x, y.y);
            pair(x[4 * j + 2], x[4 * j + 3], y.z, y.w);
        } else {
            pair(x[2 * j], x[8 + 2 * j], y.x, y.y);
            pair(x[2 * j + 1], x[8 + 2 * j + 1], y.z, y.w);
        }
    }
}

// The weights of a norm, in shared memory as a lane's values: [4][lanes of a row][4].
template <int HD>
__device__ __forceinline__ void stage_weights(float* to, const void* weight, bool f32, int r, int c) {
    const int part = c / 16, i = c % 16, at = Pieces(part, r).at[i / 8] + i % 8;
    to[(i / 4 * RowLanes<HD>::kLanes + part) * 4 + i % 4] =
        !weight ? 1.f : f32 ? S2A_LOAD(static_cast<const float*>(weight) + at)
                            : __uint_as_float(static_cast<uint32_t>(S2A_LOAD(static_cast<const unsigned short*>(weight) + at)) << 16);
}
template <int HD>
__device__ __forceinline__ void times_weights(float (&x)[16], const float* weights, int part) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float4 w = *reinterpret_cast<const float4*>(weights + (j * RowLanes<HD>::kLanes + part) * 4);
        x[4 * j] *= w.x, x[4 * j + 1] *= w.y, x[4 * j + 2] *= w.z, x[4 * j + 3] *= w.w;
    }
}

// The sum over the lanes of a row.  `mask`: the lanes that are here.
template <int HD>
__device__ __forceinline__ float sum_of_row(float x, uint32_t mask = 0xffffffffu) {
#pragma unroll
    for (int off = RowLanes<HD>::kLanes / 2; off > 0; off >>= 1) x += __shfl_xor_sync(mask, x, off);
    return x;
}

// x times s = 1 / sqrt(mean x^2 + eps); every lane of a row gets the same.  Squares that fp32 would not hold (values above 2^45, or, where eps does not
// matter either, below 2^-50) are taken of x times a power of two.  Returns s, of small rows without that power (*rest, else 1): of subnormal numbers the two
// together are infinite.
template <int HD>
__device__ __forceinline__ float normalise_row(float (&x)[16], float eps, float* rest) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
    sum = sum_of_row<HD>(sum);
    const bool large = sum > 0x1p100f, small = sum < 0x1p-100f && eps < 0x1p-100f;
    float by = 1.f;
    if (large || small) {
        constexpr int kLanes = RowLanes<HD>::kLanes;
        const uint32_t mask = ((1u << kLanes) - 1) << ((threadIdx.x & 31) & ~(kLanes - 1));
        by = large ? 0x1p-80f : 0x1p80f;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= by, sum += x[i] * x[i];
        sum = sum_of_row<HD>(sum, mask);
        eps = (eps * by) * by;
    }
    const float s = rsqrtf(sum * (1.f / HD) + eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] *= s;
    *rest = small ? by : 1.f;
    return large ? s * by : s;
}

template <int HD, bool kNorm, RotateTo kTo>
__global__ void __launch_bounds__(kRotateThreads, 4) s2a_rotate_kernel(const __grid_constant__ RotateParams p) {
    using L = RowLanes<HD>;
    constexpr bool kCache = kTo != RotateTo::kTensors, kE4M3 = kTo == RotateTo::kCacheE4M3;
    extern __shared__ __align__(16) float s_table[];  // [tokens][kTable]
    __shared__ __align__(16) float s_weights[kNorm ? 2 : 1][kNorm ? HD : 1];
    __shared__ int s_place[kCache ? L::kGroups * kRowsOfLane : 1];            // of each token in the cache, -1: of no sequence
    __shared__ long long s_cached[kCache ? L::kGroups * kRowsOfLane : 1];     // its row of the pools in head 0, -1: no page
    release_successor();
    wait_for_predecessor();
    const int standing = *reinterpret_cast<volatile int*>(p.status);
    if (kCache && blockIdx.x == 0) check_batch(p.batch, p.pool.page_log2, 0x7fffffff, p.status, p.host_status);
    const int part = static_cast<int>(threadIdx.x) % L::kLanes, group = static_cast<int>(threadIdx.x) / L::kLanes;
    int within;
    const int t0 = p.blocks.by_count(static_cast<int>(blockIdx.x), &within) * p.blocks.tokens, tokens = min(p.blocks.tokens, p.T - t0);
    const int first = within * p.blocks.rows, rows = min(p.blocks.rows, tokens * p.blocks.all - first);
    if (rows <= 0) return;
    // this lane's rows: where they are, and what is there, before anything is known about their tokens
    struct Row {
        int token, kind, head;
        bool there;
    };
    auto row = [&](int i) -> Row {
        Row w;
        const int r = i * L::kGroups + group;
        w.there = r < rows;
        int h;
        w.token = p.blocks.by_heads(first + (w.there ? r : 0), &h);
        w.kind = p.blocks.kind(h, &w.head);
        return w;
    };
    uint4 x[kRowsOfLane][2];
#pragma unroll
    for (int i = 0; i < kRowsOfLane; ++i) {
        const Row w = row(i);
        const HeadRows& in = p.in[w.kind];
        x[i][0] = x[i][1] = make_uint4(0, 0, 0, 0);
        if (w.there) load_row(in.x + (t0 + w.token) * in.stride + w.head * HD, Pieces(part, w.kind == 2 ? 0 : p.rotation.r), x[i]);
    }
    // sines and cosines of the tokens that the block's rows belong to
    const int low = p.blocks.by_heads(first), high = p.blocks.by_heads(first + rows - 1);
    if constexpr (kCache) {
        for (int i = low + static_cast<int>(threadIdx.x); i <= high; i += kRotateThreads) {
            const int t = t0 + i, b = find_sequence(p.batch.starts, p.batch.B, t);
            Sequence s;
            int place = -1;
            long long cached = -1;
            if (sequence_of(p.batch, p.pool.page_log2, 0x7fffffff, b, &s) == 0 && t >= s.row0 && t < s.row0 + s.n) {
                place = s.length - s.n + t - s.row0;
                cached = pool_row(p.batch, p.pool, b, place);
                if (cached < 0) report_bad_index(p.status, p.host_status, kBadPage);
            }
            s_place[i - low] = place, s_cached[i - low] = cached;
        }
        if (!p.rotation.positions) __syncthreads();
    }
    const int pairs = p.rotation.r / 2;
    for (int i = threadIdx.x; i < (high - low + 1) * (HD / 2); i += kRotateThreads) {
        const int at = i / (HD / 2), pair = i % (HD / 2);
        if (pair < pairs)
            make_angle<HD>(s_table + at * L::kTable, p.rotation, pair, kCache && !p.rotation.positions ? s_place[at] : position_of(p.rotation, t0 + low + at), p.backwards);
    }
    if constexpr (kNorm) {
        for (int i = threadIdx.x; i < 2 * HD; i += kRotateThreads) stage_weights<HD>(s_weights[i / HD], p.rotation.weight[i / HD], p.rotation.weight_f32, p.rotation.r, i % HD);
    }
    __syncthreads();
    if (standing != 0) return;
    // (all lanes of a warp go through all rows: sums of a row are taken by the whole warp)
#pragma unroll
    for (int i = 0; i < kRowsOfLane; ++i) {
        const Row w = row(i);
        const Pieces pieces(part, w.kind == 2 ? 0 : p.rotation.r);
        const int t = t0 + w.token, at = w.token - low;
        float y[16];
        unpack_row(x[i], y);
        if constexpr (kNorm) {
            float rest;
            normalise_row<HD>(y, p.rotation.eps, &rest);
            times_weights<HD>(y, s_weights[w.kind == 0 ? 0 : 1], part);
        }
        if (w.kind != 2) {
            turn_row<HD>(y, s_table + at * L::kTable, pieces, part, p.rotation.interleaved);
            pack_row(y, x[i]);
        }
        if constexpr (kCache) {
            const bool mine = w.there && s_place[at] >= 0;
            const long long cached = s_cached[at], to = cached + (static_cast<long long>(w.head) << p.pool.page_log2);
            void* pool = w.kind == 2 ? p.pool.v : p.pool.k;
            if constexpr (kE4M3) {
              if (__any_sync(0xffffffffu, w.kind != 0)) {
                const uint32_t words[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
                uint32_t codes[4];
                const int exp = row_to_e4m3<L::kLanes>(words, codes);
                if (mine && w.kind != 0 && cached >= 0) {
                    uint8_t* cell = static_cast<uint8_t*>(pool) + to * HD;
                    *reinterpret_cast<uint2*>(cell + pieces.at[0]) = make_uint2(codes[0], codes[1]);
                    *reinterpret_cast<uint2*>(cell + pieces.at[1]) = make_uint2(codes[2], codes[3]);
                    if (part == 0) (w.kind == 2 ? p.pool.v_exp : p.pool.k_exp)[to] = static_cast<int8_t>(exp);
                }
              }
            } else if (mine && w.kind != 0 && cached >= 0) {
                store_row(static_cast<__nv_bfloat16*>(pool) + to * HD, pieces, x[i]);
            }
            if (mine && w.kind == 0) store_row(p.out[0] + t * p.out_stride[0] + w.head * HD, pieces, x[i]);
        } else if (w.there) {
            store_row(p.out[w.kind] + t * p.out_stride[w.kind] + w.head * HD, pieces, x[i]);
        }
    }
}

// Gradients through a norm.  A block has rows of q or of k alone, in chunks of a few tokens; its sums for the weight's gradient go to p.partial, in an
// order that the sizes and the number of multiprocessors fix.  The next chunk's sines and cosines are made before a chunk is worked on.  A lane's next
// rows are on their way to a place of its own in shared memory: the sums, a row and its gradient take the registers (with one row ahead in them 106 us for
// 8192 tokens of 64 + 8 heads, so 93).
constexpr int kBwdRowsOfLane = 4;  // of a chunk: in each of the four places one, so that three rows are on their way
constexpr int kBwdBlocks = 2;      // of a multiprocessor
constexpr int kAheadBytes = kBwdRowsOfLane * 4 * 16 * kRotateThreads;
template <int HD>
__global__ void __launch_bounds__(kRotateThreads, kBwdBlocks) s2a_rotate_bwd_kernel(const __grid_constant__ RotateBwdParams p) {
    using L = RowLanes<HD>;
    extern __shared__ __align__(16) uint4 s_rows[];  // [row ahead][two pieces of x, two of the gradient][threads], then the tables [2][tokens of a chunk][kTable]
    float* s_table = reinterpret_cast<float*>(s_rows + kAheadBytes / 16);
    __shared__ __align__(16) float s_weights[HD];
    __shared__ float s_sum[kRotateThreads / 32][HD];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    const int kind = static_cast<int>(blockIdx.x) < p.blocks[0] ? 0 : 1;
    const int part = static_cast<int>(threadIdx.x) % L::kLanes, group = static_cast<int>(threadIdx.x) / L::kLanes;
    const Pieces pieces(part, p.rotation.r);
    const HeadRows in = p.in[kind], grad = p.grad[kind];
    const FastDiv by_heads = p.by_heads[kind];
    const int tokens = p.tokens[kind], blocks = p.blocks[kind], chunks = p.chunks[kind], pairs = p.rotation.r / 2;
    constexpr int kRows = L::kGroups * kBwdRowsOfLane;  // of a chunk at most: some tokens', or a part of one's
    for (int i = threadIdx.x; i < HD; i += kRotateThreads) stage_weights<HD>(s_weights, p.rotation.weight[kind], p.rotation.weight_f32, p.rotation.r, i);
    auto angles = [&](int chunk, float* table) {
        for (int i = threadIdx.x; i < tokens * (HD / 2); i += kRotateThreads) {
            const int at = i / (HD / 2), pair = i % (HD / 2), t = p.by_parts[kind](chunk) * tokens + at;
            if (pair < pairs && t < p.T) make_angle<HD>(table + at * L::kTable, p.rotation, pair, position_of(p.rotation, t), true);
        }
    };
    float sum[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    // this lane's rows of a chunk: token, and where they are from the chunk's first row on, in eights of values
    int at[kBwdRowsOfLane], x_from[kBwdRowsOfLane], g_from[kBwdRowsOfLane];
#pragma unroll
    for (int i = 0; i < kBwdRowsOfLane; ++i) {
        int head;
        at[i] = by_heads(i * L::kGroups + group, &head);
        if (tokens == 1) at[i] = 0, head = i * L::kGroups + group;  // (behind a part of its heads there are more)
        if (at[i] >= tokens) at[i] = 0, head = 0;                   // (there is none)
        x_from[i] = at[i] * static_cast<int>(in.stride / 8) + head * (HD / 8), g_from[i] = at[i] * static_cast<int>(grad.stride / 8) + head * (HD / 8);
    }
    // a chunk's rows, and the place of the first one: token, and head
    auto rows_of = [&](int chunk, int* token, int* head) -> int {
        if (chunk >= chunks) return 0;
        int part_of;
        *token = p.by_parts[kind](chunk, &part_of) * tokens, *head = part_of * kRows;
        return min(kRows, min(tokens, p.T - *token) * in.heads - *head);
    };
    uint4* const mine = s_rows + threadIdx.x;
    auto request = [&](int chunk, int i) {
        int token = 0, head = 0;
        const bool there = i * L::kGroups + group < rows_of(chunk, &token, &head);
        const __nv_bfloat16* x = in.x + (there ? token * in.stride + (head * HD + 8ll * x_from[i]) : 0);
        const __nv_bfloat16* g = grad.x + (there ? token * grad.stride + (head * HD + 8ll * g_from[i]) : 0);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            copy_async(mine + (4 * i + y) * kRotateThreads, x + pieces.at[y], there);
            copy_async(mine + (4 * i + 2 + y) * kRotateThreads, g + pieces.at[y], there);
        }
        copy_async_commit();
    };
    int chunk = static_cast<int>(blockIdx.x) - (kind ? p.blocks[0] : 0);
#pragma unroll
    for (int i = 0; i < kBwdRowsOfLane - 1; ++i) request(chunk, i);
    if (chunk < chunks) angles(chunk, s_table);
    for (int turn = 0; chunk < chunks; chunk += blocks, turn ^= 1) {
        __syncthreads();  // this chunk's table is there, and the other one is free
        if (chunk + blocks < chunks) angles(chunk + blocks, s_table + (turn ^ 1) * tokens * L::kTable);
        const float* table = s_table + turn * tokens * L::kTable;
        int token = 0, first_head = 0;
        const int rows = rows_of(chunk, &token, &first_head);
        __nv_bfloat16* const out = p.out[kind] + (static_cast<long long>(token) * in.heads + first_head + group) * HD;
#pragma unroll
        for (int i = 0; i < kBwdRowsOfLane; ++i) {
            request(i == 0 ? chunk : chunk + blocks, (i + kBwdRowsOfLane - 1) % kBwdRowsOfLane);
            copy_async_wait<kBwdRowsOfLane - 1>();
            const bool there = i * L::kGroups + group < rows;
            float x[16], g[16];
            {
                const uint4* from = mine + 4 * i * kRotateThreads;
                const uint4 now_x[2] = {from[0], from[kRotateThreads]}, now_g[2] = {from[2 * kRotateThreads], from[3 * kRotateThreads]};
                unpack_row(now_x, x);
                unpack_row(now_g, g);
            }
            turn_row<HD>(g, table + at[i] * L::kTable, pieces, part, p.rotation.interleaved);
            float rest;
            const float s = normalise_row<HD>(x, p.rotation.eps, &rest);
            if (there) {
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e] += g[e] * x[e];
            }
            times_weights<HD>(g, s_weights, part);
            float mean = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) mean += g[e] * x[e];
            mean = sum_of_row<HD>(mean) * (1.f / HD);
#pragma unroll
            for (int e = 0; e < 16; ++e) g[e] = s * (g[e] - x[e] * mean);
            if (rest != 1.f) {
#pragma unroll
                for (int e = 0; e < 16; ++e) g[e] *= rest;
            }
            uint4 w[2];
            pack_row(g, w);
            if (there) store_row(out + i * L::kGroups * HD, pieces, w);
        }
    }
    // the block's sums: over the rows of a warp, then over the warps
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int off = L::kLanes; off < 32; off <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
        if ((threadIdx.x & 31) < L::kLanes) s_sum[threadIdx.x / 32][pieces.at[i / 8] + i % 8] = sum[i];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < HD; c += kRotateThreads) {
        float all = 0.f;
        for (int i = 0; i < kRotateThreads / 32; ++i) all += s_sum[i][c];
        p.partial[static_cast<long long>(blockIdx.x) * HD + c] = all;
    }
}

// The weights' gradients from the blocks' sums: one block for q's and one for k's.
constexpr int kJoinThreads = 1024;
template <int HD>
__global__ void __launch_bounds__(kJoinThreads) s2a_rotate_join_kernel(const __grid_constant__ RotateBwdParams p) {
    constexpr int kSlices = kJoinThreads / HD;
    __shared__ float s_sum[kSlices][HD];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    const int kind = blockIdx.x, c = static_cast<int>(threadIdx.x) % HD, slice = static_cast<int>(threadIdx.x) / HD;
    const float* from = p.partial + static_cast<long long>(kind ? p.blocks[0] : 0) * HD + c;
    float sum = 0.f;
    for (int i = slice; i < p.blocks[kind]; i += kSlices) sum += __ldcg(from + static_cast<long long>(i) * HD);
    s_sum[slice][c] = sum;
    __syncthreads();
    if (slice != 0 || !p.weight_grad[kind]) return;
    for (int i = 1; i < kSlices; ++i) sum += s_sum[i][c];
    p.weight_grad[kind][c] = sum;
}

template <int HD, bool kNorm, RotateTo kTo>
cudaError_t launch_one(const RotateParams& p, cudaStream_t stream) {
    const long long tiles = (p.T + p.blocks.tokens - 1) / p.blocks.tokens;
    const int smem = std::min(p.blocks.tokens, (p.blocks.rows - 1) / p.blocks.all + 2) * RowLanes<HD>::kTable * static_cast<int>(sizeof(float));
    return launch_kernel(s2a_rotate_kernel<HD, kNorm, kTo>, static_cast<unsigned>(tiles * p.blocks.count), kRotateThreads, smem, stream, p, true);
}
template <int HD, RotateTo kTo>
cudaError_t launch_any(const RotateParams& p, bool norm, cudaStream_t stream) {
    return norm ? launch_one<HD, true, kTo>(p, stream) : launch_one<HD, false, kTo>(p, stream);
}
template <RotateTo kTo>
cudaError_t launch_to(const RotateParams& p, bool norm, int d, cudaStream_t stream) {
    return d == 64 ? launch_any<64, kTo>(p, norm, stream) : launch_any<128, kTo>(p, norm, stream);
}

template <int HD>
cudaError_t launch_gradients(const RotateBwdParams& p, cudaStream_t stream) {
    const int smem = kAheadBytes + 2 * std::max(p.tokens[0], p.tokens[1]) * RowLanes<HD>::kTable * static_cast<int>(sizeof(float));
    const cudaError_t e = launch_kernel(s2a_rotate_bwd_kernel<HD>, static_cast<unsigned>(p.blocks[0] + p.blocks[1]), kRotateThreads, smem, stream, p, true);
    return e != cudaSuccess ? e : launch_kernel(s2a_rotate_join_kernel<HD>, 2u, kJoinThreads, 0, stream, p, true);
}

}  // namespace

cudaError_t configure_rotate() {
    // (two chunks' tables are 32 KB at most)
    const cudaError_t e = cudaFuncSetAttribute(s2a_rotate_bwd_kernel<64>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAheadBytes + 32768);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(s2a_rotate_bwd_kernel<128>, cudaFuncAttributeMaxDynamicSharedMemorySize, kAheadBytes + 32768);
}

cudaError_t launch_rotate(const RotateParams& p, RotateTo to, bool norm, int d, cudaStream_t stream) {
    if (to == RotateTo::kTensors) return launch_to<RotateTo::kTensors>(p, norm, d, stream);
    return to == RotateTo::kCacheBf16 ? launch_to<RotateTo::kCacheBf16>(p, norm, d, stream) : launch_to<RotateTo::kCacheE4M3>(p, norm, d, stream);
}
cudaError_t launch_rotate_bwd(const RotateBwdParams& p, int d, cudaStream_t stream) {
    return d == 64 ? launch_gradients<64>(p, stream) : launch_gradients<128>(p, stream);
}
int rotate_rows(int d) { return (d == 64 ? RowLanes<64>::kGroups : RowLanes<128>::kGroups) * kRowsOfLane; }
int rotate_bwd_blocks(int n_sm) { return kBwdBlocks * n_sm; }
int rotate_bwd_rows(int d) { return (d == 64 ? RowLanes<64>::kGroups : RowLanes<128>::kGroups) * kBwdRowsOfLane; }

}  // namespace s2a
