// Norms of queries and keys for each head, and the rotation of positions in the same pass; forward, backward, and into the paged cache.
//
// A row is the d values of one head of a token.  With a norm y = w * x * s, s = 1 / sqrt(mean x^2 + eps), else y = x; then pair i of the
// first r values, (u, v) -> (u cos a - v sin a, u sin a + v cos a), a = position * frequency i.  Backwards the gradients of the
// pairs turn by -a, g; then the weight gets sum g * x * s, and x, with n = x * s, s (w g - n mean(w g * n)).  All of it in fp32, rounded to
// bf16 once.
//
// Angles: a frequency is a whole number of 2^-64 turns, so its product with a position, modulo 2^64, is the angle's fraction of a turn
// at any position; its upper 32 bits go to fp32 (off by 2^-25 of half a turn at most) and to sincospif.  A row is d / 16 lanes, a lane has both
// values of eight pairs (two pieces of 16 bytes, d / 8 or r / 2 values apart), so that only the sums of a norm cross lanes.  A lane's eight sines and cosines
// serve all heads of its item, a run of up to 8 heads of one token: of more is left for registers that hold loads in flight, and single
// tokens need their heads spread out.
//
// Bound by HBM: each value is read and written once (the backward of a norm reads two).
#include <cuda_fp16.h>

#include "paged_device.cuh"
#include "rotate.h"

namespace s2a {

namespace {

constexpr int kRotateThreads = 256;
constexpr int kAtOnce = 2;  // rows whose loads a lane has in flight

template <int HD>
struct RowLanes {
    static constexpr int kLanes = HD / 16;
    static constexpr int kGroups = kRotateThreads / kLanes;  // rows of a block at a time
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

// cos and sin of a lane's pairs: pair i < 8 is values i and 8 + i of its 16, or 2i and 2i + 1 where they are interleaved.
struct Angles {
    float cos[8], sin[8];
    __device__ __forceinline__ void set(const Rotation& ro, const Pieces& pieces, int position, bool backwards) {
        if (!pieces.turned) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int pair = !ro.interleaved ? pieces.at[0] + i : i < 4 ? pieces.at[0] / 2 + i : pieces.at[1] / 2 + i - 4;
            const unsigned long long turn = static_cast<unsigned long long>(static_cast<long long>(position)) * static_cast<unsigned long long>(S2A_LOAD(ro.turns + pair));
            sincospif(static_cast<float>(static_cast<int>(turn >> 32)) * 0x1p-31f, &sin[i], &cos[i]);
            if (backwards) sin[i] = -sin[i];
        }
    }
    __device__ __forceinline__ void turn(float (&x)[16], const Pieces& pieces, bool interleaved) const {
        if (!pieces.turned) return;
        auto pair = [&](float& u, float& v, int i) {
            const float a = u, b = v;
            u = a * cos[i] - b * sin[i], v = a * sin[i] + b * cos[i];
        };
        if (interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) pair(x[2 * i], x[2 * i + 1], i);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) pair(x[i], x[8 + i], i);
        }
    }
};

// A lane's weights of a norm.
__device__ __forceinline__ void load_weights(const void* weight, bool f32, const Pieces& pieces, float (&w)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int at = pieces.at[i / 8] + i % 8;
        w[i] = !weight ? 1.f : f32 ? S2A_LOAD(static_cast<const float*>(weight) + at)
                                   : __uint_as_float(static_cast<uint32_t>(S2A_LOAD(static_cast<const unsigned short*>(weight) + at)) << 16);
    }
}

// The sum over the lanes of a row.  `mask`: the lanes that are here.
template <int HD>
__device__ __forceinline__ float sum_of_row(float x, uint32_t mask = 0xffffffffu) {
#pragma unroll
    for (int off = RowLanes<HD>::kLanes / 2; off > 0; off >>= 1) x += __shfl_xor_sync(mask, x, off);
    return x;
}

// x times s = 1 / sqrt(mean x^2 + eps), which is returned; every lane of a row gets the same.  Squares that fp32 would not hold (values above
// 2^45, or, where eps does not matter either, below 2^-50) are taken of x times a power of two.
template <int HD>
__device__ __forceinline__ float normalise_row(float (&x)[16], float eps) {
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
    return s * by;
}

template <int HD, bool kNorm, RotateTo kTo>
__global__ void __launch_bounds__(kRotateThreads) s2a_rotate_kernel(const __grid_constant__ RotateParams p) {
    using L = RowLanes<HD>;
    constexpr bool kCache = kTo != RotateTo::kTensors, kE4M3 = kTo == RotateTo::kCacheE4M3;
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    if (kCache && blockIdx.x == 0) check_batch(p.batch, p.pool.page_log2, 0x7fffffff, p.status, p.host_status);
    const int part = static_cast<int>(threadIdx.x) % L::kLanes;
    const long long item = static_cast<long long>(blockIdx.x) * L::kGroups + threadIdx.x / L::kLanes;
    int run, head;
    bool there = item < static_cast<long long>(p.T) * p.runs.count;
    const int t = p.runs.by_count(there ? static_cast<int>(item) : 0, &run);
    const int kind = p.runs.kind(run, &head);
    const HeadRows in = p.in[kind];
    const int heads = min(p.runs.run, in.heads - head);
    const Pieces pieces(part, kind == 2 ? 0 : p.rotation.r);
    const __nv_bfloat16* row = in.x + t * in.stride + head * HD;
    uint4 next[kAtOnce][2];
    auto load = [&](int first) {
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            next[i][0] = next[i][1] = make_uint4(0, 0, 0, 0);
            if (there && first + i < heads) load_row(row + (first + i) * HD, pieces, next[i]);
        }
    };
    load(0);
    long long cached = -1;  // the token's row of the pools, in head 0
    int place = 0;
    if constexpr (kCache) {
        const int b = find_sequence(p.batch.starts, p.batch.B, t);
        Sequence s;
        there = there && sequence_of(p.batch, p.pool.page_log2, 0x7fffffff, b, &s) == 0 && t >= s.row0 && t < s.row0 + s.n;
        if (there) {
            place = s.length - s.n + t - s.row0;
            if (kind != 0) {
                cached = pool_row(p.batch, p.pool, b, place);
                if (cached < 0) report_bad_index(p.status, p.host_status, kBadPage), there = false;
            }
        }
    }
    Angles angles;
    float w[16];
    if (there && kind != 2) {
        angles.set(p.rotation, pieces, kCache && !p.rotation.positions ? place : position_of(p.rotation, t), p.backwards);
        if constexpr (kNorm) load_weights(p.rotation.weight[kind], p.rotation.weight_f32, pieces, w);
    }
    // (all lanes of a warp go through all turns: sums of a row are taken by the whole warp)
    for (int first = 0; first < p.runs.run; first += kAtOnce) {
        uint4 now[kAtOnce][2];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) now[i][0] = next[i][0], now[i][1] = next[i][1];
        load(first + kAtOnce);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            float x[16];
            unpack_row(now[i], x);
            if constexpr (kNorm) {
                normalise_row<HD>(x, p.rotation.eps);  // (by the whole warp)
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] *= w[e];
            }
            if (kind != 2) {
                angles.turn(x, pieces, p.rotation.interleaved);
                pack_row(x, now[i]);
            }
            const bool mine = there && first + i < heads;
            if constexpr (kCache) {
                const long long to = cached + (static_cast<long long>(head + first + i) << p.pool.page_log2);
                void* pool = kind == 2 ? p.pool.v : p.pool.k;
                if constexpr (kE4M3) {
                    const uint32_t words[8] = {now[i][0].x, now[i][0].y, now[i][0].z, now[i][0].w, now[i][1].x, now[i][1].y, now[i][1].z, now[i][1].w};
                    uint32_t codes[4];
                    const int exp = row_to_e4m3<L::kLanes>(words, codes);
                    if (mine && kind != 0) {
                        uint8_t* cell = static_cast<uint8_t*>(pool) + to * HD;
                        *reinterpret_cast<uint2*>(cell + pieces.at[0]) = make_uint2(codes[0], codes[1]);
                        *reinterpret_cast<uint2*>(cell + pieces.at[1]) = make_uint2(codes[2], codes[3]);
                        if (part == 0) (kind == 2 ? p.pool.v_exp : p.pool.k_exp)[to] = static_cast<int8_t>(exp);
                    }
                } else if (mine && kind != 0) {
                    store_row(static_cast<__nv_bfloat16*>(pool) + to * HD, pieces, now[i]);
                }
                if (mine && kind == 0) store_row(p.out[0] + t * p.out_stride[0] + (head + first + i) * HD, pieces, now[i]);
            } else if (mine) {
                store_row(p.out[kind] + t * p.out_stride[kind] + (head + first + i) * HD, pieces, now[i]);
            }
        }
    }
}

// Gradients through a norm.  A block has rows of q or of k alone; its sums for the weight's gradient go to p.partial, in an order that the sizes
// and the number of multiprocessors fix.
template <int HD>
__global__ void __launch_bounds__(kRotateThreads) s2a_rotate_bwd_kernel(const __grid_constant__ RotateBwdParams p) {
    using L = RowLanes<HD>;
    __shared__ float s_sum[kRotateThreads / 32][HD];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    const int kind = static_cast<int>(blockIdx.x) < p.blocks[0] ? 0 : 1;
    const int block = static_cast<int>(blockIdx.x) - (kind ? p.blocks[0] : 0);
    const int part = static_cast<int>(threadIdx.x) % L::kLanes;
    const Pieces pieces(part, p.rotation.r);
    const HeadRows in = p.in[kind], grad = p.grad[kind];
    const int run = p.run[kind], runs = static_cast<int>(p.by_runs[kind].d);
    const long long items = static_cast<long long>(p.T) * runs, stride = static_cast<long long>(p.blocks[kind]) * L::kGroups;
    float w[16], sum[16];
    load_weights(p.rotation.weight[kind], p.rotation.weight_f32, pieces, w);
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] = 0.f;
    const long long mine = static_cast<long long>(block) * L::kGroups + threadIdx.x / L::kLanes;
    // (whole turns for all lanes of a warp)
    for (long long item = mine; item - mine + static_cast<long long>(block) * L::kGroups < items; item += stride) {
        const bool there = item < items;
        int head;
        const int t = p.by_runs[kind](there ? static_cast<int>(item) : 0, &head);
        head *= run;
        const int heads = there ? min(run, in.heads - head) : 0;
        const __nv_bfloat16* x_row = in.x + t * in.stride + head * HD;
        const __nv_bfloat16* g_row = grad.x + t * grad.stride + head * HD;
        uint4 next_x[2], next_g[2];
        auto load = [&](int i) {
            next_x[0] = next_x[1] = next_g[0] = next_g[1] = make_uint4(0, 0, 0, 0);
            if (i < heads) load_row(x_row + i * HD, pieces, next_x), load_row(g_row + i * HD, pieces, next_g);
        };
        load(0);
        Angles angles;
        angles.set(p.rotation, pieces, position_of(p.rotation, t), true);
        for (int i = 0; i < run; ++i) {
            uint4 now[2];
            float x[16], g[16];
            unpack_row(next_x, x);
            unpack_row(next_g, g);
            load(i + 1);
            angles.turn(g, pieces, p.rotation.interleaved);
            const float s = normalise_row<HD>(x, p.rotation.eps);
            float mean = 0.f;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                if (i < heads) sum[e] += g[e] * x[e];
                g[e] *= w[e];
                mean += g[e] * x[e];
            }
            mean = sum_of_row<HD>(mean) * (1.f / HD);
#pragma unroll
            for (int e = 0; e < 16; ++e) g[e] = s * (g[e] - x[e] * mean);
            pack_row(g, now);
            if (i < heads) store_row(p.out[kind] + (static_cast<long long>(t) * in.heads + head + i) * HD, pieces, now);
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
    const long long items = static_cast<long long>(p.T) * p.runs.count;
    const unsigned grid = static_cast<unsigned>((items + RowLanes<HD>::kGroups - 1) / RowLanes<HD>::kGroups);
    return launch_kernel(s2a_rotate_kernel<HD, kNorm, kTo>, grid, kRotateThreads, 0, stream, p, true);
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
    const cudaError_t e = launch_kernel(s2a_rotate_bwd_kernel<HD>, static_cast<unsigned>(p.blocks[0] + p.blocks[1]), kRotateThreads, 0, stream, p, true);
    return e != cudaSuccess ? e : launch_kernel(s2a_rotate_join_kernel<HD>, 2u, kJoinThreads, 0, stream, p, true);
}

}  // namespace

cudaError_t launch_rotate(const RotateParams& p, RotateTo to, bool norm, int d, cudaStream_t stream) {
    if (to == RotateTo::kTensors) return launch_to<RotateTo::kTensors>(p, norm, d, stream);
    return to == RotateTo::kCacheBf16 ? launch_to<RotateTo::kCacheBf16>(p, norm, d, stream) : launch_to<RotateTo::kCacheE4M3>(p, norm, d, stream);
}
cudaError_t launch_rotate_bwd(const RotateBwdParams& p, int d, cudaStream_t stream) {
    return d == 64 ? launch_gradients<64>(p, stream) : launch_gradients<128>(p, stream);
}
int rotate_bwd_blocks(int n_sm) { return 4 * n_sm; }

}  // namespace s2a
