// What attention weight cached tokens get from the new tokens of a call.
//
// With p the position of a new token, s = scale * q . k_j over the keys j it attends and lse the logarithm of the sum of its exp(s): key j of a
// KV head gets w_j = sum exp(s - lse) over the head's query heads and the new tokens that attend j.  The sums go over rows, one for every key, so
// here, unlike in attention itself, keys stand still and rows stream past: a key's sum lives in one place and is written once, in an order that
// the sizes fix.
//
// Few rows (new tokens x query heads of a KV head): the streaming kernel.  A warp takes 16 keys at a time as the rows of S^T = K Q^T on mma.sync, eight
// rows of q as its columns.  An instruction's 16 values of the contraction may be any, as long as K and Q agree, so a lane takes 16 bytes
// of a key at a time (half of two instructions' worth, of 8-bit codes of four) straight from global memory to registers, the next 16
// keys' on their way; q lies in shared memory in the order in which lanes need it.  Each key is read once; what bounds the kernel is a block's start
// (addresses, pages and q one after the other, 2 to 3 us) and a warp's chain loads -> products -> exponentials, so it wants many warps and long pieces: 16
// x up to 8192 tokens of 32 heads 113 us (5.4 TB/s) in pieces of 1024 keys, 124 of 512, 144 of 256; 8 x up to 32k of 64 heads over 8 in 8 bits 59 us with
// six blocks on a multiprocessor (with four a sixth more).  Keys through a ring in shared memory, two or three turns ahead, left room for fewer blocks:
// 145 and 81 us.
//
// 8-bit caches are multiplied in fp16, which has their codes exactly.  Each row of q goes with a power of two that brings its largest value to
// [2^14, 2^15).  Its exponent, the key's and that of the scale are added up before one power of two multiplies the score in fp32: the product of any
// two of them may be out of range where the score is not.
#include <cuda_fp16.h>

#include "evict.h"
#include "paged_device.cuh"

namespace s2a {

namespace {

constexpr int kStreamThreads = 128;
constexpr int kMostChunkPages = 64;   // of a block's keys: 1024 keys in pages of 16

template <int HD, bool kE4M3>
struct StreamCfg {
    static constexpr int kSteps = HD / 16;                       // instructions for 16 keys and 8 rows
    static constexpr int kPieces = HD * (kE4M3 ? 1 : 2) / 64;    // of 16 bytes that a lane has of a key
    static constexpr int kStepsOfPiece = kE4M3 ? 4 : 2;
    // the first of four values that lane t of four has of step s
    __device__ static constexpr int value(int s, int t) { return (kE4M3 ? 16 : 8) * (t + 4 * (s / kStepsOfPiece)) + 4 * (s % kStepsOfPiece); }
};

// Rows of q of a sequence and KV head: row r is token r / rep, head r % rep of the KV head's.  s_exp (8 bits): a row's exponent, for score_power().
template <int HD, bool kE4M3>
__device__ __forceinline__ void stage_rows(const WeightsParams& a, const Sequence& s, int hk, int rows, uint2* s_q, float* s_lse, int* s_exp, int* s_pos) {
    using C = StreamCfg<HD, kE4M3>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int padded = (rows + 7) & ~7;
    // four lanes have a row: its values in the order of the steps
    for (int base = warp * 8; base < padded; base += kStreamThreads / 32 * 8) {
        const int r = base + lane / 4, t = lane % 4;
        const bool there = r < rows;
        const int token = (there ? r : 0) / a.rep, head = hk * a.rep + (there ? r : 0) % a.rep;
        const __nv_bfloat16* q = a.q + (static_cast<long long>(s.row0 + token) * a.H + head) * HD;
        uint2 w[C::kSteps];
#pragma unroll
        for (int x = 0; x < C::kSteps; ++x) w[x] = there ? __ldcg(reinterpret_cast<const uint2*>(q + C::value(x, t))) : make_uint2(0, 0);
        int exp = 0;
        if constexpr (kE4M3) {
            uint32_t most = 0;
#pragma unroll
            for (int x = 0; x < C::kSteps; ++x) {
                const uint32_t m = __vmaxu2(w[x].x & 0x7fff7fffu, w[x].y & 0x7fff7fffu);
                most = max(most, max(m & 0xffffu, m >> 16));
            }
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // (an infinity or a NaN stays one)
            const int e = most >= 0x7f80u ? 0 : max(static_cast<int>(most >> 7) - 127 - 14, -126);
            const float up = power_of_two(-e);
#pragma unroll
            for (int x = 0; x < C::kSteps; ++x) {
                w[x].x = pack_f16(bf16_low(w[x].x) * up, bf16_high(w[x].x) * up);
                w[x].y = pack_f16(bf16_low(w[x].y) * up, bf16_high(w[x].y) * up);
            }
            exp = a.scale_exp + e;
        }
#pragma unroll
        for (int x = 0; x < C::kSteps; ++x) s_q[((base / 8) * C::kSteps + x) * 32 + lane] = w[x];
        if (t == 0) {
            s_lse[r] = there ? __ldcg(a.lse + static_cast<long long>(head) * a.batch.T + s.row0 + token) * 1.4426950408889634f : __uint_as_float(0x7f800000u);
            if constexpr (kE4M3) s_exp[r] = exp;
            s_pos[r] = there ? s.length - s.n + token : -1;
        }
    }
}

// What the product of an 8-bit key with a row of q is multiplied with: 2^(key_exp + row_exp - 127), held to what fp32 has.  Zero below 2^-126 (products
// are below 2^31, so such a score does not count), and 2^127 above that: a product of zero is a score of zero, whatever the power.
__device__ __forceinline__ float score_power(int key_exp, int row_exp) {
    return __uint_as_float(static_cast<uint32_t>(__viaddmin_s32_relu(key_exp, row_exp, 254)) << 23);
}

// Keys from `row` of the pools on, 16 of them: a lane's pieces of keys lane / 4 and lane / 4 + 8.
template <int HD, bool kE4M3>
__device__ __forceinline__ void load_keys(const WeightsParams& a, long long row, uint4 (&w)[2][StreamCfg<HD, kE4M3>::kPieces], int (&e)[2]) {
    const int g = (threadIdx.x & 31) / 4, t = threadIdx.x & 3;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
        const uint8_t* key = static_cast<const uint8_t*>(a.pool.k) + (row + g + 8 * y) * (HD * (kE4M3 ? 1 : 2));
#pragma unroll
        for (int x = 0; x < StreamCfg<HD, kE4M3>::kPieces; ++x) w[y][x] = __ldcg(reinterpret_cast<const uint4*>(key) + t + 4 * x);
        if constexpr (kE4M3) e[y] = __ldcg(reinterpret_cast<const signed char*>(a.pool.k_exp) + row + g + 8 * y);
    }
}

template <int HD, bool kE4M3>
__global__ void __launch_bounds__(kStreamThreads, kE4M3 ? 6 : 4) s2a_weights_stream_kernel(const __grid_constant__ WeightsStreamParams p) {
    using C = StreamCfg<HD, kE4M3>;
    const WeightsParams& a = p.a;
    __shared__ uint2 s_q[kStreamedRows / 8 * C::kSteps * 32];
    __shared__ float s_lse[kStreamedRows];
    __shared__ int s_pos[kStreamedRows], s_exp[kStreamedRows];
    __shared__ int s_page[kMostChunkPages];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(a.status) != 0) return;
    if (blockIdx.x == 0) check_batch(a.batch, a.pool.page_log2, a.most_new, a.status, a.host_status);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, t = lane & 3;
    int chunk, hk;
    const int b = p.by_heads(p.by_chunks(static_cast<int>(blockIdx.x), &chunk), &hk);
    Sequence s;
    if (sequence_of(a.batch, a.pool.page_log2, a.most_new, b, &s) != 0 || s.n == 0 || s.n > a.few_rows / a.rep) return;
    const int first = s.length - s.n, last = s.length - 1, keys = 1 << p.chunk_log2;
    const KeyBlocks blocks = key_blocks(first, last, a.window, a.sinks, keys);
    if (chunk >= blocks.count) return;
    const int key0 = blocks.at(chunk) * keys;
    const HiddenKeys hidden = hidden_keys(first, last, key0, a.window, a.sinks);
    // the chunk's pages, of those keys that are attended
    const int page_keys = 1 << a.pool.page_log2;
    for (int i = threadIdx.x; i << a.pool.page_log2 < keys; i += kStreamThreads) {
        int page = -1;
        if (!hidden.all(i * page_keys, min(page_keys, keys))) {
            page = page_of(a.batch, a.pool.pages, b, (key0 >> a.pool.page_log2) + i);
            if (page < 0) report_bad_index(a.status, a.host_status, kBadPage);
        }
        s_page[i] = page;
    }
    // keys key0 + 16 i on: their row in the pools, -1 where none of them is attended or the page is not there
    auto row_of = [&](int i) -> long long {
        const int at = 16 * i;
        if (at >= keys || hidden.all(at, 16)) return -1;
        const int page = s_page[((key0 + at) >> a.pool.page_log2) - (key0 >> a.pool.page_log2)];
        if (page < 0) return -1;
        return ((static_cast<long long>(page) * a.pool.Hkv + hk) << a.pool.page_log2) + ((key0 + at) & (page_keys - 1));
    };
    const int rows = s.n * a.rep, groups = (rows + 7) / 8;
    stage_rows<HD, kE4M3>(a, s, hk, rows, s_q, s_lse, s_exp, s_pos);
    __syncthreads();
    uint4 next[2][C::kPieces];
    int next_e[2] = {0, 0};
    long long next_row = row_of(warp);
    if (next_row >= 0) load_keys<HD, kE4M3>(a, next_row, next, next_e);
    for (int i = warp; 16 * i < keys; i += kStreamThreads / 32) {
        const long long row = next_row;
        uint4 now[2][C::kPieces];
        const int now_e[2] = {next_e[0], next_e[1]};
#pragma unroll
        for (int y = 0; y < 2; ++y) {
#pragma unroll
            for (int x = 0; x < C::kPieces; ++x) now[y][x] = next[y][x];
        }
        next_row = row_of(i + kStreamThreads / 32);
        if (next_row >= 0) load_keys<HD, kE4M3>(a, next_row, next, next_e);
        if (row < 0) continue;
        const int j = key0 + 16 * i + lane / 4;  // this lane's keys are j and j + 8
        const bool whole = all_attend(first, last, key0 + 16 * i, 16, a.window, a.sinks);
        float sum[2];  // (of an 8-bit key that is NaN throughout a NaN)
#pragma unroll
        for (int y = 0; y < 2; ++y) sum[y] = kE4M3 && now_e[y] == kExpNotFinite ? __uint_as_float(0x7fffffffu) : 0.f;
        for (int group = 0; group < groups; ++group) {
            float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < C::kSteps; ++x) {
                const uint2 q = s_q[(group * C::kSteps + x) * 32 + lane];
                const uint4 &k0 = now[0][x / C::kStepsOfPiece], &k1 = now[1][x / C::kStepsOfPiece];
                const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
                const int at = x % C::kStepsOfPiece;
                if constexpr (kE4M3) {
                    uint32_t l0, h0, l1, h1;
                    e4m3_to_f16(w0[at], l0, h0);
                    e4m3_to_f16(w1[at], l1, h1);
                    mma_16x8x16<true>(c, l0, l1, h0, h1, q.x, q.y);
                } else {
                    mma_16x8x16<false>(c, w0[2 * at], w1[2 * at], w0[2 * at + 1], w1[2 * at + 1], q.x, q.y);
                }
            }
            const int r = 8 * group + 2 * t;
            const float2 lse = *reinterpret_cast<const float2*>(s_lse + r);
            int2 exp = {0, 0};
            if constexpr (kE4M3) exp = *reinterpret_cast<const int2*>(s_exp + r);
            const float scale = kE4M3 ? a.scale_part : a.scale_log2;
            float w[2][2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float s0 = c[2 * y], s1 = c[2 * y + 1];
                if constexpr (kE4M3) s0 *= score_power(now_e[y], exp.x), s1 *= score_power(now_e[y], exp.y);
                w[y][0] = fast_exp2(fmaf(s0, scale, -lse.x)), w[y][1] = fast_exp2(fmaf(s1, scale, -lse.y));
            }
            if (!whole || 8 * group + 8 > rows) {  // (else all eight rows are there and attend all of these keys)
                const int2 pos = *reinterpret_cast<const int2*>(s_pos + r);  // (below zero: no such row)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    if (whole ? pos.x < 0 : !attends(pos.x, j + 8 * y, a.window, a.sinks)) w[y][0] = 0.f;
                    if (whole ? pos.y < 0 : !attends(pos.y, j + 8 * y, a.window, a.sinks)) w[y][1] = 0.f;
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) sum[y] += w[y][0] + w[y][1];
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
            sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 1);
            sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], 2);
        }
        // lanes 0 and 1 of a key's four write keys j and j + 8
        const int mine = j + 8 * t;
        if (t < 2 && any_attends(first, last, mine, a.window, a.sinks)) {
            const long long at = row + mine - (key0 + 16 * i);
            a.received[at] = (a.before && mine < first ? __ldcg(a.before + at) : 0.f) + (t == 0 ? sum[0] : sum[1]);
        }
    }
}

template <int HD, bool kE4M3>
cudaError_t launch_stream(const WeightsStreamParams& p, cudaStream_t stream) {
    return launch_kernel(s2a_weights_stream_kernel<HD, kE4M3>, static_cast<unsigned>(p.blocks), kStreamThreads, 0, stream, p, true);
}

}  // namespace

cudaError_t launch_weights_stream(const WeightsStreamParams& p, bool e4m3, int d, cudaStream_t stream) {
    if (d == 64) return e4m3 ? launch_stream<64, true>(p, stream) : launch_stream<64, false>(p, stream);
    return e4m3 ? launch_stream<128, true>(p, stream) : launch_stream<128, false>(p, stream);
}

}  // namespace s2a
