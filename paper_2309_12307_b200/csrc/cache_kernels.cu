// New tokens into the paged cache, and back.
//
// A block takes a few tokens with all their heads, k and v: one thread for each token finds its sequence and page, then a few lanes take a row
// of d values, 16 or 32 bytes of bf16 a lane.  Both directions move each byte once; what bounds them is HBM, and for a step of single
// tokens the launch.  So a thread has the loads of four rows in flight, and when it writes those of its first rows before it is known where
// they go.  8192 and 5735 tokens of 32 heads of 128: 64 us into 8 bits and 68 back (5.4 and 5.0 TB/s), 73 and 73 in bf16 (6.2 TB/s); with one row
// at a time 82 and 82 in 8 bits.
#include <cuda_fp16.h>

#include <type_traits>

#include "paged_device.cuh"

namespace s2a {

namespace {

constexpr int kCopyThreads = 256;
constexpr int kMostTokens = 64;  // of a block

template <int HD, bool kE4M3, bool kWrite>
struct CopyCfg {
    // Of a lane.  16 codes are stored at once; eight of them are loaded, so that what they stand for, 16 bytes a lane, lies together
    // for a warp's store (with 16 a lane every store instruction fills half of its sectors).
    static constexpr int kValues = kE4M3 && kWrite ? 16 : 8;
    static constexpr int kLanes = HD / kValues;  // lanes of a row
    static constexpr int kRowsAtOnce = kCopyThreads / kLanes;
    static constexpr int kRows = 4;              // of a thread
    using Cached = typename std::conditional<kE4M3 && !kWrite, uint2, uint4>::type;
};

template <int HD, bool kE4M3, bool kWrite>
__global__ void __launch_bounds__(kCopyThreads) s2a_cache_copy_kernel(const __grid_constant__ CacheCopyParams p) {
    using C = CopyCfg<HD, kE4M3, kWrite>;
    using Cached = typename C::Cached;
    __shared__ long long s_row[kMostTokens];  // pool row of each token in head 0, -1 = none
    release_successor();
    wait_for_predecessor();
    const int standing = *reinterpret_cast<volatile int*>(p.status);
    if (blockIdx.x == 0) check_batch(p.batch, p.pool.page_log2, 0x7fffffff, p.status, p.host_status);
    const int t0 = static_cast<int>(blockIdx.x) * p.tokens_per_block;
    if (static_cast<int>(threadIdx.x) < p.tokens_per_block) {
        const int t = t0 + static_cast<int>(threadIdx.x);
        long long row = -1;
        if (t < p.batch.T && standing == 0) {
            const int b = find_sequence(p.batch.starts, p.batch.B, t);
            Sequence s;
            if (sequence_of(p.batch, p.pool.page_log2, 0x7fffffff, b, &s) == 0 && t >= s.row0 && t < s.row0 + s.n) {
                row = pool_row(p.batch, p.pool, b, s.length - s.n + t - s.row0);
                if (row < 0) report_bad_index(p.status, p.host_status, kBadPage);
            }
        }
        s_row[threadIdx.x] = row;
    }
    const int part = static_cast<int>(threadIdx.x) % C::kLanes;
    // rows of the block: of each token the heads of k, then of v
    const int rows = p.tokens_per_block * 2 * p.pool.Hkv;
    for (int turn = 0; turn < rows; turn += C::kRows * C::kRowsAtOnce) {
        const int first = turn + static_cast<int>(threadIdx.x) / C::kLanes;
        uint4 x[C::kRows][C::kValues / 8];  // bf16
        Cached code[C::kRows];
        int e[C::kRows];
        uint4* dense[C::kRows];
        Cached* cached[C::kRows];  // nullptr: no such row
        int8_t* exponent[C::kRows];
        int token[C::kRows], h[C::kRows];
#pragma unroll
        for (int i = 0; i < C::kRows; ++i) {
            const int r = first + i * C::kRowsAtOnce;
            token[i] = p.by_rows(r < rows ? r : 0, &h[i]);
            const bool is_v = h[i] >= p.pool.Hkv;
            const int hk = is_v ? h[i] - p.pool.Hkv : h[i];
            dense[i] = reinterpret_cast<uint4*>((is_v ? p.v : p.k) + (static_cast<long long>(t0 + token[i]) * p.pool.Hkv + hk) * HD + C::kValues * part);
#pragma unroll
            for (int y = 0; y < C::kValues / 8; ++y) {
                x[i][y] = make_uint4(0, 0, 0, 0);
                if (kWrite && r < rows && t0 + token[i] < p.batch.T) x[i][y] = __ldcg(dense[i] + y);  // before it is known where they go
            }
        }
        if (turn == 0) __syncthreads();  // s_row is there
#pragma unroll
        for (int i = 0; i < C::kRows; ++i) {
            const long long base = first + i * C::kRowsAtOnce < rows ? s_row[token[i]] : -1;
            const bool is_v = h[i] >= p.pool.Hkv;
            const long long row = base + (static_cast<long long>(is_v ? h[i] - p.pool.Hkv : h[i]) << p.pool.page_log2);
            cached[i] = base < 0 ? nullptr : reinterpret_cast<Cached*>(static_cast<uint8_t*>(is_v ? p.pool.v : p.pool.k) + row * (HD * (kE4M3 ? 1 : 2))) + part;
            exponent[i] = kE4M3 ? (is_v ? p.pool.v_exp : p.pool.k_exp) + row : nullptr;
            if (!kWrite && cached[i]) {
                code[i] = __ldcg(cached[i]);
                if constexpr (kE4M3) e[i] = __ldcg(reinterpret_cast<const signed char*>(exponent[i]));
            }
        }
#pragma unroll
        for (int i = 0; i < C::kRows; ++i) {
            if constexpr (!kE4M3) {
                if (cached[i]) {
                    if constexpr (kWrite) *cached[i] = x[i][0];
                    else *dense[i] = code[i];
                }
            } else if constexpr (kWrite) {
                const uint32_t w[8] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w, x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
                uint32_t pair = 0;  // the largest magnitudes of either half (a NaN stays one)
#pragma unroll
                for (int c = 0; c < 8; ++c) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(pair) : "r"(w[c] & 0x7fff7fffu));
                uint32_t most = max(pair & 0xffffu, pair >> 16);
                // (all lanes of a warp are here: a block's rows are gone through in whole turns)
#pragma unroll
                for (int off = C::kLanes / 2; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
                const int exp = row_exponent(most);
                uint32_t codes[4] = {};
                if (exp != kExpNotFinite) {
                    const float down = __uint_as_float(static_cast<uint32_t>(127 - exp) << 23);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint16_t two[2];
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            float a = bf16_low(w[2 * c + y]) * down, b = bf16_high(w[2 * c + y]) * down;
                            // 256 * 2^120 would be no bf16 number: the next smaller code
                            if (exp == 120) a = fminf(fmaxf(a, -240.f), 240.f), b = fminf(fmaxf(b, -240.f), 240.f);
                            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two[y]) : "f"(b), "f"(a));
                        }
                        asm("mov.b32 %0, {%1, %2};" : "=r"(codes[c]) : "h"(two[0]), "h"(two[1]));
                    }
                }
                if (cached[i]) {
                    *cached[i] = make_uint4(codes[0], codes[1], codes[2], codes[3]);
                    if (part == 0) *exponent[i] = static_cast<int8_t>(exp);
                }
            } else if (cached[i]) {
                const float f = e[i] == kExpNotFinite ? __uint_as_float(0x7fffffffu) : __uint_as_float(static_cast<uint32_t>(127 + e[i]) << 23);
                uint32_t out[4];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    uint32_t lo, hi;
                    e4m3_to_f16(y ? code[i].y : code[i].x, lo, hi);
                    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo)), b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                    out[2 * y] = pack_bf16(a.x * f, a.y * f), out[2 * y + 1] = pack_bf16(b.x * f, b.y * f);
                }
                *dense[i] = make_uint4(out[0], out[1], out[2], out[3]);
            }
        }
    }
}

template <int HD, bool kE4M3, bool kWrite>
cudaError_t launch_one(const CacheCopyParams& p, cudaStream_t stream) {
    using C = CopyCfg<HD, kE4M3, kWrite>;
    CacheCopyParams q = p;
    const int heads = 2 * p.pool.Hkv, turn = C::kRows * C::kRowsAtOnce;
    // about as many tokens as make one turn of the block
    q.tokens_per_block = turn / heads;
    if (q.tokens_per_block < 1) q.tokens_per_block = 1;
    if (q.tokens_per_block > kMostTokens) q.tokens_per_block = kMostTokens;
    q.by_rows = FastDiv(heads);
    const unsigned grid = static_cast<unsigned>((p.batch.T + q.tokens_per_block - 1) / q.tokens_per_block);
    return launch_kernel(s2a_cache_copy_kernel<HD, kE4M3, kWrite>, grid, kCopyThreads, 0, stream, q, true);
}

template <bool kWrite>
cudaError_t launch_copy(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream) {
    if (d == 64) return e4m3 ? launch_one<64, true, kWrite>(p, stream) : launch_one<64, false, kWrite>(p, stream);
    return e4m3 ? launch_one<128, true, kWrite>(p, stream) : launch_one<128, false, kWrite>(p, stream);
}

}  // namespace

cudaError_t launch_cache_write(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream) { return launch_copy<true>(p, e4m3, d, stream); }
cudaError_t launch_cache_read(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream) { return launch_copy<false>(p, e4m3, d, stream); }

}  // namespace s2a
