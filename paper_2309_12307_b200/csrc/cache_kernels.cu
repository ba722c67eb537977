// New tokens into the paged cache, and back.
//
// A block takes a few tokens with all their heads, k and v: one thread for each token finds its sequence and page, then
// 8 or 16 lanes take a row of d values, 16 bytes of bf16 a lane.  Both directions move each byte once; what bounds them
// is HBM, and for a step of single tokens the launch.
#include "paged_device.cuh"

namespace s2a {

namespace {

constexpr int kCopyThreads = 256;
constexpr int kMostTokens = 32;  // of a block

template <int HD, bool kE4M3, bool kWrite>
__global__ void __launch_bounds__(kCopyThreads) s2a_cache_copy_kernel(const CacheCopyParams p) {
    constexpr int kLanes = HD / 8;  // lanes of a row
    constexpr int kRowsAtOnce = kCopyThreads / kLanes;
    __shared__ long long s_row[kMostTokens];  // pool row of each token in head 0, -1 = none
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    if (blockIdx.x == 0) check_batch(p.batch, p.pool.page_log2, 0x7fffffff, p.status, p.host_status);
    const int t0 = static_cast<int>(blockIdx.x) * p.tokens_per_block;
    if (static_cast<int>(threadIdx.x) < p.tokens_per_block) {
        const int t = t0 + static_cast<int>(threadIdx.x);
        long long row = -1;
        if (t < p.batch.T) {
            const int b = find_sequence(p.batch.starts, p.batch.B, t);
            Sequence s;
            if (sequence_of(p.batch, p.pool.page_log2, 0x7fffffff, b, &s) == 0 && t >= s.row0 && t < s.row0 + s.n) {
                row = pool_row(p.batch, p.pool, b, s.length - s.n + t - s.row0);
                if (row < 0) report_bad_index(p.status, p.host_status, kBadPage);
            }
        }
        s_row[threadIdx.x] = row;
    }
    __syncthreads();
    const int part = static_cast<int>(threadIdx.x) % kLanes;
    const int heads = 2 * p.pool.Hkv;  // k's, then v's
    // all lanes of a warp take the same number of turns: the row's maximum is found with shuffles
    const int rows = p.tokens_per_block * heads;
    for (int first = 0; first < rows; first += kRowsAtOnce) {
        const int r = first + static_cast<int>(threadIdx.x) / kLanes;
        const int i = r / heads, h = r - i * heads;
        const long long base = r < rows ? s_row[i] : -1;
        const bool is_v = h >= p.pool.Hkv;
        const int hk = is_v ? h - p.pool.Hkv : h;
        const long long row = base + (static_cast<long long>(hk) << p.pool.page_log2);
        __nv_bfloat16* dense = (is_v ? p.v : p.k) + (static_cast<long long>(t0 + i) * p.pool.Hkv + hk) * HD + 8 * part;
        void* pool = is_v ? p.pool.v : p.pool.k;
        if constexpr (!kE4M3) {
            uint4* cached = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(pool) + row * HD + 8 * part);
            if (base >= 0) {
                if constexpr (kWrite) *cached = *reinterpret_cast<const uint4*>(dense);
                else *reinterpret_cast<uint4*>(dense) = *cached;
            }
        } else {
            uint2* cached = reinterpret_cast<uint2*>(static_cast<uint8_t*>(pool) + row * HD + 8 * part);
            int8_t* exponent = (is_v ? p.pool.v_exp : p.pool.k_exp) + row;
            if constexpr (kWrite) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (base >= 0) x = *reinterpret_cast<const uint4*>(dense);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
                uint32_t most = 0;
#pragma unroll
                for (int c = 0; c < 4; ++c) most = max(most, max(w[c] & 0x7fffu, w[c] >> 16 & 0x7fffu));
#pragma unroll
                for (int off = kLanes / 2; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
                const int e = row_exponent(most);
                uint32_t codes[2] = {0, 0};
                if (e != kExpNotFinite) {
                    const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
                    // 256 * 2^120 would be no bf16 number: the next smaller code
                    const float limit = e == 120 ? 240.f : 448.f;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float a = fminf(fmaxf(bf16_low(w[c]) * down, -limit), limit), b = fminf(fmaxf(bf16_high(w[c]) * down, -limit), limit);
                        uint16_t two;
                        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(b), "f"(a));
                        codes[c >> 1] |= static_cast<uint32_t>(two) << (16 * (c & 1));
                    }
                }
                if (base >= 0) {
                    *cached = make_uint2(codes[0], codes[1]);
                    if (part == 0) *exponent = static_cast<int8_t>(e);
                }
            } else if (base >= 0) {
                const uint2 c = *cached;
                const RowFactor f = row_factor(*exponent);
                uint32_t lo[2], hi[2];
                e4m3_spread(c.x, lo[0], hi[0]);
                e4m3_spread(c.y, lo[1], hi[1]);
                uint4 x;
                uint32_t* out[2][2] = {{&x.x, &x.y}, {&x.z, &x.w}};
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t even = bf16x2_mul(bf16x2_mul(lo[u], f.first), f.second), odd = bf16x2_mul(bf16x2_mul(hi[u], f.first), f.second);
                    *out[u][0] = __byte_perm(even, odd, 0x5410);
                    *out[u][1] = __byte_perm(even, odd, 0x7632);
                }
                *reinterpret_cast<uint4*>(dense) = x;
            }
        }
    }
}

template <bool kWrite>
cudaError_t launch_copy(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream) {
    CacheCopyParams q = p;
    const int rows = 8 * (kCopyThreads / (d / 8));  // eight turns a block
    q.tokens_per_block = rows / (2 * p.pool.Hkv);
    if (q.tokens_per_block < 1) q.tokens_per_block = 1;
    if (q.tokens_per_block > kMostTokens) q.tokens_per_block = kMostTokens;
    const unsigned grid = static_cast<unsigned>((p.batch.T + q.tokens_per_block - 1) / q.tokens_per_block);
    auto kernel = d == 64 ? (e4m3 ? s2a_cache_copy_kernel<64, true, kWrite> : s2a_cache_copy_kernel<64, false, kWrite>)
                          : (e4m3 ? s2a_cache_copy_kernel<128, true, kWrite> : s2a_cache_copy_kernel<128, false, kWrite>);
    return launch_kernel(kernel, grid, kCopyThreads, 0, stream, q, true);
}

}  // namespace

cudaError_t launch_cache_write(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream) { return launch_copy<true>(p, e4m3, d, stream); }
cudaError_t launch_cache_read(const CacheCopyParams& p, bool e4m3, int d, cudaStream_t stream) { return launch_copy<false>(p, e4m3, d, stream); }

}  // namespace s2a
