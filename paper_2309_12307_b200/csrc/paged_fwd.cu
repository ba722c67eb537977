// Attention of new tokens over the paged cache.
//
// With p the position of a new token, s_j = scale * q . k_j over the visible keys j <= p (with a window also j > p - window or
// j < sinks): o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m), lse = m + log of that sum, in one pass with a running
// maximum m.
//
// One warp for each new token and query head.  32 keys at a time: every lane has one key and its whole score, then every lane
// has d / 32 columns of o and adds the 32 weighted rows of v.
#include "paged_device.cuh"

namespace s2a {

namespace {

template <int HD, bool kE4M3>
__device__ __forceinline__ float cached_value(const void* pool, long long row, int c, float factor) {
    if constexpr (kE4M3) {
        uint32_t lo, hi;
        e4m3_spread(static_cast<const uint8_t*>(pool)[row * HD + c], lo, hi);
        return bf16_low(bf16x2_mul(lo, kTwoTo120)) * factor;
    } else {
        return __bfloat162float(static_cast<const __nv_bfloat16*>(pool)[row * HD + c]);
    }
}
__device__ __forceinline__ float exponent_factor(int e) {
    return e == kExpNotFinite ? __uint_as_float(0x7fffffffu) : __uint_as_float(static_cast<uint32_t>(127 + e) << 23);
}

template <int HD, bool kE4M3>
__global__ void __launch_bounds__(128) s2a_paged_fwd_kernel(const __grid_constant__ PagedFwdParams p) {
    constexpr int kCols = HD / 32;
    __shared__ float s_q[4][HD];
    release_successor();
    wait_for_predecessor();
    if (*reinterpret_cast<volatile int*>(p.status) != 0) return;
    if (blockIdx.x == 0) check_batch(p.batch, p.pool.page_log2, p.most_new, p.status, p.host_status);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long long id = static_cast<long long>(blockIdx.x) * 4 + warp;
    if (id >= static_cast<long long>(p.batch.T) * p.H) return;
    const int t = static_cast<int>(id / p.H), h = static_cast<int>(id % p.H), hk = h / p.rep;
    const int b = find_sequence(p.batch.starts, p.batch.B, t);
    Sequence s;
    if (sequence_of(p.batch, p.pool.page_log2, p.most_new, b, &s) != 0 || t < s.row0 || t >= s.row0 + s.n) return;
    if (s.n * p.rep <= p.few_rows) return;
    const int pos = s.length - s.n + t - s.row0;
    const int low = p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;  // first key of the window
    const int sinks = p.sinks < low ? p.sinks : low;
    for (int c = lane; c < HD; c += 32) s_q[warp][c] = __bfloat162float(p.q[(static_cast<long long>(t) * p.H + h) * HD + c]);
    __syncwarp();
    float m = -INFINITY, l = 0.f, acc[kCols] = {};
    const int visible = sinks + pos + 1 - low;
    for (int first = 0; first < visible; first += 32) {
        const int x = first + lane, j = x < sinks ? x : low + x - sinks;
        long long row = -1;
        float score = -INFINITY, v_factor = 1.f;
        if (x < visible) {
            row = pool_row(p.batch, p.pool, b, j);
            if (row < 0) report_bad_index(p.status, p.host_status, kBadPage);
        }
        if (row >= 0) {
            row += static_cast<long long>(hk) << p.pool.page_log2;
            float k_factor = 1.f;
            if (kE4M3) k_factor = exponent_factor(p.pool.k_exp[row]), v_factor = exponent_factor(p.pool.v_exp[row]);
            score = 0.f;
            for (int c = 0; c < HD; ++c) score = fmaf(s_q[warp][c], cached_value<HD, kE4M3>(p.pool.k, row, c, k_factor), score);
            score *= p.scale_log2;
        }
        float top = score;
        for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
        top = fmaxf(fmaxf(top, m), -3.0e38f);
        const float w = exp2f(score - top), alpha = exp2f(m - top);
        m = top;
        l = l * alpha + w;
        for (int c = 0; c < kCols; ++c) acc[c] *= alpha;
        for (int i = 0; i < 32; ++i) {
            const float wi = __shfl_sync(0xffffffffu, w, i), fi = __shfl_sync(0xffffffffu, v_factor, i);
            const long long ri = __shfl_sync(0xffffffffu, row, i);
            if (ri < 0) continue;
            for (int c = 0; c < kCols; ++c) acc[c] = fmaf(wi, cached_value<HD, kE4M3>(p.pool.v, ri, c * 32 + lane, fi), acc[c]);
        }
    }
    for (int off = 16; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    for (int c = 0; c < kCols; ++c) p.o[(static_cast<long long>(t) * p.H + h) * HD + c * 32 + lane] = __float2bfloat16(acc[c] / l);
    if (lane == 0) p.lse[static_cast<long long>(h) * p.batch.T + t] = (m + log2f(l)) * 0.6931471805599453f;
}

}  // namespace

cudaError_t launch_paged_fwd(const PagedFwdParams& p, bool e4m3, int d, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>((static_cast<long long>(p.batch.T) * p.H + 3) / 4);
    auto kernel = d == 64 ? (e4m3 ? s2a_paged_fwd_kernel<64, true> : s2a_paged_fwd_kernel<64, false>)
                          : (e4m3 ? s2a_paged_fwd_kernel<128, true> : s2a_paged_fwd_kernel<128, false>);
    return launch_kernel(kernel, grid, 128, 0, stream, p, true);
}

}  // namespace s2a
