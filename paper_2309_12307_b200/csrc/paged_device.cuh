// Device code shared by the kernels of the paged cache.
#pragma once

#include "paged.h"
#include "sm100_ptx.cuh"

namespace s2a {

// Notes a value out of range in the device status word and its host-visible mirror (the first code stays).
__device__ __forceinline__ void report_bad_index(int* status, int* host_status, int code) {
    if (atomicCAS(status, 0, code) == 0) {
        *reinterpret_cast<volatile int*>(host_status) = code;
        __threadfence_system();
    }
}

// By one block of a launch: every sequence of the batch is looked at, also those that no block works on.
__device__ __forceinline__ void check_batch(const PagedBatch& batch, int page_log2, int most_new, int* status, int* host_status) {
    for (int b = threadIdx.x; b < batch.B; b += blockDim.x) {
        Sequence s;
        if (const int bad = sequence_of(batch, page_log2, most_new, b, &s)) report_bad_index(status, host_status, bad);
    }
}

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 2^e, -127 (which stands for less than that) <= e <= 127
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(127 + e) << 23); }

// Of a row that kLanes neighbouring lanes have (16 bf16 values each, pairs in w): the power of two it is cached with, kExpNotFinite for one with an
// infinity or a NaN, and the codes of the lane's values (of such a row zeros).  By a whole warp.
template <int kLanes>
__device__ __forceinline__ int row_to_e4m3(const uint32_t (&w)[8], uint32_t (&codes)[4]) {
    uint32_t pair = 0;  // the largest magnitudes of either half (a NaN stays one)
#pragma unroll
    for (int c = 0; c < 8; ++c) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(pair) : "r"(w[c] & 0x7fff7fffu));
    uint32_t most = max(pair & 0xffffu, pair >> 16);
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, off));
    const int exp = row_exponent(most);
#pragma unroll
    for (int c = 0; c < 4; ++c) codes[c] = 0;
    if (exp == kExpNotFinite) return exp;
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
    return exp;
}

// Copies of 16 bytes from global to shared memory, in groups; a thread waits for its own (all but the last kLeft groups).
__device__ __forceinline__ void copy_async(void* to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(there ? 16 : 0) : "memory");  // (zeros where it is not there)
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

constexpr float kLeast = -3.0e38f;  // a running maximum before the first key: finite, so that differences are numbers

}  // namespace s2a
