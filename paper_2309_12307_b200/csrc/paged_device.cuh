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

// Four 8-bit floats (e4m3) as bf16, each times 2^-120: the bits of sign, exponent and fraction are moved to where bf16
// has them, which also holds for exponent 0.  lo = values 0 and 2, hi = values 1 and 3.
__device__ __forceinline__ void e4m3_spread(uint32_t w, uint32_t& lo, uint32_t& hi) {
    lo = ((w << 8) & 0x80008000u) | ((w << 4) & 0x07f007f0u);
    hi = (w & 0x80008000u) | ((w >> 4) & 0x07f007f0u);
}
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// 2^120 * 2^e as a product of two bf16 numbers (the sum of the exponents can be too large for one), each twice in a
// word; NaN for a row that is not finite.
struct RowFactor {
    uint32_t first, second;
};
__device__ __forceinline__ RowFactor row_factor(int e) {
    const int low = e < 7 ? e : 7;
    const uint32_t a = e == kExpNotFinite ? 0x7fffu : static_cast<uint32_t>(127 + 120 + low) << 7, b = static_cast<uint32_t>(127 + e - low) << 7;
    return {a | a << 16, b | b << 16};
}
constexpr uint32_t kTwoTo120 = ((127u + 120u) << 7) * 0x10001u;

__device__ __forceinline__ float bf16_low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

}  // namespace s2a
