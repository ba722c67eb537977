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

constexpr float kLeast = -3.0e38f;  // a running maximum before the first key: finite, so that differences are numbers

}  // namespace s2a
