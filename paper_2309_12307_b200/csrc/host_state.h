// What the host entry points share: the state of a device, errors, tensor maps.  Defined in api.cu.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <mutex>

namespace s2a {

struct DeviceState {
    bool ready = false;
    int* status_ptr = nullptr;        // device address of the status word
    volatile int* host_word = nullptr;  // this device's mirror, host address
    int* host_word_dev = nullptr;     // the same word as the device sees it
    int n_sm = 0;                     // multiprocessors
    cudaError_t paged_error = cudaSuccess;  // what kept the paged cache's attention kernels from being set up
    int cluster_slots[4][17] = {};    // of the paged cache's splitting kernel, see configure_paged_split()
    // s2a_fwd_bwd_host only: copy streams and the events that order them against the caller's stream
    bool host_path_ready = false;
    cudaStream_t copy_in = nullptr, copy_out = nullptr;
    cudaEvent_t ev_start = nullptr, ev_done = nullptr, ev_in_done = nullptr;
    cudaEvent_t ev_qkv = nullptr, ev_do = nullptr, ev_fwd = nullptr, ev_bwd = nullptr;  // recorded again for every chunk
    std::mutex host_path;  // held by the call that enqueues: its events must not be recorded by another one in between
};

// Notes `e` for s2a_last_cuda_error() and returns S2A_ERR_CUDA.
int cuda_fail(cudaError_t e);
// Per-device set-up (once): architecture check, kernel attributes, address of the status word.
int prepare_device(DeviceState** out);
// The same for attention over the paged cache: an error too where its kernels could not be set up.
int prepare_paged(DeviceState** out);
// S2A_OK, or what an earlier launch on the device has reported and s2a_device_status() has not read yet.
int standing_status(const DeviceState* ds);
// Tensor map of `rank` dimensions over a tensor of `type`; strides (bytes) of all dimensions but the first.
int encode_tmap(CUtensorMap* tm, CUtensorMapDataType type, CUtensorMapSwizzle swizzle, const void* base, int rank, const cuuint64_t* dims,
                const cuuint64_t* strides, const cuuint32_t* box);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace s2a
