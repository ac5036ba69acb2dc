// The internal streams that grouped calls fork into.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <mutex>

#include "tcgen05.cuh"

namespace od {

// ---- internal streams of the grouped step ---------------------------------------------------
// The steps of two launch batches (matrices of different plans) share nothing, so a grouped call
// may run them side by side: the caller's stream forks into up to kMaxLanes internal streams,
// every batch runs its whole stage sequence on one of them, and the caller's stream joins them
// again before the call returns.  Order on the device is fixed by events only; the host never
// waits.  The latency-bound r x r factor kernel of one batch and the ramp-up and tail of every
// persistent kernel then overlap the kernels of the other batches.  Results per matrix do not
// depend on this: every matrix goes through the same kernels with the same launch geometry.
constexpr int kMaxLanes = 8;
inline std::atomic<int> g_lanes{4};

struct DeviceLanes {
    std::mutex mu;                   // one grouped call at a time forks into the lanes of a device
    bool ready = false;
    cudaStream_t lane[kMaxLanes] = {};
    cudaEvent_t fork = nullptr, done[kMaxLanes] = {};
};

// Lanes of the current device; streams and events are created on the first call that needs them
// (no device memory is allocated).
inline DeviceLanes* device_lanes() {
    static DeviceLanes table[kMaxDevices];
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    DeviceLanes* d = &table[dev];
    std::lock_guard<std::mutex> lock(d->mu);
    if (!d->ready) {
        bool ok = cudaEventCreateWithFlags(&d->fork, cudaEventDisableTiming) == cudaSuccess;
        for (int i = 0; i < kMaxLanes && ok; ++i)
            ok = cudaStreamCreateWithFlags(&d->lane[i], cudaStreamNonBlocking) == cudaSuccess &&
                 cudaEventCreateWithFlags(&d->done[i], cudaEventDisableTiming) == cudaSuccess;
        if (!ok) return nullptr;
        d->ready = true;
    }
    return d;
}

}  // namespace od
