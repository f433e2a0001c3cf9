// Host helpers that the entry points share: the current device for the length of a call, staging buffers of plan uploads.
#pragma once

#include <algorithm>
#include <new>
#include <vector>

#include "internal.h"

namespace ap {

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) { prev = -1; (void)cudaGetLastError(); }
        if (prev == dev) {                 // (already there: nothing to set, nothing to put back)
            ok = true;
            prev = -1;
            return;
        }
        ok = cudaSetDevice(dev) == cudaSuccess;
        if (!ok) (void)cudaGetLastError();
    }
    ~DeviceGuard() {
        if (prev >= 0 && ok) (void)cudaSetDevice(prev);
    }
};

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

inline void release_plan_buffer(PlanBuffer &b) {
    if (b.uploaded) (void)cudaEventDestroy(b.uploaded);
    if (b.host) (void)cudaFreeHost(b.host);
    if (b.dev) (void)cudaFree(b.dev);
    b = PlanBuffer{};
}

inline int acquire_plan_buffer(std::vector<PlanBuffer> &spare, size_t n_ints, PlanBuffer *out) {
    for (size_t i = 0; i < spare.size(); ++i) {
        if (spare[i].capacity >= n_ints) {
            *out = spare[i];
            spare.erase(spare.begin() + (long)i);
            // the previous upload from this staging area must have been consumed
            if (cudaEventSynchronize(out->uploaded) != cudaSuccess) {
                (void)cudaGetLastError();
                return AP_ERR_CUDA;
            }
            return AP_OK;
        }
    }
    PlanBuffer b;
    b.capacity = std::max<size_t>(n_ints + n_ints / 2, 4096);
    if (cudaMallocHost((void **)&b.host, b.capacity * sizeof(int32_t)) != cudaSuccess ||
        cudaMalloc((void **)&b.dev, b.capacity * sizeof(int32_t)) != cudaSuccess ||
        cudaEventCreateWithFlags(&b.uploaded, cudaEventDisableTiming) != cudaSuccess) {
        (void)cudaGetLastError();
        release_plan_buffer(b);
        return AP_ERR_CUDA;
    }
    *out = b;
    return AP_OK;
}

// Back to the pool for the next plan; freed if there is no host memory to remember it (no exception leaves a C entry).
inline void give_back_plan_buffer(std::vector<PlanBuffer> &spare, PlanBuffer &b) {
    try {
        spare.push_back(b);
    } catch (const std::bad_alloc &) {
        release_plan_buffer(b);
    }
}

}  // namespace ap
