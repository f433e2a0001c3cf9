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

inline cudaEvent_t take_event(ap_kv_pool *pool) {
    if (!pool->spare_events.empty()) {
        cudaEvent_t e = pool->spare_events.back();
        pool->spare_events.pop_back();
        return e;
    }
    cudaEvent_t e = nullptr;
    if (cudaEventCreate(&e) != cudaSuccess) { (void)cudaGetLastError(); return nullptr; }
    return e;
}

// Brackets one kernel launch with events when profiling is on.
struct TimedScope {
    ap_kv_pool *pool;
    cudaStream_t stream;
    TimedLaunch rec{};
    bool on = false;
    TimedScope(ap_kv_pool *p, int kernel, cudaStream_t st) : pool(p), stream(st) {
        if (!p->profiling) return;
        rec.kernel = kernel;
        rec.start = take_event(p);
        rec.stop = take_event(p);
        on = rec.start && rec.stop && cudaEventRecord(rec.start, st) == cudaSuccess;
    }
    ~TimedScope() {
        if (!on) return;
        if (cudaEventRecord(rec.stop, stream) != cudaSuccess) return;
        try {
            pool->timed.push_back(rec);
        } catch (const std::bad_alloc &) {          // (this launch goes uncounted)
            (void)cudaEventDestroy(rec.start);
            (void)cudaEventDestroy(rec.stop);
        }
    }
};

}  // namespace ap
