// Short causal convolution over an iteration's packed rows, with the last inputs of every sequence kept in a slot.
//
//   out[t][c] = act(bias[c] + sum_j weight[c][j] x[t - W + 1 + j][c])
//
// HBM-bound: x is read and out written once.  A thread takes 8 channels (16 bytes of a row) of a unit of up to kConvRun
// rows and slides the window over them in registers, so a row is loaded once per unit and W - 1 rows twice.  The thread
// of a sequence's first unit reads the slot (the inputs before the first row) and then writes it (the last W - 1 inputs):
// the same thread does both, so no block reads what another has overwritten.
#include "layers.h"
#include "ptx.cuh"

namespace ap {

namespace {

using namespace ptx;

constexpr int kConvThreads = 128;

__device__ __forceinline__ void widen8(uint4 v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

template <int W>
__global__ void __launch_bounds__(kConvThreads)
conv_kernel(const StateUnit *__restrict__ units, int n_units, int groups, const uint16_t *x, const uint16_t *weight,
            const uint16_t *bias, uint16_t *out, uint16_t *slots, int64_t xs, int64_t os, int silu) {
    const int64_t at = (int64_t)blockIdx.x * kConvThreads + threadIdx.x;
    const int u = (int)(at / groups);
    const int64_t c0 = (at - (int64_t)u * groups) * 8;
    const int64_t channels = (int64_t)groups * 8;
    griddep_launch_dependents();
    if (u >= n_units) return;
    const StateUnit unit = units[u];
    griddep_wait();
    float w[W][8];
    {
        uint32_t raw[4 * W];                              // 8 channels' W weights, next to one another
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint4 v = load16(weight + c0 * W + 8 * i);
            raw[4 * i] = v.x, raw[4 * i + 1] = v.y, raw[4 * i + 2] = v.z, raw[4 * i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const int k = i * W + j;
                w[j][i] = __uint_as_float(k & 1 ? raw[k >> 1] & 0xFFFF0000u : raw[k >> 1] << 16);
            }
    }
    float base[8] = {};
    if (bias) widen8(load16(bias + c0), base);
    const uint16_t *xc = x + c0;
    uint4 seen[W - 1];                                    // the W - 1 inputs before the next row
    if (unit.flags & kUnitFirst) {
        uint16_t *slot = slots + (int64_t)unit.slot * (W - 1) * channels + c0;
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            seen[j] = (unit.flags & kUnitKept) ? load16(slot + j * channels) : make_uint4(0, 0, 0, 0);
        const int64_t end = (int64_t)unit.row0 + unit.seq_rows;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int back = W - 1 - j;                   // rows from the end
            uint4 v = make_uint4(0, 0, 0, 0);
            if (back <= unit.seq_rows) {
                v = load16(xc + (end - back) * xs);
            } else if (unit.flags & kUnitKept) {          // fewer new rows than the window: what was there moves up
                v = load16(slot + (j + unit.seq_rows) * channels);          // (a place that is written after this one)
            }
            *(uint4 *)(slot + j * channels) = v;
        }
    } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) seen[j] = load16(xc + ((int64_t)unit.row0 - (W - 1) + j) * xs);
    }
    const uint16_t *xr = xc + (int64_t)unit.row0 * xs;
    uint16_t *o = out + (int64_t)unit.row0 * os + c0;
    constexpr int kAhead = 4;                             // rows loaded together
    for (int t0 = 0; t0 < unit.rows; t0 += kAhead) {
        uint4 next[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (t0 + i < unit.rows) next[i] = load16(xr + (int64_t)(t0 + i) * xs);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (t0 + i >= unit.rows) break;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = base[e];
#pragma unroll
            for (int j = 0; j < W; ++j) {
                float v[8];
                widen8(j < W - 1 ? seen[j] : next[i], v);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(w[j][e], v[e], y[e]);
            }
            if (silu) {
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = __fdividef(y[e], 1.f + exp2_approx(-1.4426950408889634f * y[e]));
            }
            *(uint4 *)(o + (int64_t)(t0 + i) * os) = make_uint4(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]),
                                                                 pack_bf16x2(y[4], y[5]), pack_bf16x2(y[6], y[7]));
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) seen[j] = seen[j + 1];
            seen[W - 2] = next[i];
        }
    }
}

template <int W>
cudaError_t launch_conv_t(const ap_state_pool *pool, const ap_state_plan *plan, const ap_conv_desc &conv, const void *x,
                          const void *weight, const void *bias, void *out, cudaStream_t stream) {
    const int groups = pool->desc.channels / 8;
    const int64_t threads = (int64_t)plan->n_conv * groups;
    const cudaError_t e = launch_overlapped(conv_kernel<W>, (unsigned)((threads + kConvThreads - 1) / kConvThreads),
                                            (unsigned)kConvThreads, 0, stream, plan->d_conv, plan->n_conv, groups,
                                            (const uint16_t *)x, (const uint16_t *)weight, (const uint16_t *)bias,
                                            (uint16_t *)out, (uint16_t *)pool->desc.conv_base, conv.x_row_stride,
                                            conv.out_row_stride, conv.silu);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_conv(const ap_state_pool *pool, const ap_state_plan *plan, const ap_conv_desc &conv, const void *x,
                        const void *weight, const void *bias, void *out, cudaStream_t stream) {
    switch (pool->desc.conv_width) {
        case 2: return launch_conv_t<2>(pool, plan, conv, x, weight, bias, out, stream);
        case 3: return launch_conv_t<3>(pool, plan, conv, x, weight, bias, out, stream);
        default: return launch_conv_t<4>(pool, plan, conv, x, weight, bias, out, stream);
    }
}

}  // namespace ap
