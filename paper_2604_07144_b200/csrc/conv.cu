// Short causal convolution over an iteration's packed rows, with the last inputs of every sequence kept in a slot.
//
//   out[t][c] = act(bias[c] + sum_j weight[c][j] x[t - W + 1 + j][c])
//
// HBM-bound: x is read and out written once.  A thread takes 4 channels (8 bytes of a row) of a unit, a run of rows of a
// sequence, and slides the window over them in registers, in fp32, kAhead rows loaded at a time; a row is loaded once per unit
// and W - 1 rows twice.  The thread of a sequence's first unit reads the slot (the inputs before the first row) and then
// writes it (the last W - 1 inputs): the same thread does both, so no block reads what another has overwritten.
// 8 x 1024 rows of 8192 channels: 49.7 us, 5.4 TB/s of 6.6 (x's rows 32 KB apart); the exponentials and reciprocals of the
// activation keep the special-function unit 65 % busy.  Eight rows ahead with registers for them (5 blocks an SM) 57.7 us, six
// 51.2; eight blocks an SM spill: 65.
#include "layers.h"
#include "ptx.cuh"

namespace ap {

namespace {

using namespace ptx;

constexpr int kAhead = 4;                                 // rows loaded together

struct Four {                                             // four channels in fp32
    float2 lo, hi;
};
__device__ __forceinline__ Four widen4(uint2 v) {
    return {make_float2(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u)),
            make_float2(__uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u))};
}
// y / (1 + e^-y)
__device__ __forceinline__ float2 silu2(float2 y) {
    float2 e = __fmul2_rn(y, make_float2(-1.4426950408889634f, -1.4426950408889634f));
    e = __fadd2_rn(make_float2(exp2_approx(e.x), exp2_approx(e.y)), make_float2(1.f, 1.f));
    return __fmul2_rn(y, make_float2(rcp_approx(e.x), rcp_approx(e.y)));
}

template <int W, bool kSilu>
__global__ void __launch_bounds__(kConvThreads, 7)
conv_kernel(const StateUnit *__restrict__ units, int blocks_c, int64_t channels, const uint16_t *x, const uint16_t *weight,
            const uint16_t *bias, uint16_t *out, uint16_t *slots, int64_t xs, int64_t os) {
    const StateUnit unit = units[(int)blockIdx.x / blocks_c];
    const int64_t c0 = ((int64_t)((int)blockIdx.x % blocks_c) * kConvThreads + threadIdx.x) * 4;
    griddep_launch_dependents();
    if (c0 >= channels) return;
    griddep_wait();
    const uint16_t *xr = x + (int64_t)unit.row0 * xs + c0;
    uint2 next[kAhead];
    const uint16_t *ahead = xr;                           // the row to load next
    auto load_rows = [&](int t0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i, ahead += xs)
            if (t0 + i < unit.rows) next[i] = load8(ahead);
    };
    load_rows(0);
    uint2 before[W - 1];                                  // the W - 1 inputs before the first row
    if (unit.flags & kUnitFirst) {
        uint16_t *slot = slots + (int64_t)unit.slot * (W - 1) * channels + c0;
        uint2 last[W - 1];                                // the last W - 1 inputs of the sequence
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            before[j] = last[j] = make_uint2(0, 0);
            const int back = W - 1 - j;                   // rows from the end
            if (unit.flags & kUnitKept) before[j] = load8(slot + j * channels);
            if (back <= unit.seq_rows) last[j] = load8(xr + (int64_t)(unit.seq_rows - back) * xs);
            else if (unit.flags & kUnitKept) last[j] = load8(slot + (j + unit.seq_rows) * channels);   // (fewer rows than the window)
        }
#pragma unroll
        for (int j = 0; j < W - 1; ++j) *(uint2 *)(slot + j * channels) = last[j];
    } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) before[j] = load8(xr + (j - (W - 1)) * xs);
    }
    Four w[W], base = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    {
        uint32_t raw[2 * W];                              // 4 channels' W weights, next to one another
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint2 v = load8(weight + c0 * W + 4 * i);
            raw[2 * i] = v.x, raw[2 * i + 1] = v.y;
        }
        auto number = [&](int c, int j) {
            const int k = c * W + j;
            return __uint_as_float(k & 1 ? raw[k >> 1] & 0xFFFF0000u : raw[k >> 1] << 16);
        };
#pragma unroll
        for (int j = 0; j < W; ++j) w[j] = {make_float2(number(0, j), number(1, j)), make_float2(number(2, j), number(3, j))};
        if (bias) base = widen4(load8(bias + c0));
    }
    Four seen[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) seen[j] = widen4(before[j]);
    uint16_t *o = out + (int64_t)unit.row0 * os + c0;
    auto row = [&](uint2 in) {
        const Four v = widen4(in);
        Four y = base;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const Four &u = j < W - 1 ? seen[j] : v;
            y.lo = __ffma2_rn(w[j].lo, u.lo, y.lo);
            y.hi = __ffma2_rn(w[j].hi, u.hi, y.hi);
        }
        if (kSilu) y.lo = silu2(y.lo), y.hi = silu2(y.hi);
        *(uint2 *)o = make_uint2(pack_bf16x2(y.lo.x, y.lo.y), pack_bf16x2(y.hi.x, y.hi.y));
        o += os;
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) seen[j] = seen[j + 1];
        seen[W - 2] = v;
    };
    int t0 = 0;
    for (; t0 + kAhead <= unit.rows; t0 += kAhead) {       // (whole groups: no test between rows, and the window moves for nothing)
        uint2 now[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) now[i] = next[i];
        load_rows(t0 + kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) row(now[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (t0 + i < unit.rows) row(next[i]);
}

template <int W>
cudaError_t launch_conv_t(const ap_state_pool *pool, const ap_state_plan *plan, const ap_conv_desc &conv, cudaStream_t stream) {
    const int blocks_c = (pool->desc.channels / 4 + kConvThreads - 1) / kConvThreads;
    const cudaError_t e = launch_overlapped(conv.silu ? conv_kernel<W, true> : conv_kernel<W, false>, (unsigned)(plan->n_conv * blocks_c),
                                            (unsigned)kConvThreads, 0, stream, plan->d_conv, blocks_c, (int64_t)pool->desc.channels,
                                            (const uint16_t *)conv.x, (const uint16_t *)conv.weight, (const uint16_t *)conv.bias, (uint16_t *)conv.out,
                                            (uint16_t *)pool->desc.conv_base, conv.x_row_stride, conv.out_row_stride);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_conv(const ap_state_pool *pool, const ap_state_plan *plan, const ap_conv_desc &conv, cudaStream_t stream) {
    switch (pool->desc.conv_width) {
        case 2: return launch_conv_t<2>(pool, plan, conv, stream);
        case 3: return launch_conv_t<3>(pool, plan, conv, stream);
        default: return launch_conv_t<4>(pool, plan, conv, stream);
    }
}

}  // namespace ap
