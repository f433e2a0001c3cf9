// Selective state space scan over an iteration's packed rows, with every sequence's state kept in a slot.
//
//   d = softplus(dt[t][c] + dt_bias[c]),  h[c][n] <- e^(d a[c][n]) h[c][n] + d x[t][c] b[t][n],
//   y = sum_n c[t][n] h[c][n] + d_skip[c] x[t][c],  out = y z / (1 + e^-z)
//
// A sequence's tokens follow one another, channels and states are independent.  A prompt costs an exponential per
// (token, channel, state): at 16 states the special-function unit (16 a clock and SM) bounds it, ahead of HBM: 8 x 1024 rows
// of 8192 channels are 1.07 G exponentials, 240 us of that unit alone, and 83 us of HBM.  Measured: 361 us (the unit 69 % busy,
// load/store wavefronts 68 %, issue slots 59 %: 115 instructions per 32 channels and row).  A single token costs its
// state, read and written: 128 sequences of 8192 channels 24.4 us, 5.9 TB/s (at 64 states 87.9, 6.2 TB/s; at 8 15.4, 4.9 TB/s, where
// what a channel costs beside its states counts).
//
// Work split of prompts.  H states of a channel are a lane's, L = N / H lanes make a channel, and a warp walks 32 / L channels
// alone: no barrier but its own.  Rows come in tiles of 16 by asynchronous copies, a tile ahead.  Steps and gates are worked
// out by tile, two channels a lane on packed fp32, so that no lane of a channel repeats another's; what all channels share, b
// and c, stands in shared memory in fp32.  The lanes of a channel exchange halves of their rows' partial sums until each has
// whole ones.
#include <type_traits>

#include "layers.h"
#include "ptx.cuh"

namespace ap {

namespace {

using namespace ptx;

// Single tokens: a block takes a second sequence once there are kStepBlocks blocks an SM: a's share of what is read halves
// (128 sequences: 24.4 us, with one 25.0, with four 24.2; 64 tokens beside 512 rows 58.5, with one 61.0, with four 59.4).
constexpr int kStepBlocks = 6, kStepRows = 2;

// Single tokens: kLanes lanes have a channel's states, kVec next to one another each, so that a load of a warp is one run of
// memory, kAcross channels; a lane has kCh channels.
template <int N>
struct Step {
    static constexpr int kLanes = N < 16 ? 4 : N / 4, kVec = N / kLanes;
    static constexpr int kAcross = 32 / kLanes, kCh = 4;
    static constexpr int kThreads = 128;
    static constexpr int kWarpCh = kAcross * kCh, kBlockCh = kThreads / 32 * kWarpCh;
};

// Prompts: a lane has H states of one channel.
constexpr int kTile = 16;                                      // rows staged at a time
constexpr int kGroup = 8;                                      // rows walked in one piece of code (four: 369 us for 361, sixteen 373)
template <int N, int H>
struct Walk {
    static constexpr int kLanes = N / H;                       // lanes of a channel
    static constexpr int kCh = 32 / kLanes;                    // channels of a warp
    // A block is a warp; blocks of an SM: 16 of 128 registers.  (Two warps a block: 376 us for 361, places come free later;
    // 18 and 20 warps of fewer registers spill: 433 and 489 where 16 took 383.)
    static constexpr int kBlocks = 16;
    // staging: a lane takes two channels next to one another
    static constexpr int kTwos = kCh / 2, kRowsAtOnce = 32 / kTwos, kPasses = kTile / kRowsAtOnce;
    static_assert(H == 8 && kCh >= 4 && kTile % kRowsAtOnce == 0, "eight states a lane: a 16-byte piece of b");
};

__device__ __forceinline__ float2 widen2(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// ln(1 + e^x) = max(x, 0) + log1p(e^-|x|); log1p(u) / u on [0, 1] by a polynomial fitted for relative error (3.4e-8; 1.5e-7
// with the roundings; for x far below 0 the exponential's argument adds |x| 2^-24).
__device__ __forceinline__ float softplus(float x) {
    const float u = exp2_approx(-1.4426950408889634f * fabsf(x));
    float p = -0.0032440212f;
    p = fmaf(p, u, 0.0198514443f);
    p = fmaf(p, u, -0.0569594987f);
    p = fmaf(p, u, 0.106036514f);
    p = fmaf(p, u, -0.153055906f);
    p = fmaf(p, u, 0.196759388f);
    p = fmaf(p, u, -0.249541342f);
    p = fmaf(p, u, 0.333299637f);
    p = fmaf(p, u, -0.499999017f);
    p = fmaf(p, u, 1.f);
    return fmaf(p, u, fmaxf(x, 0.f));                          // (a NaN comes through u)
}

// The same for two values, on packed fp32.
__device__ __forceinline__ float2 softplus2(float2 x) {
    const float2 t = __fmul2_rn(make_float2(fabsf(x.x), fabsf(x.y)), make_float2(-1.4426950408889634f, -1.4426950408889634f));
    const float2 u = make_float2(exp2_approx(t.x), exp2_approx(t.y));
    auto two = [](float c) { return make_float2(c, c); };
    float2 p = __ffma2_rn(two(-0.0032440212f), u, two(0.0198514443f));
    p = __ffma2_rn(p, u, two(-0.0569594987f));
    p = __ffma2_rn(p, u, two(0.106036514f));
    p = __ffma2_rn(p, u, two(-0.153055906f));
    p = __ffma2_rn(p, u, two(0.196759388f));
    p = __ffma2_rn(p, u, two(-0.249541342f));
    p = __ffma2_rn(p, u, two(0.333299637f));
    p = __ffma2_rn(p, u, two(-0.499999017f));
    p = __ffma2_rn(p, u, two(1.f));
    return __ffma2_rn(p, u, make_float2(fmaxf(x.x, 0.f), fmaxf(x.y, 0.f)));
}

__device__ __forceinline__ float max_nan(float a, float b) {   // a NaN wins
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float min_nan(float a, float b) {
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

__device__ __forceinline__ float2 as_floats(uint2 v) { return make_float2(__uint_as_float(v.x), __uint_as_float(v.y)); }

__device__ __forceinline__ float2 gate2(float2 y, float2 z) {
    float2 e = __fmul2_rn(z, make_float2(-1.4426950408889634f, -1.4426950408889634f));
    e = __fadd2_rn(make_float2(exp2_approx(e.x), exp2_approx(e.y)), make_float2(1.f, 1.f));
    return __fmul2_rn(y, __fmul2_rn(z, make_float2(rcp_approx(e.x), rcp_approx(e.y))));
}

__device__ __forceinline__ float gate(float y, float z) { return y * (z * rcp_approx(1.f + exp2_approx(-1.4426950408889634f * z))); }

// Sums over kLanes lanes of four channels' partial sums: lane q of them ends with the sum of channel q * 4 / kLanes.
template <int kLanes>
__device__ __forceinline__ float lanes_sum(const float (&y)[4], int q) {
    // half of the lanes keep channels 0, 1 and give away 2, 3; then each half of those keeps one
    const bool high = q & kLanes / 2, odd = q & kLanes / 4;
    float a = high ? y[2] : y[0], b = high ? y[3] : y[1];
    a += __shfl_xor_sync(0xffffffffu, high ? y[0] : y[2], kLanes / 2);
    b += __shfl_xor_sync(0xffffffffu, high ? y[1] : y[3], kLanes / 2);
    a = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, kLanes / 4);
#pragma unroll
    for (int o = kLanes / 8; o > 0; o /= 2) a += __shfl_xor_sync(0xffffffffu, a, o);
    return a;
}

// 2^x for two values on the FMA pipe: n = round(x), f = x - n in [-0.5, 0.5], 2^f = 1 + f g(f) with a quartic g fitted for
// relative error (4.7e-7, near 0 8.4e-8: 2^f is off by 2.2e-7 at most, roundings included, and by less the smaller f is, where
// decays that last are multiplied thousands of times), 2^n by adding n to the exponent field.  For |x| <= kNear.
constexpr float kNear = 120.f;
__device__ __forceinline__ float2 exp2_pair(float2 x) {
    const float2 magic = make_float2(12582912.f, 12582912.f);              // 1.5 * 2^23: x + magic holds round(x) in its low bits
    const float2 t = __fadd2_rn(x, magic);
    const float2 n = __fadd2_rn(t, make_float2(-12582912.f, -12582912.f));
    const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
    float2 p = __ffma2_rn(f, make_float2(0.00133335381f, 0.00133335381f), make_float2(0.00966624543f, 0.00966624543f));
    p = __ffma2_rn(p, f, make_float2(0.0555050038f, 0.0555050038f));
    p = __ffma2_rn(p, f, make_float2(0.240223512f, 0.240223512f));
    p = __ffma2_rn(p, f, make_float2(0.693147123f, 0.693147123f));
    p = __ffma2_rn(p, f, make_float2(1.f, 1.f));
    return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)),
                       __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
}

// 2^x, to be multiplied to `state`, for |x| > kNear: by itself it may leave fp32's range where their product does not.  So the state
// takes its root at once, and the root is returned to be multiplied by again.  (The root is finite: a state of zero stays zero.)
// For a pair, whatever its x: twice the error of ex2 then.
__device__ __forceinline__ float2 exp2_far(float2 x, float2 &state) {
    const float2 half = __fmul2_rn(x, make_float2(0.5f, 0.5f));
    const float2 root = make_float2(exp2_approx(min_nan(half.x, 127.9f)), exp2_approx(min_nan(half.y, 127.9f)));
    state = __fmul2_rn(state, root);
    return root;
}
// The same for one of a pair that may be near.
__device__ __forceinline__ float exp2_far(float x, float &state) {
    const bool far = !(fabsf(x) <= kNear);
    const float e = exp2_approx(far ? min_nan(0.5f * x, 127.9f) : x);
    state *= far ? e : 1.f;
    return e;
}

// One pair of states in kPolyEvery takes the FMA pipe for its exponential (8 x 1024 rows: one in eight 361 us, none 363, in four
// 382; 8192 rows of 4096 channels, where half the walks form states alone: 314, 323, 326).
constexpr int kPolyEvery = 8;
// States that a lane holds.  With 16 a lane has a channel, and the 14 warps an SM of 8 x 1024 rows of 8192 channels do not
// hide their chains (447 us where 8 took 394); with 4 the lanes' own work doubles (498 us).
constexpr int kHeldStates = 8;

template <int N, int H>
struct WalkSmem {                                              // a warp's own
    alignas(16) uint16_t x[2][kTile][Walk<N, H>::kCh];         // (read again with the gates, while the next tile's comes in)
    alignas(16) uint16_t dt[kTile][Walk<N, H>::kCh], z[kTile][Walk<N, H>::kCh];
    alignas(16) uint16_t b_in[kTile][N], c_in[kTile][N];
    float4 b[2][kTile][N / 8], c[2][kTile][N / 8];             // [h]: states 8 i + 4 h .. + 3
    alignas(16) float2 step[kTile][Walk<N, H>::kCh];           // d and d x
    alignas(16) float y[kTile][Walk<N, H>::kCh];
    float bias[Walk<N, H>::kCh], skip[Walk<N, H>::kCh];
};

template <int kBytes>
__device__ __forceinline__ void copy_async(void *to, const void *from) {  // global to shared
    if constexpr (kBytes == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(to)), "l"(from), "n"(kBytes) : "memory");
}

// A warp's copies of the rows of one tensor, kCols numbers each, kSize numbers a copy.
template <int kCols, int kSize>
struct Copy {
    static constexpr int kChunks = kCols / kSize, kRows = 32 / kChunks;           // copies of a row, rows of a round
    static constexpr int kRounds = (kTile + kRows - 1) / kRows;
    const uint16_t *from;      // this lane's first piece of the tile's rows
    uint16_t *to;
    int64_t stride;
    int row, rows;             // this lane's first row; rows there are (0: none for this lane)
    __device__ __forceinline__ Copy(int lane, uint16_t *tile, const uint16_t *base, int64_t stride, int64_t row0, int64_t col, int64_t end, int rows)
        : stride(stride), row(lane / kChunks) {
        const int e = lane % kChunks * kSize;
        from = base + (row0 + row) * stride + col + e;
        to = tile + row * kCols + e;
        this->rows = col + e < end && row < kTile ? rows : 0;
    }
    __device__ __forceinline__ void tile(int t0, int place = 0) {         // (place: of tiles next to one another)
#pragma unroll
        for (int i = 0; i < kRounds; ++i)
            if (t0 + row + i * kRows < rows) copy_async<2 * kSize>(to + (place * kTile + i * kRows) * kCols, from + i * kRows * stride);
        from += kTile * stride;
    }
};

// One piece of a sequence for a warp's channels.
template <int N, int H, bool kStateOnly>
__device__ __forceinline__ void walk_unit(const StateUnit &unit, int64_t c0, const ScanArgs &g, WalkSmem<N, H> &sm) {
    using S = Walk<N, H>;
    constexpr int K = H / 2, L = S::kLanes;
    const int lane = threadIdx.x & 31;
    const int64_t D = g.channels;
    // walking: this lane's channel, and which of its states
    const int part = lane / S::kCh, cl = lane % S::kCh;
    const int64_t ch = c0 + cl;
    const bool in = ch < D;
    const int rows_all = unit.rows;
    const int64_t row0 = unit.row0;
    float2 h[K], a2[K];
    float widest = 0.f;                                        // largest |a log2 e| of the warp
    auto load_held = [&](const float *row, float2 (&to)[K]) {  // this lane's states of a channel's row
#pragma unroll
        for (int i = 0; i < K; i += 2) {
            const uint4 v = load16(row + part * H + 2 * i);
            to[i] = make_float2(__uint_as_float(v.x), __uint_as_float(v.y));
            to[i + 1] = make_float2(__uint_as_float(v.z), __uint_as_float(v.w));
        }
    };
#pragma unroll
    for (int k = 0; k < K; ++k) h[k] = a2[k] = make_float2(0.f, 0.f);
    if (in) {
        load_held(g.a + ch * N, a2);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            a2[k] = __fmul2_rn(a2[k], make_float2(1.4426950408889634f, 1.4426950408889634f));
            // (finite: rows past the end have steps of 0, and e^(0 a) has to be 1)
            a2[k] = make_float2(max_nan(min_nan(a2[k].x, 3e38f), -3e38f), max_nan(min_nan(a2[k].y, 3e38f), -3e38f));
            widest = max_nan(widest, max_nan(fabsf(a2[k].x), fabsf(a2[k].y)));
        }
        if (unit.seg > 0 && !kStateOnly) {
            // the state behind the pieces before this one: each piece's own, and what is left of the state before it
            load_held(g.seg_state + ((int64_t)unit.seg_first * D + ch) * N, h);
            for (int s = 1; s < unit.seg; ++s) {
                const int64_t at = (int64_t)(unit.seg_first + s) * D + ch;
                const float step = __uint_as_float(load4(g.seg_dt + at));
                float2 own[K];
                load_held(g.seg_state + at * N, own);
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    // e^(a sum d) may leave fp32's range where its product with h does not: four factors of its fourth root,
                    // each within 2^+-126 (beyond them any state but zero is past the range), so that a state of zero stays zero
                    auto root = [](float x) { return exp2_approx(max_nan(min_nan(0.25f * x, 126.f), -126.f)); };
                    const float2 r = make_float2(root(step * a2[k].x), root(step * a2[k].y));
                    h[k] = __ffma2_rn(r, __fmul2_rn(r, __fmul2_rn(r, __fmul2_rn(r, h[k]))), own[k]);
                }
            }
        } else if ((unit.flags & kUnitFirst) && (unit.flags & kUnitKept)) {
            load_held(g.state + ((int64_t)unit.slot * D + ch) * N, h);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) widest = max_nan(widest, __shfl_xor_sync(0xffffffffu, widest, o));

    // staging: this lane's two channels and first row
    const int two = lane % S::kTwos * 2, row_in = lane / S::kTwos;
    const bool s_in = c0 + two < D;                            // (channels come in eights)
    if (row_in == 0) {
        float2 bias = make_float2(0.f, 0.f), skip = bias;
        if (s_in && g.dt_bias) bias = as_floats(load8(g.dt_bias + c0 + two));
        if (!kStateOnly && s_in && g.d_skip) skip = as_floats(load8(g.d_skip + c0 + two));
        *(float2 *)&sm.bias[two] = bias, *(float2 *)&sm.skip[two] = skip;
    }
    float2 total = make_float2(0.f, 0.f);
    uint16_t *out = g.out + (row0 + row_in) * g.os + c0 + two;
    const int out_rows = s_in ? rows_all : 0;

    // Asynchronous copies of a tile's rows into shared memory, a tile a call.  Rows past the unit are left as they are, and not
    // used.
    constexpr int kAsync = S::kCh >= 8 ? 8 : S::kCh;           // channels of a copy
    Copy<S::kCh, kAsync> copy_x(lane, &sm.x[0][0][0], g.x, g.xs, row0, c0, D, rows_all);
    Copy<S::kCh, kAsync> copy_dt(lane, &sm.dt[0][0], g.dt, g.dts, row0, c0, D, rows_all);
    Copy<S::kCh, kAsync> copy_z(lane, &sm.z[0][0], g.z, g.zs, row0, c0, D, kStateOnly || !g.z ? 0 : rows_all);
    Copy<N, 8> copy_b(lane, &sm.b_in[0][0], g.b, g.bs, row0, 0, N, rows_all);
    Copy<N, 8> copy_c(lane, &sm.c_in[0][0], g.c, g.cs, row0, 0, N, kStateOnly ? 0 : rows_all);
    auto copy_in = [&](int t0) {
        copy_x.tile(t0, t0 / kTile & 1);
        copy_dt.tile(t0);
        copy_b.tile(t0);
        if (!kStateOnly) copy_c.tile(t0);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    copy_in(0);
    for (int t0 = 0; t0 < rows_all; t0 += kTile) {
        const int rows = min(kTile, rows_all - t0), place = t0 / kTile & 1;
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
        // the gates are wanted last: they come while the rows are walked
        if (!kStateOnly) copy_z.tile(t0);
        asm volatile("cp.async.commit_group;" ::: "memory");
        // b and c in fp32 (rows past the end: zeros, which their steps of 0 multiply)
#pragma unroll
        for (int i = lane; i < kTile * N / 8; i += 32) {
            const bool past = i * 8 / N >= rows;
            auto widen8 = [&](const uint16_t *from, float4 *to) {
                uint4 v = *(const uint4 *)from;
                if (past) v = make_uint4(0, 0, 0, 0);
                const float2 a = widen2(v.x), b = widen2(v.y), c = widen2(v.z), d = widen2(v.w);
                to[0] = make_float4(a.x, a.y, b.x, b.y);
                to[kTile * N / 8] = make_float4(c.x, c.y, d.x, d.y);
            };
            widen8(&sm.b_in[0][0] + i * 8, &sm.b[0][0][0] + i);
            if (!kStateOnly) widen8(&sm.c_in[0][0] + i * 8, &sm.c[0][0][0] + i);
        }
        // every row's step and step times input
        float longest = 0.f;
        {
            const float2 bias = *(const float2 *)&sm.bias[two];
#pragma unroll
            for (int p = 0; p < S::kPasses; ++p) {
                const int r = p * S::kRowsAtOnce + row_in;
                float2 d = __fadd2_rn(widen2(*(const uint32_t *)&sm.dt[r][two]), bias);
                if (g.softplus) d = softplus2(d);
                float2 dx = __fmul2_rn(d, widen2(*(const uint32_t *)&sm.x[place][r][two]));
                if (rows < kTile && r >= rows) d = dx = make_float2(0.f, 0.f);      // (past the end the state stays as it is)
                longest = max3_nan(longest, fabsf(d.x), fabsf(d.y));
                if (kStateOnly) total = __fadd2_rn(total, d);
                *(float4 *)&sm.step[r][two] = make_float4(d.x, dx.x, d.y, dx.y);
            }
        }
        // (far also where a step or an a is NaN)
        const bool far = __any_sync(0xffffffffu, !(longest * widest <= kNear));
        __syncwarp();
        copy_in(t0 + kTile);                                   // (past the end: an empty group)
        auto walk = [&](auto near) {
#pragma unroll 1
            for (int r0 = 0; r0 < rows; r0 += kGroup) {
                float y[kGroup];
#pragma unroll
                for (int r = 0; r < kGroup; ++r) {
                    const float2 step = sm.step[r0 + r][cl];
                    const float2 d2 = make_float2(step.x, step.x), dx2 = make_float2(step.y, step.y);
                    float2 b[K], c[K], sum = make_float2(0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < K; k += 2) {
                        const float4 u = sm.b[k / 2][r0 + r][part];
                        b[k] = make_float2(u.x, u.y), b[k + 1] = make_float2(u.z, u.w);
                        if (!kStateOnly) {
                            const float4 v = sm.c[k / 2][r0 + r][part];
                            c[k] = make_float2(v.x, v.y), c[k + 1] = make_float2(v.z, v.w);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < K; ++k) {
                        float2 e = __fmul2_rn(d2, a2[k]);
                        if (!decltype(near)::value) {
                            e = exp2_far(e, h[k]);
                        } else if ((r * K + k) % kPolyEvery == kPolyEvery - 1) {
                            e = exp2_pair(e);
                        } else {
                            e.x = exp2_approx(e.x);
                            e.y = exp2_approx(e.y);
                        }
                        h[k] = __ffma2_rn(e, h[k], __fmul2_rn(dx2, b[k]));
                        if (!kStateOnly) sum = k == 0 ? __fmul2_rn(h[k], c[k]) : __ffma2_rn(h[k], c[k], sum);
                    }
                    y[r] = sum.x + sum.y;
                }
                if constexpr (!kStateOnly) {
                    // the lanes of a channel exchange every other row of theirs until each has whole sums: of rows
                    // mine, mine + L, ..., so that the lanes' rows of a store lie next to one another
                    constexpr int kShare = L > kGroup ? L / kGroup : 1;       // lanes that have the same row
                    int mine = 0;
#pragma unroll
                    for (int o = L / 2, n = kGroup / 2, bit = 1; o > 0; o /= 2, n /= 2, bit *= 2) {
                        const bool high = part & o;
                        if (n > 0) {
#pragma unroll
                            for (int i = 0; i < n; ++i) {
                                const float keep = high ? y[2 * i + 1] : y[2 * i], give = high ? y[2 * i] : y[2 * i + 1];
                                y[i] = keep + __shfl_xor_sync(0xffffffffu, give, o * S::kCh);
                            }
                            mine += high ? bit : 0;
                        } else {
                            y[0] += __shfl_xor_sync(0xffffffffu, y[0], o * S::kCh);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < (kGroup > L ? kGroup / L : 1); ++i)
                        if (part % kShare == 0) sm.y[r0 + mine + i * L][cl] = y[i];
                }
            }
        };
        if (far) walk(std::false_type());
        else walk(std::true_type());
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
        if constexpr (!kStateOnly) {
            const float2 skip = *(const float2 *)&sm.skip[two];
#pragma unroll
            for (int p = 0; p < S::kPasses; ++p) {
                const int r = p * S::kRowsAtOnce + row_in;
                float2 y = __ffma2_rn(skip, widen2(*(const uint32_t *)&sm.x[place][r][two]), *(const float2 *)&sm.y[r][two]);
                if (g.z) y = gate2(y, widen2(*(const uint32_t *)&sm.z[r][two]));
                if (r < out_rows - t0) *(uint32_t *)(out + p * S::kRowsAtOnce * g.os) = pack_bf16x2(y.x, y.y);
            }
            out += kTile * g.os;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    // the state behind the rows: the sequence's, or what the pieces after this one begin with
    if (in) {
        auto store_held = [&](float *row) {
#pragma unroll
            for (int i = 0; i < K; i += 2)
                *(float4 *)(row + part * H + 2 * i) = make_float4(h[i].x, h[i].y, h[i + 1].x, h[i + 1].y);
        };
        if (unit.flags & kUnitLast)
            store_held(g.state + ((int64_t)unit.slot * D + ch) * N);
        else if (kStateOnly || unit.seg == 0)
            store_held(g.seg_state + ((int64_t)(unit.seg_first + unit.seg) * D + ch) * N);
    }
    if (kStateOnly) {
#pragma unroll
        for (int o = S::kTwos; o < 32; o *= 2) {
            total.x += __shfl_xor_sync(0xffffffffu, total.x, o);
            total.y += __shfl_xor_sync(0xffffffffu, total.y, o);
        }
        if (s_in && row_in == 0) *(float2 *)(g.seg_dt + (int64_t)(unit.seg_first + unit.seg) * D + c0 + two) = total;
    }
}

// Sequences with one new token: everything in registers.  Lane q of a channel's works out the step and the result of its channel
// number q * kCh / kLanes.  A warp takes sequences u0 .. u1 for its channels, whose a it loads once.  The states are not wanted
// again before the next iteration: stored as the first to leave the L2, they leave it to what is (26.3 -> 24.8 us).  Seven blocks
// of 72 registers an SM (eight of 64: 24.8 us too, at 64 states 95.4 for 88.8).  Exponents past kNear are looked for pair by pair
// (one vote a sequence and two forms of the code: 24.3 us, one token 2.20 for 2.14, 8 states 15.2 for 15.2, 64 states 88.3 for 87.8).
template <int N>
__device__ __forceinline__ void step_units(const StateUnit *__restrict__ units, int u0, int u1, int64_t c0, const ScanArgs &g) {
    using S = Step<N>;
    const int lane = threadIdx.x & 31, q = lane & (S::kLanes - 1);
    const int64_t D = g.channels;
    const int64_t wc = c0 + lane / S::kLanes;              // this lane's first channel, of the warp's from c0 on
    const int64_t own = wc + q * S::kCh / S::kLanes * S::kAcross;
    const bool in = own < D;
    const int64_t left = D - c0;                           // (channels come in eights: those across are there or not together)
    constexpr int P = S::kVec / 2;
    auto load_held = [&](const float *p, float2 (&to)[P]) {
        if constexpr (P == 2) {
            const uint4 v = load16(p);
            to[0] = as_floats(make_uint2(v.x, v.y)), to[1] = as_floats(make_uint2(v.z, v.w));
        } else {
            to[0] = as_floats(load8(p));
        }
    };
    float2 a2[S::kCh][P];
#pragma unroll
    for (int c = 0; c < S::kCh; ++c) {
#pragma unroll
        for (int i = 0; i < P; ++i) a2[c][i] = make_float2(0.f, 0.f);
        if (S::kAcross * c < left) load_held(g.a + (wc + S::kAcross * c) * N + q * S::kVec, a2[c]);
    }
    const float bias = in && g.dt_bias ? __uint_as_float(load4(g.dt_bias + own)) : 0.f;
    const float skip = in && g.d_skip ? __uint_as_float(load4(g.d_skip + own)) : 0.f;
    auto number = [](uint16_t v) { return __uint_as_float((uint32_t)v << 16); };
#pragma unroll 1
    for (int u = u0; u < u1; ++u) {
        const int64_t row = units[u].row0;
        float *state = g.state + ((int64_t)units[u].slot * D + wc) * N + q * S::kVec;
        const bool kept = units[u].flags & kUnitKept;
        float2 h[S::kCh][P];
#pragma unroll
        for (int c = 0; c < S::kCh; ++c) {
#pragma unroll
            for (int i = 0; i < P; ++i) h[c][i] = make_float2(0.f, 0.f);
            if (kept && S::kAcross * c < left) load_held(state + S::kAcross * c * N, h[c]);
        }
        float x = 0.f, d = 0.f, z = 0.f;
        if (in) {
            x = number(load2(g.x + row * g.xs + own));
            d = number(load2(g.dt + row * g.dts + own));
            if (g.z) z = number(load2(g.z + row * g.zs + own));
        }
        float2 b[P], cc[P];
        const uint16_t *bp = g.b + row * g.bs + S::kVec * q, *cp = g.c + row * g.cs + S::kVec * q;
        if constexpr (P == 2) {
            const uint2 bv = load8(bp), cv = load8(cp);
            b[0] = widen2(bv.x), b[1] = widen2(bv.y), cc[0] = widen2(cv.x), cc[1] = widen2(cv.y);
        } else {
            b[0] = widen2(load4(bp)), cc[0] = widen2(load4(cp));
        }
        d += bias;
        if (g.softplus) d = softplus(d);
        const float dx = d * x;
        d *= 1.4426950408889634f;
        float y[S::kCh];
#pragma unroll
        for (int c = 0; c < S::kCh; ++c) {
            const int from = (lane & -S::kLanes) | (c * S::kLanes / S::kCh);
            const float dc = __shfl_sync(0xffffffffu, d, from), dxc = __shfl_sync(0xffffffffu, dx, from);
            const float2 d2 = make_float2(dc, dc), dx2 = make_float2(dxc, dxc);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 e = __fmul2_rn(d2, a2[c][i]);
                if (!(max3_nan(0.f, fabsf(e.x), fabsf(e.y)) <= kNear)) {
                    e = make_float2(exp2_far(e.x, h[c][i].x), exp2_far(e.y, h[c][i].y));
                } else {
                    e.x = exp2_approx(e.x), e.y = exp2_approx(e.y);
                }
                h[c][i] = __ffma2_rn(e, h[c][i], __fmul2_rn(dx2, b[i]));
                sum = __ffma2_rn(h[c][i], cc[i], sum);
            }
            y[c] = sum.x + sum.y;
            if (S::kAcross * c < left) {
                float *p = state + S::kAcross * c * N;
                if constexpr (P == 2) __stcs((float4 *)p, make_float4(h[c][0].x, h[c][0].y, h[c][1].x, h[c][1].y));
                else __stcs((float2 *)p, h[c][0]);
            }
        }
        float sum = lanes_sum<S::kLanes>(y, q);
        if (in && q % (S::kLanes / S::kCh) == 0) {
            sum = fmaf(skip, x, sum);
            if (g.z) sum = gate(sum, z);
            *(__nv_bfloat16 *)(g.out + row * g.os + own) = __float2bfloat16_rn(sum);
        }
    }
}

template <int N>
__global__ void __launch_bounds__(Step<N>::kThreads, 7)
scan_step_kernel(const StateUnit *__restrict__ units, int n_units, int rows, int blocks_c, const ScanArgs g) {
    const int u0 = (int)blockIdx.x / blocks_c * rows, cb = (int)blockIdx.x % blocks_c;
    const int64_t c0 = (int64_t)cb * Step<N>::kBlockCh + (threadIdx.x >> 5) * Step<N>::kWarpCh;
    griddep_launch_dependents();
    if (c0 >= g.channels) return;
    griddep_wait();
    step_units<N>(units, u0, min(u0 + rows, n_units), c0, g);
}

// Single tokens that an iteration has beside its prompts: warps of their own behind the walks', in the same launch, so that
// their loads fill what the walks leave of HBM and their warps the places that the last walks leave (64 tokens beside 512
// rows of a prompt, 8192 channels: 58 us; as a launch of their own behind it 63, in front of the walks 62; 61 beside the ragged
// chunks at 64 states: 90, 105, 101).
struct Singles {
    const StateUnit *units;
    int n, rows, blocks_c;      // sequences; of a warp; warps for the channels
};

template <int N, int H>
__global__ void __launch_bounds__(32, Walk<N, H>::kBlocks)
scan_kernel(const StateUnit *__restrict__ units, int64_t n_warps, int blocks_c, const Singles singles, const ScanArgs g) {
    extern __shared__ __align__(16) uint8_t raw[];
    int64_t at = blockIdx.x;
    griddep_launch_dependents();
    if (at >= n_warps) {
        at -= n_warps;
        const int u0 = (int)(at / singles.blocks_c) * singles.rows;
        griddep_wait();
        step_units<N>(singles.units, u0, min(u0 + singles.rows, singles.n), at % singles.blocks_c * Step<N>::kWarpCh, g);
        return;
    }
    const StateUnit unit = units[at / blocks_c];
    const int64_t c0 = at % blocks_c * Walk<N, H>::kCh;
    WalkSmem<N, H> &sm = *(WalkSmem<N, H> *)raw;
    // Columns past the last channel, which no copy fills, are worked out with the others: whether a tile is far may not hang on
    // what another kernel left there.
    if (c0 + Walk<N, H>::kCh > g.channels) {
        auto clear = [](auto &numbers) {
            for (int i = threadIdx.x; i < (int)sizeof(numbers) / 16; i += 32) ((uint4 *)&numbers)[i] = make_uint4(0, 0, 0, 0);
        };
        clear(sm.x);
        clear(sm.dt);
        __syncwarp();
    }
    griddep_wait();
    if (unit.flags & kUnitStateOnly) walk_unit<N, H, true>(unit, c0, g, sm);
    else walk_unit<N, H, false>(unit, c0, g, sm);
}

template <int N>
cudaError_t launch_scan_t(const ap_state_pool *pool, const ap_state_plan *plan, const ScanArgs &args, cudaStream_t stream) {
    constexpr int H = kHeldStates;
    constexpr size_t kSmem = sizeof(WalkSmem<N, H>);
    static_assert(kSmem <= 48 << 10, "within what a kernel may have unasked");
    const int walk_c = (pool->desc.channels + Walk<N, H>::kCh - 1) / Walk<N, H>::kCh;
    // a's share of what is read falls with the sequences of a block; blocks enough for the GPU come first
    const int step_c = (pool->desc.channels + Step<N>::kBlockCh - 1) / Step<N>::kBlockCh;
    const int64_t spare = (int64_t)plan->n_single * step_c / ((int64_t)kStepBlocks * pool->sm_count);
    const int rows = spare < 2 ? 1 : spare > kStepRows ? kStepRows : (int)spare;
    const int groups = (plan->n_single + rows - 1) / rows;
    const Singles singles{plan->d_single, plan->n_single, rows, (pool->desc.channels + Step<N>::kWarpCh - 1) / Step<N>::kWarpCh};
    auto launch = [&](const StateUnit *units, int n, bool with) {
        const int64_t warps = (int64_t)n * walk_c;
        return launch_overlapped(scan_kernel<N, H>, (unsigned)(warps + (with ? (int64_t)groups * singles.blocks_c : 0)), 32u, kSmem, stream, units,
                                 warps, walk_c, singles, args);
    };
    cudaError_t e = cudaSuccess;
    if (plan->n_first > 0) e = launch(plan->d_first, plan->n_first, plan->n_single > 0 && plan->n_second == 0);
    if (e == cudaSuccess && plan->n_second > 0) e = launch(plan->d_second, plan->n_second, plan->n_single > 0);
    if (plan->n_first == 0 && plan->n_single > 0)
        e = launch_overlapped(scan_step_kernel<N>, (unsigned)(groups * step_c), (unsigned)Step<N>::kThreads, 0, stream, plan->d_single,
                              plan->n_single, rows, step_c, args);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int scan_warp_channels(int state_dim) {
    switch (state_dim) {
        case 8: return Walk<8, kHeldStates>::kCh;
        case 16: return Walk<16, kHeldStates>::kCh;
        case 32: return Walk<32, kHeldStates>::kCh;
        default: return Walk<64, kHeldStates>::kCh;
    }
}

cudaError_t launch_scan(const ap_state_pool *pool, const ap_state_plan *plan, const ScanArgs &args, cudaStream_t stream) {
    switch (pool->desc.state_dim) {
        case 8: return launch_scan_t<8>(pool, plan, args, stream);
        case 16: return launch_scan_t<16>(pool, plan, args, stream);
        case 32: return launch_scan_t<32>(pool, plan, args, stream);
        default: return launch_scan_t<64>(pool, plan, args, stream);
    }
}

}  // namespace ap
