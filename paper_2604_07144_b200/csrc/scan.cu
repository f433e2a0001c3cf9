// Selective state space scan over an iteration's packed rows, with every sequence's state kept in a slot.
//
//   d = softplus(dt[t][c] + dt_bias[c]),  h[c][n] <- e^(d a[c][n]) h[c][n] + d x[t][c] b[t][n],
//   y = sum_n c[t][n] h[c][n] + d_skip[c] x[t][c],  out = y z / (1 + e^-z)
//
// A sequence's tokens follow one another, channels and states are independent.  A prompt costs an exponential per
// (token, channel, state): at 16 states the special-function unit (16 a clock and SM) bounds it, ahead of HBM.  A single
// token costs its state, read and written: HBM.
//
// Work split.  A quad of lanes takes kCh channels (four at 16 states); a lane holds N / 4 states of each of them.  Against
// a lane per channel this halves what the lanes read from shared memory per update (b and c serve four channels, d and
// d x four lanes) and leaves every lane with one channel's sum, by exchanging partial sums inside the quad.
#include "layers.h"
#include "ptx.cuh"

namespace ap {

namespace {

using namespace ptx;

constexpr int kScanWarps = 4, kScanThreads = 32 * kScanWarps;

template <int N>
struct Scan {
    static constexpr int kHeld = N / 4;                        // states a lane holds of a channel
    static constexpr int kCh = kHeld <= 4 ? 4 : 16 / kHeld;    // channels of a quad: 16 states a lane at most
    static constexpr int kBlockCh = kScanWarps * 8 * kCh;
    static constexpr int kVec = kHeld < 4 ? kHeld : 4;         // states that lie together: lane q has 4 kVec i + kVec q + e
    static constexpr int kVecs = kHeld / kVec;
    static constexpr int kGroups = kBlockCh / 8;               // 16-byte groups of a row's channels
    static constexpr int kRowsAtOnce = kScanThreads / kGroups; // rows that the block stages at once
    static constexpr int kPasses = kScanTile / kRowsAtOnce;
};

__device__ __forceinline__ float2 widen2(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// ln(1 + e^x) = max(x, 0) + log1p(e^-|x|); log1p(u) / u on [0, 1] by a polynomial fitted for relative error (4.7e-9,
// 1.4e-7 with the roundings).
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

__device__ __forceinline__ float gate(float y, float z) { return y * __fdividef(z, 1.f + exp2_approx(-1.4426950408889634f * z)); }

// kHeld consecutive-by-vector fp32 values of a lane: states 4 kVec i + kVec q + e
template <int N>
__device__ __forceinline__ void load_states(const float *row, int q, float (&h)[Scan<N>::kHeld]) {
    using S = Scan<N>;
#pragma unroll
    for (int i = 0; i < S::kVecs; ++i) {
        const float *p = row + 4 * S::kVec * i + S::kVec * q;
        if constexpr (S::kVec == 4) {
            const uint4 v = load16(p);
            h[4 * i] = __uint_as_float(v.x), h[4 * i + 1] = __uint_as_float(v.y);
            h[4 * i + 2] = __uint_as_float(v.z), h[4 * i + 3] = __uint_as_float(v.w);
        } else {
            const uint2 v = load8(p);
            h[0] = __uint_as_float(v.x), h[1] = __uint_as_float(v.y);
        }
    }
}

template <int N>
__device__ __forceinline__ void store_states(float *row, int q, const float (&h)[Scan<N>::kHeld]) {
    using S = Scan<N>;
#pragma unroll
    for (int i = 0; i < S::kVecs; ++i) {
        float *p = row + 4 * S::kVec * i + S::kVec * q;
        if constexpr (S::kVec == 4) *(float4 *)p = make_float4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
        else *(float2 *)p = make_float2(h[0], h[1]);
    }
}

// Sums a quad's partial sums: lane q ends with the sum of channel q * kCh / 4.
template <int kCh>
__device__ __forceinline__ float quad_sum(const float (&y)[kCh], int q) {
    if constexpr (kCh == 4) {
        // lanes 0, 1 keep channels 0, 1 and give away 2, 3; then each keeps one
        const bool high = q & 2, odd = q & 1;
        float a = high ? y[2] : y[0], b = high ? y[3] : y[1];
        a += __shfl_xor_sync(0xffffffffu, high ? y[0] : y[2], 2);
        b += __shfl_xor_sync(0xffffffffu, high ? y[1] : y[3], 2);
        return (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 1);
    } else if constexpr (kCh == 2) {
        const bool high = q & 2;
        const float a = (high ? y[1] : y[0]) + __shfl_xor_sync(0xffffffffu, high ? y[0] : y[1], 2);
        return a + __shfl_xor_sync(0xffffffffu, a, 1);
    } else {
        const float a = y[0] + __shfl_xor_sync(0xffffffffu, y[0], 2);
        return a + __shfl_xor_sync(0xffffffffu, a, 1);
    }
}

template <int N>
struct ScanSmem {
    float d[kScanTile][Scan<N>::kBlockCh];       // steps
    float dx[kScanTile][Scan<N>::kBlockCh];      // step times input
    float y[kScanTile][Scan<N>::kBlockCh];       // d_skip x, then the row's result before the gate
    float b[kScanTile][N], c[kScanTile][N];
};

// One piece of a sequence for kBlockCh channels.  Rows are staged kScanTile at a time: x and dt (16-byte groups of
// channels, all threads) become d, d x and d_skip x in shared memory; the quads walk the rows; the gate is applied on the
// way out.  The next tile's loads are in flight while the rows of this one are walked.
template <int N, bool kStateOnly>
__device__ __forceinline__ void scan_unit(const StateUnit &unit, int cb, const ScanArgs &g, ScanSmem<N> &sm) {
    using S = Scan<N>;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3;
    const int64_t D = g.channels;
    // staging: this thread's group of channels and first row
    const int grp = tid % S::kGroups, row_in = tid / S::kGroups;
    const int64_t sc = (int64_t)cb * S::kBlockCh + grp * 8;
    const bool s_in = sc < D;                                  // (channels come in eights)
    float bias[8] = {}, skip[8] = {};
    if (s_in && g.dt_bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) bias[i] = __uint_as_float(load4(g.dt_bias + sc + i));
    }
    if (!kStateOnly && s_in && g.d_skip) {
#pragma unroll
        for (int i = 0; i < 8; ++i) skip[i] = __uint_as_float(load4(g.d_skip + sc + i));
    }
    // walking: this lane's channels and states
    const int lc = warp * 8 * S::kCh + (lane >> 2) * S::kCh;   // the quad's first channel in the block
    const int64_t wc = (int64_t)cb * S::kBlockCh + lc;
    float h[S::kCh][S::kHeld], a2[S::kCh][S::kHeld], total[S::kCh];
#pragma unroll
    for (int c = 0; c < S::kCh; ++c) {
        total[c] = 0.f;
#pragma unroll
        for (int i = 0; i < S::kHeld; ++i) h[c][i] = a2[c][i] = 0.f;
        if (wc + c >= D) continue;
        load_states<N>(g.a + (wc + c) * N, q, a2[c]);
#pragma unroll
        for (int i = 0; i < S::kHeld; ++i) a2[c][i] *= 1.4426950408889634f;
        if (unit.seg > 0 && !kStateOnly) {
            // the state behind the pieces before this one: each piece's own, and what is left of the state before it
            load_states<N>(g.seg_state + ((int64_t)unit.seg_first * D + wc + c) * N, q, h[c]);
            for (int s = 1; s < unit.seg; ++s) {
                const int64_t at = (int64_t)(unit.seg_first + s) * D + wc + c;
                const float step = __uint_as_float(load4(g.seg_dt + at));
                float own[S::kHeld];
                load_states<N>(g.seg_state + at * N, q, own);
#pragma unroll
                for (int i = 0; i < S::kHeld; ++i) h[c][i] = fmaf(exp2_approx(step * a2[c][i]), h[c][i], own[i]);
            }
        } else if ((unit.flags & kUnitFirst) && (unit.flags & kUnitKept)) {
            load_states<N>(g.state + ((int64_t)unit.slot * D + wc + c) * N, q, h[c]);
        }
    }

    uint4 xr[S::kPasses], tr[S::kPasses], zr[S::kPasses];
    constexpr int kBcGroups = N / 8;                           // 16-byte groups of a row of b (of c)
    constexpr int kBcLoads = (kScanTile * kBcGroups + kScanThreads - 1) / kScanThreads;
    uint4 br[kBcLoads], cr[kBcLoads];
    auto load_tile = [&](int t0) {
#pragma unroll
        for (int p = 0; p < S::kPasses; ++p) {
            const int t = t0 + p * S::kRowsAtOnce + row_in;
            xr[p] = tr[p] = make_uint4(0, 0, 0, 0);
            if (s_in && t < unit.rows) {
                xr[p] = load16(g.x + (unit.row0 + (int64_t)t) * g.xs + sc);
                tr[p] = load16(g.dt + (unit.row0 + (int64_t)t) * g.dts + sc);
            }
        }
#pragma unroll
        for (int p = 0; p < kBcLoads; ++p) {
            const int i = p * kScanThreads + tid, t = t0 + i / kBcGroups;
            br[p] = cr[p] = make_uint4(0, 0, 0, 0);
            if (i < kScanTile * kBcGroups && t < unit.rows) {
                br[p] = load16(g.b + (unit.row0 + (int64_t)t) * g.bs + i % kBcGroups * 8);
                if (!kStateOnly) cr[p] = load16(g.c + (unit.row0 + (int64_t)t) * g.cs + i % kBcGroups * 8);
            }
        }
    };
    load_tile(0);
    for (int t0 = 0; t0 < unit.rows; t0 += kScanTile) {
        const int rows = min(kScanTile, unit.rows - t0);
#pragma unroll
        for (int p = 0; p < S::kPasses; ++p) {
            const int r = p * S::kRowsAtOnce + row_in;
            const uint32_t xw[4] = {xr[p].x, xr[p].y, xr[p].z, xr[p].w}, tw[4] = {tr[p].x, tr[p].y, tr[p].z, tr[p].w};
            float *d = &sm.d[r][grp * 8], *dx = &sm.dx[r][grp * 8], *y = &sm.y[r][grp * 8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 x = widen2(xw[i]);
                float2 s = widen2(tw[i]);
                s.x += bias[2 * i], s.y += bias[2 * i + 1];
                if (g.softplus) s.x = softplus(s.x), s.y = softplus(s.y);
                *(float2 *)(d + 2 * i) = s;
                *(float2 *)(dx + 2 * i) = make_float2(s.x * x.x, s.y * x.y);
                if (!kStateOnly) *(float2 *)(y + 2 * i) = make_float2(skip[2 * i] * x.x, skip[2 * i + 1] * x.y);
            }
        }
#pragma unroll
        for (int p = 0; p < kBcLoads; ++p) {
            const int i = p * kScanThreads + tid;
            if (i < kScanTile * kBcGroups) {
                float *bd = &sm.b[i / kBcGroups][i % kBcGroups * 8], *cd = &sm.c[i / kBcGroups][i % kBcGroups * 8];
                const uint32_t bw[4] = {br[p].x, br[p].y, br[p].z, br[p].w}, cw[4] = {cr[p].x, cr[p].y, cr[p].z, cr[p].w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    *(float2 *)(bd + 2 * k) = widen2(bw[k]);
                    if (!kStateOnly) *(float2 *)(cd + 2 * k) = widen2(cw[k]);
                }
            }
        }
        __syncthreads();
        if (t0 + kScanTile < unit.rows) load_tile(t0 + kScanTile);
        if (!kStateOnly && g.z) {
#pragma unroll
            for (int p = 0; p < S::kPasses; ++p) {
                const int t = t0 + p * S::kRowsAtOnce + row_in;
                zr[p] = make_uint4(0, 0, 0, 0);
                if (s_in && t < unit.rows) zr[p] = load16(g.z + (unit.row0 + (int64_t)t) * g.zs + sc);
            }
        }
#pragma unroll 2
        for (int r = 0; r < rows; ++r) {
            float d[S::kCh], dx[S::kCh], b[S::kHeld], cc[S::kHeld];
            if constexpr (S::kCh == 4) {
                const float4 u = *(const float4 *)&sm.d[r][lc], v = *(const float4 *)&sm.dx[r][lc];
                d[0] = u.x, d[1] = u.y, d[2] = u.z, d[3] = u.w;
                dx[0] = v.x, dx[1] = v.y, dx[2] = v.z, dx[3] = v.w;
            } else {
#pragma unroll
                for (int c = 0; c < S::kCh; ++c) d[c] = sm.d[r][lc + c], dx[c] = sm.dx[r][lc + c];
            }
#pragma unroll
            for (int i = 0; i < S::kVecs; ++i) {
#pragma unroll
                for (int e = 0; e < S::kVec; ++e) {
                    b[i * S::kVec + e] = sm.b[r][4 * S::kVec * i + S::kVec * q + e];
                    if (!kStateOnly) cc[i * S::kVec + e] = sm.c[r][4 * S::kVec * i + S::kVec * q + e];
                }
            }
            float y[S::kCh];
#pragma unroll
            for (int c = 0; c < S::kCh; ++c) {
                float2 sum = make_float2(0.f, 0.f);
                const float2 d2 = make_float2(d[c], d[c]), dx2 = make_float2(dx[c], dx[c]);
#pragma unroll
                for (int i = 0; i < S::kHeld; i += 2) {
                    float2 e = __fmul2_rn(d2, make_float2(a2[c][i], a2[c][i + 1]));
                    e.x = exp2_approx(e.x);
                    e.y = exp2_approx(e.y);
                    const float2 in = __fmul2_rn(dx2, make_float2(b[i], b[i + 1]));
                    const float2 hn = __ffma2_rn(e, make_float2(h[c][i], h[c][i + 1]), in);
                    h[c][i] = hn.x, h[c][i + 1] = hn.y;
                    if (!kStateOnly) sum = __ffma2_rn(hn, make_float2(cc[i], cc[i + 1]), sum);
                }
                y[c] = sum.x + sum.y;
                if (kStateOnly) total[c] += d[c];
            }
            if constexpr (!kStateOnly) {
                const float mine = quad_sum<S::kCh>(y, q);
                if (S::kCh == 4 || q % (4 / S::kCh) == 0) sm.y[r][lc + q * S::kCh / 4] += mine;
            }
        }
        __syncthreads();
        if constexpr (!kStateOnly) {
#pragma unroll
            for (int p = 0; p < S::kPasses; ++p) {
                const int r = p * S::kRowsAtOnce + row_in;
                if (!s_in || r >= rows) continue;
                const float *y = &sm.y[r][grp * 8];
                const uint32_t zw[4] = {zr[p].x, zr[p].y, zr[p].z, zr[p].w};
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float2 v = *(const float2 *)(y + 2 * i);
                    if (g.z) {
                        const float2 z = widen2(zw[i]);
                        v = make_float2(gate(v.x, z.x), gate(v.y, z.y));
                    }
                    o[i] = pack_bf16x2(v.x, v.y);
                }
                *(uint4 *)(g.out + (unit.row0 + (int64_t)(t0 + r)) * g.os + sc) = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
    }
    // the state behind the rows: the sequence's, or what the pieces after this one begin with
#pragma unroll
    for (int c = 0; c < S::kCh; ++c) {
        if (wc + c >= D) continue;
        if (unit.flags & kUnitLast) {
            store_states<N>(g.state + ((int64_t)unit.slot * D + wc + c) * N, q, h[c]);
        } else if (kStateOnly || unit.seg == 0) {
            const int64_t at = (int64_t)(unit.seg_first + unit.seg) * D + wc + c;
            store_states<N>(g.seg_state + at * N, q, h[c]);
            if (kStateOnly && q == 0) g.seg_dt[at] = total[c];
        }
    }
}

template <int N>
__global__ void __launch_bounds__(kScanThreads)
scan_kernel(const StateUnit *__restrict__ units, int blocks_c, const ScanArgs g) {
    extern __shared__ __align__(16) uint8_t raw[];
    ScanSmem<N> &sm = *(ScanSmem<N> *)raw;
    const int u = (int)blockIdx.x / blocks_c, cb = (int)blockIdx.x % blocks_c;
    const StateUnit unit = units[u];
    griddep_launch_dependents();
    griddep_wait();
    if (unit.flags & kUnitStateOnly) scan_unit<N, true>(unit, cb, g, sm);
    else scan_unit<N, false>(unit, cb, g, sm);
}

// Sequences with one new token: everything in registers, lane q of a quad works out channel q * kCh / 4's step and result.
template <int N>
__global__ void __launch_bounds__(kScanThreads)
scan_step_kernel(const StateUnit *__restrict__ units, int blocks_c, const ScanArgs g) {
    using S = Scan<N>;
    const int u = (int)blockIdx.x / blocks_c, cb = (int)blockIdx.x % blocks_c;
    const int lane = threadIdx.x & 31, q = lane & 3;
    const StateUnit unit = units[u];
    const int64_t D = g.channels, row = unit.row0;
    const int64_t wc = (int64_t)cb * S::kBlockCh + (threadIdx.x >> 5) * 8 * S::kCh + (lane >> 2) * S::kCh;
    griddep_launch_dependents();
    griddep_wait();
    float *state = g.state + ((int64_t)unit.slot * D + wc) * N;
    float h[S::kCh][S::kHeld] = {};
    if (unit.flags & kUnitKept) {
#pragma unroll
        for (int c = 0; c < S::kCh; ++c)
            if (wc + c < D) load_states<N>(state + c * N, q, h[c]);
    }
    const int64_t own = wc + q * S::kCh / 4;               // this lane's channel
    const bool in = own < D;
    auto number = [&](const uint16_t *p, int64_t at) { return __uint_as_float((uint32_t)*(const volatile uint16_t *)(p + at) << 16); };
    const float x = in ? number(g.x, row * g.xs + own) : 0.f;
    float d = in ? number(g.dt, row * g.dts + own) : 0.f;
    if (in && g.dt_bias) d += __uint_as_float(load4(g.dt_bias + own));
    if (g.softplus) d = softplus(d);
    float b[S::kHeld], cc[S::kHeld];
#pragma unroll
    for (int i = 0; i < S::kVecs; ++i)
#pragma unroll
        for (int e = 0; e < S::kVec; e += 2) {
            const int n = 4 * S::kVec * i + S::kVec * q + e;
            const float2 bv = widen2(load4(g.b + row * g.bs + n)), cv = widen2(load4(g.c + row * g.cs + n));
            b[i * S::kVec + e] = bv.x, b[i * S::kVec + e + 1] = bv.y;
            cc[i * S::kVec + e] = cv.x, cc[i * S::kVec + e + 1] = cv.y;
        }
    float y[S::kCh];
#pragma unroll
    for (int c = 0; c < S::kCh; ++c) {
        const int from = (lane & ~3) | (c * (4 / S::kCh));
        const float dc = __shfl_sync(0xffffffffu, d, from), dxc = dc * __shfl_sync(0xffffffffu, x, from);
        y[c] = 0.f;
        if (wc + c >= D) continue;
        float a[S::kHeld];
        load_states<N>(g.a + (wc + c) * N, q, a);
#pragma unroll
        for (int i = 0; i < S::kHeld; ++i) {
            h[c][i] = fmaf(exp2_approx(dc * (1.4426950408889634f * a[i])), h[c][i], dxc * b[i]);
            y[c] = fmaf(cc[i], h[c][i], y[c]);
        }
        store_states<N>(state + c * N, q, h[c]);
    }
    float sum = quad_sum<S::kCh>(y, q);
    if (in && (S::kCh == 4 || q % (4 / S::kCh) == 0)) {
        if (g.d_skip) sum = fmaf(__uint_as_float(load4(g.d_skip + own)), x, sum);
        if (g.z) sum = gate(sum, number(g.z, row * g.zs + own));
        *(__nv_bfloat16 *)(g.out + row * g.os + own) = __float2bfloat16_rn(sum);
    }
}

template <int N>
cudaError_t launch_scan_t(const ap_state_pool *pool, const ap_state_plan *plan, const ScanArgs &args, cudaStream_t stream) {
    static bool configured[64] = {};
    const int dev = pool->desc.device & 63;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(scan_kernel<N>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)sizeof(ScanSmem<N>));
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const int blocks_c = (pool->desc.channels + Scan<N>::kBlockCh - 1) / Scan<N>::kBlockCh;
    cudaError_t e = cudaSuccess;
    if (plan->n_first > 0)
        e = launch_overlapped(scan_kernel<N>, (unsigned)(plan->n_first * blocks_c), (unsigned)kScanThreads, sizeof(ScanSmem<N>),
                              stream, plan->d_first, blocks_c, args);
    if (e == cudaSuccess && plan->n_second > 0)
        e = launch_overlapped(scan_kernel<N>, (unsigned)(plan->n_second * blocks_c), (unsigned)kScanThreads, sizeof(ScanSmem<N>),
                              stream, plan->d_second, blocks_c, args);
    if (e == cudaSuccess && plan->n_single > 0)
        e = launch_overlapped(scan_step_kernel<N>, (unsigned)(plan->n_single * blocks_c), (unsigned)kScanThreads, 0, stream,
                              plan->d_single, blocks_c, args);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

int scan_block_channels(int state_dim) {
    return state_dim == 64 ? Scan<64>::kBlockCh : state_dim == 32 ? Scan<32>::kBlockCh : Scan<16>::kBlockCh;
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
