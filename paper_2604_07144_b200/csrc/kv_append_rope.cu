// Append with the rotary position embedding applied on the way: K is rotated by its position and goes to
// its page, V goes to its page as it is, q is rotated into a buffer of its own (or in place).  One pass over
// the new tokens' q, k and v, bound by HBM: 2 Hq + 4 Hkv head rows of traffic per token.
//
// Pair i of a head (elements i and i + R/2, or 2i and 2i + 1) turns by the angle p f_i:
//     (a, b) -> (a cos - b sin, b cos + a sin).
// The angle of a far position needs more than 32 bits: p f_i / 2 pi is formed in 64 bits, whole turns are
// taken off there, and only the fraction goes to fp32 sine and cosine.  Those are computed once per token
// and shared by its heads through shared memory, ahead of the wait for the kernel before.  The rotation is fp32
// and rounds once, to bf16.
// 8192 rows at 32 / 8 heads of 128 (201 MB): 32.2 us, 6.25 TB/s, 0.95 of copy bandwidth (33.5 us, 0.92, in a loop of
// seconds); 4 rows at 8 / 2 heads of 64: 1.4 us in a graph.
#include <algorithm>

#include "internal.h"
#include "kv4.cuh"
#include "ptx.cuh"

namespace ap {

namespace {

constexpr int kPassHeads = 32;      // kv heads whose rotated K waits in shared memory for quantisation
constexpr int kAhead = 2;           // units of a thread loaded before the angles are ready
constexpr int kMaxThreads = 256;

// One block per token.  A thread's unit is 16 elements of one head row, two 16-byte chunks that turn
// together: for half-split pairs chunk u with chunk u + R/16, for neighbouring pairs chunks 2u and 2u + 1;
// either way they need the angles 8u .. 8u + 7.  Chunks past R are copied, two at a time.
template <int D, bool kFour>
__global__ void __launch_bounds__(kMaxThreads)
rope_append_kernel(const __grid_constant__ RopeParams rope, uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                   const uint4 *q, const uint4 *__restrict__ k_new, const uint4 *__restrict__ v_new, uint4 *q_rot,
                   int64_t q_stride, int64_t k_stride, int64_t v_stride, const int32_t *__restrict__ append_dst,
                   const int32_t *__restrict__ positions, int Hq, int Hkv, int num_pages, int *status) {
    using T = kv4::Tile<D>;
    constexpr int kChunks = D / 8, kUnits = D / 16;
    __shared__ float2 trig[D / 2];
    __shared__ uint4 k_rows[kFour ? kPassHeads * kChunks : 1];
    const int64_t row = blockIdx.x;
    const int32_t dst = __ldg(append_dst + row), pos = __ldg(positions + row);
    const int32_t page = dst >> 4, slot = dst & 15;
    auto first_chunk = [&](int u) { return u >= rope.units ? 2 * u : rope.interleaved ? 2 * u : u; };
    auto second_chunk = [&](int u) { return u >= rope.units || rope.interleaved ? 2 * u + 1 : u + rope.units; };
    auto rotate = [&](int u, uint4 &x, uint4 &y) {
        if (u >= rope.units) return;
        uint32_t a[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
        const float2 *cs = trig + 8 * u;
        if (rope.interleaved) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {                    // word i holds pair 8u + i
                const float2 t = cs[i];
                const float p = __uint_as_float(a[i] << 16), r = __uint_as_float(a[i] & 0xFFFF0000u);
                a[i] = ptx::pack_bf16x2(p * t.x - r * t.y, r * t.x + p * t.y);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {                    // words i and 4 + i hold pairs 8u + 2i, 8u + 2i + 1
                const float2 t0 = cs[2 * i], t1 = cs[2 * i + 1];
                const float p0 = __uint_as_float(a[i] << 16), p1 = __uint_as_float(a[i] & 0xFFFF0000u);
                const float r0 = __uint_as_float(a[4 + i] << 16), r1 = __uint_as_float(a[4 + i] & 0xFFFF0000u);
                a[i] = ptx::pack_bf16x2(p0 * t0.x - r0 * t0.y, p1 * t1.x - r1 * t1.y);
                a[4 + i] = ptx::pack_bf16x2(r0 * t0.x + p0 * t0.y, r1 * t1.x + p1 * t1.y);
            }
        }
        x = make_uint4(a[0], a[1], a[2], a[3]);
        y = make_uint4(a[4], a[5], a[6], a[7]);
    };
    // q rows, then (bf16 pool) K rows and V rows: where unit `id` reads and writes
    const int n = (Hq + (kFour ? 0 : 2 * Hkv)) * kUnits;
    struct Unit { const uint4 *src; uint4 *out; int c0, c1, u; bool turns; };
    auto unit_of = [&](int id) {
        Unit w;
        w.u = id % kUnits;
        const int h = id / kUnits;
        if (h < Hq) {
            w.src = q + row * q_stride + h * kChunks;
            w.out = q_rot + (row * Hq + h) * kChunks;
        } else {
            const bool is_v = h >= Hq + Hkv;
            const int g = h - Hq - (is_v ? Hkv : 0);
            w.src = (is_v ? v_new + row * v_stride : k_new + row * k_stride) + g * kChunks;
            w.out = reinterpret_cast<uint4 *>(is_v ? v_pool : k_pool) + (((int64_t)page * Hkv + g) * kPageSize + slot) * kChunks;
        }
        w.c0 = first_chunk(w.u);
        w.c1 = second_chunk(w.u);
        w.turns = kFour || h < Hq + Hkv;
        return w;
    };
    const int step = blockDim.x;
    for (int i = threadIdx.x; i < 8 * rope.units; i += step) {
        double turns = (double)pos * rope.turn[i];
        turns -= rint(turns);
        float s, c;
        sincospif((float)(2.0 * turns), &s, &c);
        trig[i] = make_float2(c * rope.amplitude, s * rope.amplitude);
    }
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    if (page < 0 || page >= num_pages) {                     // (the whole block)
        if (threadIdx.x == 0) ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        return;
    }
    // A thread's first kAhead units are loaded ahead of the barrier that waits for the angles.  (Past L1, which
    // would keep what is read once.)
    uint4 x[kAhead], y[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int id = threadIdx.x + i * step;
        if (id < n) {
            const Unit w = unit_of(id);
            x[i] = __ldcg(w.src + w.c0);
            y[i] = __ldcg(w.src + w.c1);
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int id = threadIdx.x + i * step;
        if (id < n) {
            const Unit w = unit_of(id);
            if (w.turns) rotate(w.u, x[i], y[i]);
            w.out[w.c0] = x[i];
            w.out[w.c1] = y[i];
        }
    }
    for (int id = threadIdx.x + kAhead * step; id < n; id += step) {
        const Unit w = unit_of(id);
        uint4 a = __ldcg(w.src + w.c0), b = __ldcg(w.src + w.c1);
        if (w.turns) rotate(w.u, a, b);
        w.out[w.c0] = a;
        w.out[w.c1] = b;
    }
    if constexpr (kFour) {
        // K: rotated and rounded to bf16 in shared memory, then quantised from there, 32 heads at a time; V: quantised
        const int64_t tiles = (int64_t)page * Hkv;
        auto store = [&](uint8_t *pool, int g, int c, uint32_t w, float step) {
            uint8_t *tile = pool + (tiles + g) * T::kBytes;
            *reinterpret_cast<uint32_t *>(tile + slot * T::kRowBytes + 4 * kv4::stored_word<D>(c)) = w;
            if ((c & 3) == 0)
                *reinterpret_cast<uint16_t *>(tile + T::kCodeBytes + 2 * (slot * T::kGroups + (c >> 2))) =
                    (uint16_t)(__float_as_uint(step) >> 16);
        };
        for (int h0 = 0; h0 < Hkv; h0 += kPassHeads) {
            const int heads = min(kPassHeads, Hkv - h0);
            __syncthreads();
            for (int id = threadIdx.x; id < heads * kUnits; id += blockDim.x) {
                const int u = id % kUnits, g = id / kUnits;
                const uint4 *src = k_new + row * k_stride + (h0 + g) * kChunks;
                const int c0 = first_chunk(u), c1 = second_chunk(u);
                uint4 x = __ldcg(src + c0), y = __ldcg(src + c1);
                rotate(u, x, y);
                k_rows[g * kChunks + c0] = x;
                k_rows[g * kChunks + c1] = y;
            }
            __syncthreads();
            const int chunks = heads * kChunks;
            for (int base = 0; base < chunks; base += blockDim.x) {      // whole warps: the quantiser shuffles
                const int i = base + (int)threadIdx.x, at = min(i, chunks - 1), g = at / kChunks, c = at % kChunks;
                float ks, vs;
                const uint32_t kw = kv4::quantise8(k_rows[at], ks);
                const uint32_t vw = kv4::quantise8(__ldcg(v_new + row * v_stride + (h0 + g) * kChunks + c), vs);
                if (i < chunks) {
                    store(k_pool, h0 + g, c, kw, ks);
                    store(v_pool, h0 + g, c, vw, vs);
                }
            }
        }
    }
}

template <int D, bool kFour>
cudaError_t launch_t(const ap_kv_pool *pool, const ap_plan *plan, const RopeParams &rope, const void *q, const void *k_new,
                     const void *v_new, void *q_rot, int64_t q_stride, int64_t k_stride, int64_t v_stride, cudaStream_t stream) {
    const int Hkv = pool->desc.num_kv_heads, Hq = q ? plan->num_q_heads : 0;
    // Few rows: a thread per unit, as wide as it goes, for latency.  Many: as many passes as needed with every thread
    // busy in each, so that blocks are small and several share an SM.
    const int units = (Hq + 2 * Hkv) * (D / 16);
    const int passes = plan->info.n_new <= 2 * pool->sm_count ? (units + kMaxThreads - 1) / kMaxThreads
                                                              : std::max(kAhead, (units + kMaxThreads - 1) / kMaxThreads);
    const unsigned threads = (unsigned)(((units + passes - 1) / passes + 31) / 32 * 32);
    return launch_overlapped(rope_append_kernel<D, kFour>, (unsigned)plan->info.n_new, threads, 0, stream, rope,
                             (uint8_t *)pool->desc.k_base, (uint8_t *)pool->desc.v_base, (const uint4 *)q, (const uint4 *)k_new,
                             (const uint4 *)v_new, (uint4 *)q_rot, q_stride / 8, k_stride / 8, v_stride / 8, plan->d_append_dst,
                             plan->d_positions, Hq, Hkv, pool->desc.num_pages, pool->status_dev);
}

}  // namespace

cudaError_t launch_kv_append_rope(const ap_kv_pool *pool, const ap_plan *plan, const RopeParams &rope, const void *q,
                                  const void *k_new, const void *v_new, void *q_rot, int64_t q_stride, int64_t k_stride,
                                  int64_t v_stride, cudaStream_t stream) {
    cudaError_t e;
    if (pool->four_bit)
        e = pool->desc.head_dim == 128
                ? launch_t<128, true>(pool, plan, rope, q, k_new, v_new, q_rot, q_stride, k_stride, v_stride, stream)
                : launch_t<64, true>(pool, plan, rope, q, k_new, v_new, q_rot, q_stride, k_stride, v_stride, stream);
    else
        e = pool->desc.head_dim == 128
                ? launch_t<128, false>(pool, plan, rope, q, k_new, v_new, q_rot, q_stride, k_stride, v_stride, stream)
                : launch_t<64, false>(pool, plan, rope, q, k_new, v_new, q_rot, q_stride, k_stride, v_stride, stream);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ap
