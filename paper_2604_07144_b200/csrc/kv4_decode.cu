// Decode attention over a 4-bit paged cache: split-K flash-decoding like the bf16 kernel's, on the same
// kind of item lists, but built of warps that work for themselves.
//
// At 4.5 bits a value a (page, kv head) tile is 1152 bytes (d = 128): too small for one TMA request each (an
// SM's TMA unit handles ~14 M requests/s, 16 GB/s at that size; HBM gives an SM 43), and what an SM has to do
// per byte is 3.6 times the bf16 kernel's.  So every warp copies its own tiles with 16-byte cp.async into a
// private ring of kDepth pairs of pages, and no warp ever waits for another one: there is no barrier in the
// kernel.  An item is a range of a row's pages for a block of HB kv heads (8, 4, 2 or 1, the largest that
// divides the pool's); each of the plan's lists belongs to HB warps of a block, one per kv head, which read
// the HB tiles that lie together in HBM.  (With blocks of warps that share a head and fold their results at
// an item's end, barriers and uneven shares cost 20 of 49 us on 64 rows of 128 .. 8192 tokens.  One block of 16
// warps per SM, not two of eight: an SM's scheduler prefers its older block's warps, which ran through their
// lists in 145 us where the younger block's took 181.)
//
// Most of what an SM issues lies on the way from nibbles to MMA operands (LOP3, PRMT, shifts on the ALU pipe: one
// warp instruction in two clocks), so that way is short.  The bits of a byte b, put into a bf16 pattern with
// nothing above them, ARE the number b 2^-133 (bits 0 .. 6 are a subnormal's mantissa, and from bit 7, the
// exponent's last, the scale goes on linearly).  One AND therefore turns two nibbles of a word into two bf16
// numbers, c 2^-133 where they lie at bits 0 .. 3 of their halves and c 2^-129 at bits 4 .. 7; a shift by
// eight brings the other four.  Tensor cores and HFMA2 take subnormal operands exactly.
//   S^T_g = c_K (2^a Q_g)^T    per group g of 32 elements, M = 16 tokens, N = 8 query heads (mma.sync
//                              m16n8k16).  Q is scaled by a power of two per head (its largest element to
//                              2^120; elements facing nibbles at bits 4 .. 7 by 2^-4 less), which is exact;
//                              the step of (token, group) multiplies what comes out, and the codes' offset,
//                              -8 sum_g s_g sum q, is a further small MMA over the steps themselves (sum q in
//                              three bf16 parts): S = sum_g s_g (sum c q - 8 sum q);
//   softmax                    running maximum and sum in fp32, shuffles across the token lanes, once per two
//                              pages; O is rescaled only when some lane's maximum has moved;
//   O^T += V^T P^T             V is widened to bf16 in registers, exactly: c 2^-133 times 2^127 (c 2^-129 times
//                              2^123) is c / 64, and fma(c / 64, 64 s, -8 s) is (c - 8) s.
// The order of d inside a product is free, so lanes take the words of a row as they are stored: K fragments
// read 16 bytes of a row per lane, V fragments 8 bytes of four rows per lane, pairs of rows interleaved with
// PRMT.
//
// Measured: 16 rows of 32 - 64 k tokens at 64 / 8 heads of 128 (841 MB) 165 us, 5.1 TB/s, 0.78 of copy bandwidth (194 us in
// a loop of seconds, where the power limit takes the clock down); 64 rows of 128 .. 8192 tokens at 32 / 8
// heads (126 MB) 35.3 us.  Copying alone, without the arithmetic, takes 132 and 27.5 us.  331 warp
// instructions per tile (K and V of 16 tokens): 127 on the ALU pipe and 72 HFMA2, each one per two clocks of a
// scheduler, and 17 MMAs, one per eight.  No pipe is full: issue slots are 70 % busy, the ALU pipe 54 %; a warp's
// products and its widening take turns.  More warps (20 at 96 registers: 188 us) and fewer (12: 195) are slower.
//
// At the end of an item a warp has its head's complete (m, l, O) in registers and writes the bf16 output or, for
// a stream cut across lists, an fp32 partial for the merge kernel.
#include <algorithm>

#include "decode_splitk.cuh"
#include "kv4.cuh"

namespace ap {

namespace {

using namespace ptx;
using namespace kv4;

constexpr int kWarps = kKv4WarpsPerSm;   // of a full block
constexpr int kThreads = kWarps * 32;
constexpr int kDepth = 2;                // pairs of pages in a warp's ring (K and V tile of each)

template <int D>
struct Kv4Cfg {
    static constexpr int kPageBytes = 2 * Tile<D>::kBytes;        // K tile, V tile
    static constexpr int kSlotBytes = 2 * kPageBytes;
    static constexpr int kRingBytes = kDepth * kSlotBytes;        // of a warp
    static_assert(kWarps * kRingBytes <= 227 * 1024, "fits the shared memory of an SM");
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
    uint16_t v;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}

constexpr uint32_t kLow = 0x000F000Fu, kHigh = 0x00F000F0u;     // two nibbles of a word, one in each half

// D(16x8, f32) = A(16x16, bf16) B(16x8, bf16), or D += A B.  Not volatile: the compiler may interleave them.
__device__ __forceinline__ void mma_zero(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_add(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// Where 16-byte chunk `c` of a tile's codes (row * chunks per row + chunk) lies in a ring slot: chunks are
// permuted within their 128-byte line so that the rows 2t that a V fragment reads at once, which lie 256 (128)
// bytes apart, fall into different banks.
template <int D>
__device__ __forceinline__ int ring_chunk(int c) {
    const int line = c >> 3;
    return D == 128 ? c ^ (2 * (line & 3)) : c ^ (2 * (line & 1));
}

template <int D, bool kWin>
__global__ void __launch_bounds__(kThreads, 1)
kv4_decode_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool, const __nv_bfloat16 *__restrict__ q,
                  const DecodeItem *__restrict__ items, const int32_t *__restrict__ cta_begin, const int32_t *__restrict__ bt_flat,
                  float *o_part, float *lse_part, __nv_bfloat16 *__restrict__ out, float *__restrict__ lse_out, int Hq, int Hkv,
                  int G, int HB, int n_lists, int num_pages, float scale_log2, int *status, int window, int sinks) {
    using Cfg = Kv4Cfg<D>;
    using T = Tile<D>;
    constexpr int NG = T::kGroups;          // groups of a row: 4 (2)
    constexpr int NW = D / 64;              // V words of a token per lane: 2 (1)
    constexpr int kCodeChunks = T::kCodeBytes / 16, kStepChunks = (T::kBytes - T::kCodeBytes) / 16;
    constexpr int kRowChunks = T::kRowBytes / 16;
    extern __shared__ __align__(128) uint8_t smem[];

    // what is the same in all lanes passes through a broadcast, so that the compiler can keep it on the uniform
    // datapath (addresses, loop counters, branches) instead of the ALU
    auto uniform = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int g = lane >> 2, t = lane & 3;
    const int list = blockIdx.x * ((int)(blockDim.x >> 5) / HB) + warp / HB, my_head = warp % HB;
    if (list >= n_lists) {
        griddep_launch_dependents();
        griddep_wait();
        return;
    }
    const int item_begin = uniform(__ldg(cta_begin + list)), n_items = uniform(__ldg(cta_begin + list + 1)) - item_begin;
    auto get_item = [&](int n) {
        const int4 *src = reinterpret_cast<const int4 *>(items + item_begin + n);
        const int4 x = __ldg(src), y = __ldg(src + 1);
        return DecodeItem{uniform(x.x), uniform(x.y), uniform(x.z), uniform(x.w), uniform(y.x), uniform(y.y), uniform(y.z), uniform(y.w)};
    };

    // ---- the warp's stream of page pairs: a cursor that runs ahead of the consumer, across items; block-table
    // entries are loaded a pair before they are needed
    int cur_item = -1, cur_left = 0, cur_head = 0;            // cur_left: pages of the item still ahead
    const int32_t *cur_bt = bt_flat;
    int32_t next_page0 = 0, next_page1 = 0;
    int next_head = 0, next_n = 0;                            // n pages of the next pair (0: past the last)
    auto fetch = [&]() {
        while (cur_left <= 0) {
            if (++cur_item >= n_items) {
                cur_item = n_items;
                next_n = 0;
                return;
            }
            const DecodeItem it = get_item(cur_item);
            cur_left = it.page_count;
            cur_bt = bt_flat + it.bt_offset + it.page_begin;
            cur_head = it.kv_head + my_head;
        }
        next_head = cur_head;
        next_page0 = __ldg(cur_bt);
        next_n = 1;
        if (cur_left > 1) {
            next_page1 = __ldg(cur_bt + 1);
            next_n = 2;
        }
        cur_bt += 2;
        cur_left -= 2;
    };
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * Cfg::kRingBytes);
    // a lane's share of a tile's copy: code chunks lane (and lane + 32, four lines on), and, for the first
    // lanes, a chunk of K's or V's steps
    const uint32_t c_dst = 16 * ring_chunk<D>(lane);
    const uint32_t c_src = 16 * lane;
    const bool step_lane = lane < 2 * kStepChunks, k_steps = lane < kStepChunks;
    const uint32_t s_dst = (k_steps ? 0 : T::kBytes) + 16 * (kCodeChunks + lane % kStepChunks);
    const uint8_t *const s_src = (k_steps ? k_pool : v_pool) + 16 * (kCodeChunks + lane % kStepChunks);
    fetch();
    griddep_launch_dependents();
    griddep_wait();              // all of the above reads the plan only
    auto issue_page = [&](uint32_t d, int32_t page) {
        if ((uint32_t)page >= (uint32_t)num_pages) {
            record_status(status, AP_ERR_BAD_BLOCK_TABLE);
            page = 0;
        }
        const int64_t tile = (int64_t)((uint64_t)((uint32_t)page * (uint32_t)Hkv + (uint32_t)next_head) * (uint32_t)T::kBytes);
        const uint8_t *k = k_pool + tile + c_src, *v = v_pool + tile + c_src;
        cp_async16(d + c_dst, k);
        cp_async16(d + c_dst + T::kBytes, v);
        if constexpr (kCodeChunks > 32) {
            cp_async16(d + c_dst + 512, k + 512);
            cp_async16(d + c_dst + T::kBytes + 512, v + 512);
        }
        if (step_lane) cp_async16(d + s_dst, s_src + tile);
    };
    auto issue = [&](int slot) {
        const uint32_t dst = ring + (uint32_t)(slot * Cfg::kSlotBytes);
        if (next_n > 0) {
            issue_page(dst, uniform(next_page0));
            if (next_n > 1) issue_page(dst + Cfg::kPageBytes, uniform(next_page1));
            fetch();
        }
        cp_async_commit();       // (an empty group past the last pair keeps the count of groups in step)
    };
    // the first pair at once, the ring's others after the first item's queries: with all of them ahead (32 MB over the
    // GPU) the first pair's data came 2 us later
    issue(0);

    // a lane's places in a tile: K words of rows g and g + 8 (four or two lines on), K steps; V words of rows
    // 2t and 2t + 1 (and 2t + 8, 2t + 9), V steps
    const uint32_t k_off = D == 128 ? 16 * ring_chunk<D>(g * kRowChunks + t)
                                    : 16 * ring_chunk<D>(g * kRowChunks + (t >> 1)) + 8 * (t & 1);
    const uint32_t v_chunk = D == 128 ? g >> 1 : g >> 2, v_byte = D == 128 ? 8 * (g & 1) : 4 * (g & 3);
    const uint32_t v_off0 = T::kBytes + 16 * ring_chunk<D>(2 * t * kRowChunks + v_chunk) + v_byte;
    const uint32_t v_off1 = T::kBytes + 16 * ring_chunk<D>((2 * t + 1) * kRowChunks + v_chunk) + v_byte;
    constexpr uint32_t kRow8 = 8 * T::kRowBytes;           // rows r and r + 8 are permuted alike
    const uint32_t ks_off = T::kCodeBytes + 2 * NG * g;
    const uint32_t vs_off = T::kBytes + T::kCodeBytes + 2 * NG * 2 * t + (D == 128 ? 4 : 2) * (g & 1);

    int slot = 0;
    for (int n = 0; n < n_items; ++n) {
        const DecodeItem item = get_item(n);
        const int kv_head = item.kv_head + my_head;
        // ---- Q^T as the B operand, in the order in which a lane's word of K holds the elements, scaled; the
        // accumulators' start; and what turns a score into a power of two's exponent, per column (head)
        uint32_t qf[NG][4], off0 = 0, off1 = 0;
        float f_col[2];
        {
            uint4 x[NG];
            uint32_t amax = 0;
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                x[gr] = make_uint4(0, 0, 0, 0);
                if (g < G)
                    x[gr] = __ldcg(reinterpret_cast<const uint4 *>(q + ((size_t)item.q_row * Hq + (size_t)kv_head * G + g) * D + 32 * gr + 8 * t));
                const uint32_t w[4] = {x[gr].x, x[gr].y, x[gr].z, x[gr].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) amax = max(amax, max((w[i] << 16) & 0x7FFFFFFFu, w[i] & 0x7FFF0000u));
            }
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            const int a = min(max(120 + 127 - (int)(amax >> 23), 7), 126);
            const float up = __int_as_float((a + 127) << 23);                          // 2^a
            const float up_off = up * -7.3468396926392969e-40f;                        // -8 2^(a - 133) = -2^(a - 130)
            const float f = scale_log2 * __int_as_float((133 - a + 127) << 23);        // scale log2(e) 2^(133 - a)
#pragma unroll
            for (int gr = 0; gr < NG; ++gr) {
                const uint32_t w[4] = {x[gr].x, x[gr].y, x[gr].z, x[gr].w};
                // (sum q is formed of the queries as they are: 32 scaled ones of 2^123 and more would overflow it)
                float e[8], sum = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float lo = __uint_as_float(w[i] << 16), hi = __uint_as_float(w[i] & 0xFFFF0000u);
                    e[2 * i] = lo * up;
                    e[2 * i + 1] = hi * up;
                    sum += lo + hi;
                }
                qf[gr][0] = pack_bf16x2(e[0], e[4]);
                qf[gr][1] = pack_bf16x2(e[1] * 0.0625f, e[5] * 0.0625f);
                qf[gr][2] = pack_bf16x2(e[2], e[6]);
                qf[gr][3] = pack_bf16x2(e[3] * 0.0625f, e[7] * 0.0625f);
                sum += __shfl_xor_sync(0xffffffffu, sum, 1);
                sum += __shfl_xor_sync(0xffffffffu, sum, 2);
                // -8 sum q of this group in three bf16 parts (24 bits), in the units of the accumulators; element
                // gr & 1 of the B registers whose k indices the part's steps have in the offset product
                const float part0 = sum * up_off;
                const float hi = __uint_as_float(__float_as_uint(part0) & 0xFFFF0000u), rest = part0 - hi;
                const float mid = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u), lo = rest - mid;
                auto put = [&](uint32_t &reg, float v) { reg |= (pack_bf16x2(v, 0.f) & 0xFFFFu) << (16 * (gr & 1)); };
                if constexpr (D == 128) {      // k = 0 .. 3: high parts of groups 0 .. 3, 4 .. 7: middle, 8 .. 11: low
                    if (t == gr / 2) { put(off0, hi); put(off1, lo); }
                    if (t == 2 + gr / 2) put(off0, mid);
                } else {                       // k = 0, 1: high, 2, 3: middle, 4, 5: low
                    put(off0, t == 0 ? hi : t == 1 ? mid : t == 2 ? lo : 0.f);
                }
            }
            f_col[0] = __shfl_sync(0xffffffffu, f, 8 * t);
            f_col[1] = __shfl_sync(0xffffffffu, f, 8 * t + 4);
        }
        if (n == 0) {
#pragma unroll 1
            for (int i = 1; i < kDepth; ++i) issue(i);
        }
        // running maximum of the scores (f_col makes exponents of 2 of them), sum and O
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[4 * NW][4];
#pragma unroll
        for (int i = 0; i < 4 * NW; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

        const int page_end = item.page_begin + item.page_count;
#pragma unroll 1
        for (int p = item.page_begin; p < page_end; p += 2) {
            cp_async_wait<kDepth - 1>();
            __syncwarp();
            const uint32_t base = ring + (uint32_t)(slot * Cfg::kSlotBytes);
            // ---- S^T of both pages (all loads ahead of the products)
            float s[2][4];
            {
                uint32_t w[2][2][NG], st[2][2][NG / 2], so[2][2];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t tile = base + u * Cfg::kPageBytes;
                        if constexpr (D == 128) {
                            const uint4 x = lds128(tile + k_off + r * kRow8);
                            w[u][r][0] = x.x; w[u][r][1] = x.y; w[u][r][2] = x.z; w[u][r][3] = x.w;
                            const uint2 y = lds64(tile + ks_off + r * 16 * NG);
                            st[u][r][0] = y.x; st[u][r][1] = y.y;
                            so[u][r] = lds32(tile + ks_off + r * 16 * NG + 4 * (t & 1));
                        } else {
                            const uint2 x = lds64(tile + k_off + r * kRow8);
                            w[u][r][0] = x.x; w[u][r][1] = x.y;
                            so[u][r] = st[u][r][0] = lds32(tile + ks_off + r * 16 * NG);
                        }
                    }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    // sum_g s_g (-8 sum_g q): steps are bf16 numbers, a small product of its own
                    mma_zero(s[u], so[u][0], so[u][1], so[u][0], so[u][1], off0, off1);
#pragma unroll
                    for (int gr = 0; gr < NG; ++gr) {
                        const uint32_t x = w[u][0][gr], y = w[u][1][gr], x8 = x >> 8, y8 = y >> 8;
                        float acc[4];
                        mma_zero(acc, x & kLow, y & kLow, x & kHigh, y & kHigh, qf[gr][0], qf[gr][1]);
                        mma_add(acc, x8 & kLow, y8 & kLow, x8 & kHigh, y8 & kHigh, qf[gr][2], qf[gr][3]);
                        const uint32_t u0 = st[u][0][gr / 2], u1 = st[u][1][gr / 2];
                        const float s0 = __uint_as_float(gr & 1 ? u0 & 0xFFFF0000u : u0 << 16);
                        const float s1 = __uint_as_float(gr & 1 ? u1 & 0xFFFF0000u : u1 << 16);
                        s[u][0] = fmaf(acc[0], s0, s[u][0]); s[u][1] = fmaf(acc[1], s0, s[u][1]);
                        s[u][2] = fmaf(acc[2], s1, s[u][2]); s[u][3] = fmaf(acc[3], s1, s[u][3]);
                    }
                }
            }
            // ---- V words and steps, tokens 2t, 2t + 1, 2t + 8, 2t + 9; the first page's ahead of the softmax
            uint32_t vw[2][4][NW], vs[2][4];
            auto load_v = [&](int u) {
                const uint32_t tile = base + u * Cfg::kPageBytes;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const uint32_t at = tile + (r & 1 ? v_off1 : v_off0) + (r >> 1) * kRow8;
                    const uint32_t st = tile + vs_off + ((r & 1) + 8 * (r >> 1)) * 2 * NG;
                    if constexpr (D == 128) {
                        const uint2 x = lds64(at);
                        vw[u][r][0] = x.x; vw[u][r][1] = x.y;
                        vs[u][r] = lds32(st);
                    } else {
                        vw[u][r][0] = lds32(at);
                        vs[u][r] = lds16(st);
                    }
                }
            };
            load_v(0);
            // ---- hidden tokens: past the context, before the window, or of a second page that is not there;
            // whatever they hold, they weigh nothing
            const int page1 = p + 1;
            const bool some_hidden = page1 >= page_end || (page1 + 1) * kPageSize > item.kv_len ||
                                     (kWin && p * kPageSize < item.kv_len - window && (page1 + 1) * kPageSize > sinks);
            auto hidden = [&](int u, int tok) {
                const int page = p + u, key = page * kPageSize + tok;
                return page >= page_end || key >= item.kv_len || (kWin && key >= sinks && key < item.kv_len - window);
            };
            if (some_hidden) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (hidden(u, g)) s[u][0] = s[u][1] = -INFINITY;
                    if (hidden(u, g + 8)) s[u][2] = s[u][3] = -INFINITY;
                }
            }
            // ---- online softmax over the pages' tokens (the first page has a visible one)
            float mx0 = fmaxf(fmaxf(s[0][0], s[0][2]), fmaxf(s[1][0], s[1][2]));
            float mx1 = fmaxf(fmaxf(s[0][1], s[0][3]), fmaxf(s[1][1], s[1][3]));
#pragma unroll
            for (int sh = 4; sh <= 16; sh <<= 1) {
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, sh));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, sh));
            }
            if (__any_sync(0xffffffffu, mx0 > m0 || mx1 > m1)) {
                const float mn0 = fmaxf(m0, mx0), mn1 = fmaxf(m1, mx1);
                const float al0 = exp2_approx((m0 - mn0) * f_col[0]), al1 = exp2_approx((m1 - mn1) * f_col[1]);
                l0 *= al0;
                l1 *= al1;
                m0 = mn0;
                m1 = mn1;
#pragma unroll
                for (int i = 0; i < 4 * NW; ++i) {
                    o[i][0] *= al0; o[i][1] *= al1; o[i][2] *= al0; o[i][3] *= al1;
                }
            }
            // The weights go to the tensor cores in bf16, each off by at most 2^-8 of itself; their sum takes them as they
            // are.  The outputs' RMS error rises from the last rounding's 0.0017 to 0.0020 .. 0.0023; weights in two
            // parts would double the products of P V.
            const float mf0 = m0 * f_col[0], mf1 = m1 * f_col[1];
            uint32_t b0[2], b1[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float p0 = exp2_approx(s[u][0] * f_col[0] - mf0), p1 = exp2_approx(s[u][1] * f_col[1] - mf1);
                const float p2 = exp2_approx(s[u][2] * f_col[0] - mf0), p3 = exp2_approx(s[u][3] * f_col[1] - mf1);
                l0 += p0 + p2;
                l1 += p1 + p3;
                b0[u] = decode::movmatrix_trans(pack_bf16x2(p0, p1));
                b1[u] = decode::movmatrix_trans(pack_bf16x2(p2, p3));
            }
            // ---- O^T += V^T P^T
            load_v(1);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if (some_hidden) {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (hidden(u, 2 * t + (r & 1) + 8 * (r >> 1))) vs[u][r] = 0;
                }
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    const uint32_t sel = w == 0 ? 0x5410u : 0x7632u;
                    const uint32_t sa = prmt(vs[u][0], vs[u][1], sel), sb = prmt(vs[u][2], vs[u][3], sel);
                    const uint32_t sa64 = mul_bf16x2(sa, 0x42804280u), sb64 = mul_bf16x2(sb, 0x42804280u);   // 64 s
                    const uint32_t na = mul_bf16x2(sa, 0xC100C100u), nb = mul_bf16x2(sb, 0xC100C100u);       // -8 s
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t hs = half == 0 ? 0x5410u : 0x7632u;
                        const uint32_t x = prmt(vw[u][0][w], vw[u][1][w], hs), y = prmt(vw[u][2][w], vw[u][3][w], hs);
                        const uint32_t x8 = x >> 8, y8 = y >> 8;
                        auto even = [&](uint32_t v, uint32_t s64, uint32_t n) {       // nibbles at bits 0 .. 3: times 2^127
                            return fma_bf16x2(mul_bf16x2(v & kLow, 0x7F007F00u), s64, n);
                        };
                        auto odd = [&](uint32_t v, uint32_t s64, uint32_t n) {        // at bits 4 .. 7: times 2^123
                            return fma_bf16x2(mul_bf16x2(v & kHigh, 0x7D007D00u), s64, n);
                        };
                        mma_add(o[4 * w + 2 * half], even(x, sa64, na), odd(x, sa64, na), even(y, sb64, nb), odd(y, sb64, nb),
                                       b0[u], b1[u]);
                        mma_add(o[4 * w + 2 * half + 1], even(x8, sa64, na), odd(x8, sa64, na), even(y8, sb64, nb),
                                       odd(y8, sb64, nb), b0[u], b1[u]);
                    }
                }
            }
            __syncwarp();
            issue(slot);
            slot = slot + 1 == kDepth ? 0 : slot + 1;
        }

        // ---- the item's end: this lane has columns d0 .. d0 + 7 (per V word) of heads 2t and 2t + 1
#pragma unroll
        for (int sh = 4; sh <= 16; sh <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, sh);
            l1 += __shfl_xor_sync(0xffffffffu, l1, sh);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int h = 2 * t + c;
            if (h >= G) continue;
            const float l = c ? l1 : l0, inv = 1.f / l;
            const float lse = ((c ? m1 * f_col[1] : m0 * f_col[0]) + log2f(l)) * 0.6931471805599453f;
            const size_t row = item.part_slot < 0 ? (size_t)item.q_row * Hq + (size_t)kv_head * G + h
                                                  : (size_t)item.part_slot * (HB * G) + my_head * G + h;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const int d0 = D == 128 ? 32 * (2 * (g & 1) + w) + 8 * (g >> 1) : 32 * (g & 1) + 8 * (g >> 1);
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = o[4 * w + i][c] * inv;
                    v[2 * i + 1] = o[4 * w + i][2 + c] * inv;
                }
                if (item.part_slot < 0) {
                    *reinterpret_cast<uint4 *>(out + row * D + d0) = make_uint4(
                        pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
                } else {
                    *reinterpret_cast<float4 *>(o_part + row * D + d0) = make_float4(v[0], v[1], v[2], v[3]);
                    *reinterpret_cast<float4 *>(o_part + row * D + d0 + 4) = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
            if (g == 0) {
                if (item.part_slot >= 0) lse_part[row] = lse;
                else if (lse_out) lse_out[row] = lse;
            }
        }
    }
    cp_async_wait<0>();
}

// Merges the partials of a cut stream, query head by query head:
//   lse = m* + ln sum_k exp(lse_k - m*),  o = sum_k exp(lse_k - lse) o_k,  m* = max_k lse_k.
// A kernel of its own, overlapped with the decode kernel's end: with 64 query heads and ~20 partials each, the
// warp that finishes a stream would still be merging for 30 us when all others are through (192 -> 221 us on 16
// rows of 32 - 64 k tokens).  W warps share a head's partials (1 where streams have at most 8, else 4); the first eight
// rows of o that a warp needs are loaded along with the lse values, so that up to 8 W partials take one round trip.
constexpr int kMergeWarps = 4;
constexpr int kMergeBatch = 8;

template <int D, int W>
__global__ void __launch_bounds__(kMergeWarps * 32)
kv4_merge_kernel(const MergeEntry *__restrict__ merges, const float *__restrict__ o_part, const float *__restrict__ lse_part,
                 __nv_bfloat16 *__restrict__ out, float *__restrict__ lse_out, int Hq, int PH, int G, int n_heads) {
    __shared__ float4 sums[W > 1 ? kMergeWarps : 1][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, part = warp % W;
    const int head = min((int)blockIdx.x * (kMergeWarps / W) + warp / W, n_heads - 1);     // (a last block may repeat the last head)
    const MergeEntry me = merges[head / PH];
    const int ph = head % PH, n = me.part_count;
    const bool col_ok = lane * 4 < D;
    griddep_launch_dependents();
    griddep_wait();
    const float *lse = lse_part + (size_t)me.part_begin * PH + ph;
    const float4 *o = reinterpret_cast<const float4 *>(o_part + ((size_t)me.part_begin * PH + ph) * D) + lane;
    auto load = [&](int k) { return k < n && col_ok ? __ldcg(o + (size_t)k * PH * (D / 4)) : make_float4(0.f, 0.f, 0.f, 0.f); };
    float4 x[kMergeBatch];
#pragma unroll
    for (int i = 0; i < kMergeBatch; ++i) x[i] = load(part + i * W);
    const float mine = lane < n ? __ldcg(lse + (size_t)lane * PH) : -INFINITY;
    float mx = mine;
    for (int k = lane + 32; k < n; k += 32) mx = fmaxf(mx, __ldcg(lse + (size_t)k * PH));
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, sh));
    float sum = __expf(mine - mx);
    for (int k = lane + 32; k < n; k += 32) sum += __expf(__ldcg(lse + (size_t)k * PH) - mx);
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
    const float total = mx + __logf(sum);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = part; k0 < n; k0 += W * kMergeBatch) {
        if (k0 != part) {
#pragma unroll
            for (int i = 0; i < kMergeBatch; ++i) x[i] = load(k0 + i * W);
        }
#pragma unroll
        for (int i = 0; i < kMergeBatch; ++i) {
            const int k = k0 + i * W;
            if (k >= n) break;
            const float w = __expf(__ldcg(lse + (size_t)k * PH) - total);
            acc.x += w * x[i].x; acc.y += w * x[i].y; acc.z += w * x[i].z; acc.w += w * x[i].w;
        }
    }
    if constexpr (W > 1) {
        sums[warp][lane] = acc;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int i = 1; i < W; ++i) {
            const float4 y = sums[warp + i][lane];
            acc.x += y.x; acc.y += y.y; acc.z += y.z; acc.w += y.w;
        }
    }
    const size_t row = (size_t)me.q_row * Hq + (size_t)me.kv_head * G + ph;
    if (col_ok)
        *reinterpret_cast<uint2 *>(out + row * D + lane * 4) = make_uint2(pack_bf16x2(acc.x, acc.y), pack_bf16x2(acc.z, acc.w));
    if (lane == 0 && lse_out) lse_out[row] = total;
}

template <int D, int W>
cudaError_t launch_merge(const ap_plan *plan, void *out, float *lse, const float *o_part, const float *lse_part, cudaStream_t stream) {
    const int part_heads = plan->head_block * plan->group, n_heads = (int)plan->info.merge_entries * part_heads;
    constexpr int kPerBlock = kMergeWarps / W;
    return launch_overlapped(kv4_merge_kernel<D, W>, (unsigned)((n_heads + kPerBlock - 1) / kPerBlock), (unsigned)(kMergeWarps * 32), 0,
                             stream, plan->d_merge, o_part, lse_part, (__nv_bfloat16 *)out, lse, plan->num_q_heads, part_heads,
                             plan->group, n_heads);
}

template <int D, bool kWin>
cudaError_t launch_t(const ap_kv_pool *pool, const ap_plan *plan, const void *q, void *out, float *lse, float *o_part,
                     float *lse_part, cudaStream_t stream) {
    using Cfg = Kv4Cfg<D>;
    static bool configured[64] = {};
    const int dev = pool->desc.device & 63;
    if (!configured[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(kv4_decode_kernel<D, kWin>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   kWarps * Cfg::kRingBytes);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const float scale_log2 = plan->scale * 1.4426950408889634f;
    // few lists are spread over the SMs, one per block if they go round
    const int HB = plan->head_block, lists = (int)plan->info.decode_ctas;
    const int per_block = std::min(kWarps / HB, (lists + pool->sm_count - 1) / pool->sm_count);
    cudaError_t e = launch_overlapped(
        kv4_decode_kernel<D, kWin>, (unsigned)((lists + per_block - 1) / per_block), (unsigned)(per_block * HB * 32),
        (size_t)(per_block * HB * Cfg::kRingBytes),
        stream, (const uint8_t *)pool->desc.k_base, (const uint8_t *)pool->desc.v_base, (const __nv_bfloat16 *)q, plan->d_items,
        plan->d_cta_begin, plan->d_bt_flat, o_part, lse_part, (__nv_bfloat16 *)out, lse, plan->num_q_heads,
        pool->desc.num_kv_heads, plan->group, plan->head_block, lists, pool->desc.num_pages, scale_log2, pool->status_dev,
        plan->window, plan->sinks);
    if (e == cudaSuccess && plan->info.merge_entries > 0)
        e = plan->max_parts <= kMergeBatch ? launch_merge<D, 1>(plan, out, lse, o_part, lse_part, stream)
                                           : launch_merge<D, kMergeWarps>(plan, out, lse, o_part, lse_part, stream);
    return e;
}

}  // namespace

cudaError_t launch_kv4_decode(const ap_kv_pool *pool, const ap_plan *plan, const void *q, void *out, float *lse, float *o_part,
                              float *lse_part, cudaStream_t stream) {
    cudaError_t e;
    if (plan->window > 0)
        e = pool->desc.head_dim == 128 ? launch_t<128, true>(pool, plan, q, out, lse, o_part, lse_part, stream)
                                       : launch_t<64, true>(pool, plan, q, out, lse, o_part, lse_part, stream);
    else
        e = pool->desc.head_dim == 128 ? launch_t<128, false>(pool, plan, q, out, lse, o_part, lse_part, stream)
                                       : launch_t<64, false>(pool, plan, q, out, lse, o_part, lse_part, stream);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ap
