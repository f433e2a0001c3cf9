// Causal attention of whole prompts, packed one after the other, K and V read from the projection's rows.
//
// Prompts of more than kShortRows tokens go to the tensor cores (tcgen05, accumulators in tensor memory), shorter ones
// to a kernel of mma.sync tiles; a plan with both launches both, but for a few short ones beside longer ones.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <new>
#include <utility>

#include "host_util.h"
#include "layers.h"
#include "prefill_tcgen05.cuh"

namespace ap {

namespace {

using namespace ptx;
using prefill::exp2_poly2;
using prefill::instr_desc;
using prefill::kMmaWarp;
using prefill::kPrefillThreads;
using prefill::kProducerWarp;
using prefill::kRescaleThreshold;
using prefill::kTileM;
using prefill::kTileN;
using prefill::kv_seq_k;
using prefill::kv_seq_v;
using prefill::max2;
using prefill::max3;
using prefill::PrefillCfg;
using prefill::rescale_o;
using prefill::smem_desc;

// 64 prompts of 64 tokens (32 q heads, 8 kv heads of 128): 26.4 us in the short kernel, 38.0 on the tensor cores; of 96: 58.3
// (with room for 128 rows) and 39.9.
constexpr int kShortRows = 64;
// A few short prompts beside longer ones are units of theirs, up to kFewUnits / 4 an SM, and spare a launch: 7 beside 9 of up to 1000
// tokens 37 us for 40, 7 beside one of 300 8.8 for 11.2, 11 (1.2 units an SM) 28.7 for 30.1; 15 (1.6) would be 12.3 for 11.7.
constexpr int kFewUnits = 5;
constexpr int kUnitSteps = 2;             // what a unit costs beside its steps, in steps
constexpr uint64_t kDrainNs = 100000000;  // bound of the waits for copies and products under way, after a wait that ran out

// ----------------------------------------------------- tensor-core units --
//
// A unit is 128 rows of a prompt for two q heads of a kv head (or one), over the prompt's rows up to its own last one.  Roles and
// tensor-memory columns are those of the paged prefill kernel (prefill_tcgen05.cuh): two softmax groups of 128 threads, a
// producer warp, an MMA-issuing warp per tile, one score region that the tiles use in turn.  What differs:
//   - 128 rows of K (of V) come in one request of 32 KB instead of eight of 4 KB through a block table, as
//     [half][128 rows][64] with the 128-byte swizzle, and begin at any row.
//   - A block stays and works through a list of units (the host deals them out, longest first, to the least loaded block).
//     Barriers and ring run on across units: while a unit's last weights and results are under way, the next one's Q, K and
//     V come in and its first scores are formed.  With a block a unit those were 3700 clocks of start and 1700 of gap
//     between blocks, of 12600 for a unit of one step (64 prompts of 128 tokens: 63 us, now 40).
//   - Results leave through shared memory as whole rows (a thread has a row: straight to memory each store touched 32).
// 8192 tokens at 32 / 8 heads of 128: 437 us, 1258 TFLOP/s, at the clock that the power limit leaves (1.5 GHz).  A step of the
// two tiles takes 2820 clocks, 2200 of them the tensor pipe's; a group's own chain (copy 280, maxima 520, exponentials 1490,
// then waits for P V and the next scores) is as long.  A score region for each tile, P written over it: 470 us, the chain
// then holds both products as well.  Units of one tile (equal q and kv heads, the last head of an odd group) leave softmax and
// tensor pipe to take turns: at 32 / 32 heads 619 us for the same products, at 30 / 10 468.  Heads of 64: 416 us for half the
// products (661 TFLOP/s): the exponentials, as many, bound it.
template <int D>
struct PromptCfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kQBytes = kTileM * D * 2, kKvTileBytes = kTileN * D * 2;
    static constexpr int kSlots = 4;                                  // of the ring of K and V tiles
    static constexpr int kStageBytes = 32 * 128;                      // a warp's rows on their way out, 64 columns at a time
    static constexpr int kOffQ = 0;                                   // [2] tiles A, B
    static constexpr int kOffK = 2 * kQBytes;
    static constexpr int kOffStage = kOffK + kSlots * kKvTileBytes;
    static constexpr int kOffBar = kOffStage + 8 * kStageBytes;
    static constexpr int kSmemBytes = 1024 + kOffBar + 256;
};

template <int D, int kTiles>
__global__ void __launch_bounds__(kPrefillThreads, 1)
prompt_tcgen05_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                      const __grid_constant__ CUtensorMap v_map, const PromptTile *__restrict__ tiles,
                      const int32_t *__restrict__ begin, __nv_bfloat16 *__restrict__ out, float *__restrict__ lse_out, int Hq,
                      float scale_log2, int *status, uint64_t wait_limit_ns) {
    using Cfg = PromptCfg<D>;
    using Cols = PrefillCfg<D>;
    constexpr int kSlots = Cfg::kSlots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = (uint8_t *)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t *bars = (uint64_t *)(smem + Cfg::kOffBar);
    uint64_t *q_full = bars + 0;                 // a unit's Q is there
    uint64_t *q_empty = bars + 1;                // its last scores are formed
    uint64_t *kv_full = bars + 2;                // [kSlots]
    uint64_t *kv_empty = kv_full + kSlots;       // [kSlots]
    uint64_t *s_full = kv_empty + kSlots;        // [2] per tile
    uint64_t *p_full = s_full + 2;               // [2]
    uint64_t *pv_done = p_full + 2;              // [2] O_x += P_x V of a step has completed
    uint64_t *s_out = pv_done + 2;               // [2] tile x's scores have been copied out of the shared region
    uint64_t *o_empty = s_out + 2;               // [2] a unit's O_x has been read
    uint32_t *tmem_slot = (uint32_t *)(o_empty + 2);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    volatile uint32_t *issued = tmem_slot + 2;   // the producer's: ring entries, units
    uint64_t *drained = (uint64_t *)(tmem_slot + 4);   // [2] after a wait that ran out: tile x's products have ended

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int first = begin[blockIdx.x], end = begin[blockIdx.x + 1];
    auto steps_of = [](const PromptTile &t) { return (t.row0 - t.start + t.rows + kTileN - 1) / kTileN; };

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        mbar_init(q_empty, kTiles);
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(&kv_full[s], 1);
            mbar_init(&kv_empty[s], kTiles);     // one commit per issuing warp
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(&s_full[x], 1);
            mbar_init(&p_full[x], 4);            // one arrival per softmax warp
            mbar_init(&pv_done[x], 1);
            mbar_init(&s_out[x], 4);
            mbar_init(&o_empty[x], 4);
            mbar_init(&drained[x], 1);
        }
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(tmem_slot, Cols::kTmemCols);
        tmem_relinquish();
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = *tmem_slot;
    griddep_launch_dependents();
    griddep_wait();                              // the preamble reads only the plan

    // Every role walks the block's units.  u: units so far, n: steps of them; ring entry e is in slot e % kSlots.
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == kProducerWarp) {
            // -------------------------------------------------- producer --
            if (lane == 0) {
                prefetch_tensormap(&q_map);
                prefetch_tensormap(&k_map);
                prefetch_tensormap(&v_map);
                bool ok = true;
                uint32_t e = 0, u = 0;
                for (int i = first; ok && i < end; ++i, ++u) {
                    const PromptTile tile = tiles[i];
                    const int n_steps = steps_of(tile), n_entries = 2 * n_steps;
                    if (u > 0 && !wait_or_abort(q_empty, (u - 1) & 1u, abort_flag, wait_limit_ns)) { ok = false; break; }
                    mbar_arrive_expect_tx(q_full, (uint32_t)(kTiles * Cfg::kQBytes));
                    tma_load_3d(smem + Cfg::kOffQ, &q_map, q_full, 0, tile.row0, tile.q_head * Cfg::kHalves);
                    if (kTiles == 2)
                        tma_load_3d(smem + Cfg::kOffQ + Cfg::kQBytes, &q_map, q_full, 0, tile.row0, tile.q_head_b * Cfg::kHalves);
                    // a unit's entries in the order K_0, K_1, V_0, K_2, V_1, ...
                    for (int m = 0; m < n_entries; ++m, ++e) {
                        const bool is_k = m == 0 || ((m & 1) && m < n_entries - 1);
                        const int j = is_k ? (m + 1) / 2 : (m == n_entries - 1 ? n_steps - 1 : m / 2 - 1);
                        const uint32_t s = e % kSlots;
                        if (!wait_or_abort(&kv_empty[s], (e / kSlots & 1u) ^ 1u, abort_flag, wait_limit_ns)) { ok = false; break; }
                        // (rows past the packed batch's last read as zeros; they count)
                        mbar_arrive_expect_tx(&kv_full[s], (uint32_t)Cfg::kKvTileBytes);
                        tma_load_3d(smem + Cfg::kOffK + s * Cfg::kKvTileBytes, is_k ? &k_map : &v_map, &kv_full[s], 0,
                                    tile.start + j * kTileN, tile.kv_head * Cfg::kHalves);
                    }
                }
                issued[0] = e;
                issued[1] = u;                           // (a unit given up among its entries counts: its Q is under way)
                if (!ok) {
                    record_status(status, AP_ERR_TIMEOUT);
                    *abort_flag = 1;
                }
            }
            __syncwarp();
        } else if (warp == kMmaWarp || (warp == kMmaWarp + 1 && kTiles == 2)) {
            // ----------------------------------------------- MMA issuers --
            const int x = warp - kMmaWarp;
            const uint32_t leader = elect_one();
            constexpr uint32_t kIdescQK = instr_desc(kTileM, kTileN, false);
            constexpr uint32_t kIdescPV = instr_desc(kTileM, D, true);
            // All three operands lie as [half][128 rows][64], 8-row groups 1024 B apart, halves 16 KB apart.
            constexpr uint32_t kHalfBytes = kTileN * 128;
            const uint64_t q_desc0 = smem_desc(smem_u32(smem + Cfg::kOffQ + x * Cfg::kQBytes), 16, 1024);
            const uint64_t k_desc0 = smem_desc(smem_u32(smem + Cfg::kOffK), 16, 1024);
            const uint64_t v_desc0 = smem_desc(smem_u32(smem + Cfg::kOffK), kHalfBytes, 1024);
            const uint32_t q_lo = (uint32_t)q_desc0, q_hi = (uint32_t)(q_desc0 >> 32);
            const uint32_t k_lo = (uint32_t)k_desc0, k_hi = (uint32_t)(k_desc0 >> 32);
            const uint32_t v_lo = (uint32_t)v_desc0, v_hi = (uint32_t)(v_desc0 >> 32);
            const uint32_t t_s = tmem + Cols::kColS, t_p = tmem + Cols::kColP + x * 64, t_o = tmem + Cols::kColO + x * 128;
            bool ok = true;
            auto wait = [&](uint64_t *bar, uint32_t phase) {
                if (ok) ok = wait_or_abort(bar, phase & 1u, abort_flag, wait_limit_ns);
            };
            // S = Q_x K^T with K in ring entry `e`, the tile's use number `use` of the score region.  The region passes from
            // tile to tile through two barriers with one waiter each: scores may be formed once those before them have been
            // copied out.
            auto issue_qk = [&](uint32_t e, uint32_t use) {
                const uint32_t s = e % kSlots;
                wait(&kv_full[s], e / kSlots);
                if (kTiles == 2 && x == 1) wait(&s_out[0], use);
                else if (use > 0) wait(&s_out[kTiles - 1], use - 1);
                if (!ok) return;
                tcgen05_fence_after();
                const uint32_t b0 = k_lo + ((s * Cfg::kKvTileBytes) >> 4);
#pragma unroll
                for (int kh = 0; kh < D / 64; ++kh)
                    umma_ss_x4(leader, t_s, q_lo + ((kh * kHalfBytes) >> 4), q_hi, b0 + ((kh * kHalfBytes) >> 4), k_hi, kIdescQK,
                               kh > 0 ? 1u : 0u, 32u >> 4, 32u >> 4);
                umma_commit(leader, &s_full[x]);
                umma_commit(leader, &kv_empty[s]);
            };
            uint32_t e0 = 0, n = 0, u = 0;
            for (int i = first; ok && i < end; ++i, ++u) {
                const PromptTile tile = tiles[i];
                const int n_steps = steps_of(tile);
                wait(q_full, u);
                issue_qk(e0, n);
                if (n_steps == 1 && ok) umma_commit(leader, q_empty);
                for (int j = 0; ok && j < n_steps; ++j) {
                    if (j + 1 < n_steps) {           // the next scores of the tile go ahead of this step's P V
                        issue_qk(e0 + (uint32_t)kv_seq_k(j + 1), n + j + 1);
                        if (j + 2 == n_steps && ok) umma_commit(leader, q_empty);
                    }
                    const uint32_t ev = e0 + (uint32_t)kv_seq_v(j, n_steps), s = ev % kSlots;
                    wait(&kv_full[s], ev / kSlots);
                    wait(&p_full[x], n + j);
                    if (j == 0 && u > 0) wait(&o_empty[x], u - 1);
                    if (!ok) break;
                    tcgen05_fence_after();
                    // O_x += P_x V, 16 keys an instruction: 8 columns of P, 2 groups of 8 rows of V
                    const uint32_t b0 = v_lo + ((s * Cfg::kKvTileBytes) >> 4);
                    constexpr uint32_t kVStep = (2 * 1024) >> 4;
#pragma unroll
                    for (int kq = 0; kq < kTileN / 64; ++kq)
                        umma_ts_x4(leader, t_o, t_p + kq * 32, b0 + kq * 4 * kVStep, v_hi, kIdescPV, (j == 0 && kq == 0) ? 0u : 1u, 8u,
                                   kVStep);
                    umma_commit(leader, &pv_done[x]);
                    umma_commit(leader, &kv_empty[s]);
                }
                e0 += 2 * n_steps;
                n += n_steps;
            }
            if (!ok && leader) {
                record_status(status, AP_ERR_TIMEOUT);
                *abort_flag = 1;
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // ------------------------------------------------------- softmax --
        const int x = warp >> 2;                                     // tile A or B
        if (x < kTiles) {
            const int r = threadIdx.x & 127;                         // query row = TMEM lane
            const uint32_t lane_addr = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            const uint32_t col_s = Cols::kColS, col_p = Cols::kColP + x * 64, col_o = Cols::kColO + x * 128;
            bool ok = true;
            uint32_t n = 0, e0 = 0;
            for (int i = first; ok && i < end; ++i) {
                const PromptTile tile = tiles[i];
                const int pos0 = tile.row0 - tile.start;             // position of the first row in its prompt
                const int kv_len = pos0 + tile.rows, n_steps = steps_of(tile);
                const int q_head = x == 0 ? tile.q_head : tile.q_head_b;
                const int my_pos = min(pos0 + r, kv_len - 1);        // last key this row sees
                float m_used = -INFINITY, l = 0.f;
                for (int j = 0; j < n_steps; ++j) {
                    // S_x(j) complete: copy this row's 128 scores out and give the region back at once
                    if (!wait_or_abort(&s_full[x], (n + j) & 1u, abort_flag, wait_limit_ns)) { ok = false; break; }
                    tcgen05_fence_after();
                    uint32_t sreg[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(lane_addr + col_s + c * 32, sreg[c]);
                    tmem_ld_wait();
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_out[x]);
                    const int tok0 = j * kTileN;
                    float mx = -INFINITY;
                    if (tok0 + kTileN - 1 > pos0) {
                        // diagonal or last step: one bit per key says whether the row sees it
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t seen = prefill::low_bits(my_pos + 1 - (tok0 + c * 32));
#pragma unroll
                            for (int k = 0; k < 32; ++k)
                                if (!(seen >> k & 1u)) sreg[c][k] = 0xFF800000u;            // -inf
                        }
                    }
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int k = 0; k < 32; k += 2)
                            mx = max3(mx, __uint_as_float(sreg[c][k]), __uint_as_float(sreg[c][k + 1]));
                    // P_x and O_x belong to the tensor pipe until O_x += P_x V of the step before is done
                    if (j > 0) {
                        if (!wait_or_abort(&pv_done[x], (n + j - 1) & 1u, abort_flag, wait_limit_ns)) { ok = false; break; }
                        tcgen05_fence_after();
                    }
                    // Keep the old reference max unless some row of the warp moved by more than the threshold: P stays
                    // bounded by 2^threshold and O needs no rescale most steps.
                    const float m_new = max2(m_used, mx);
                    const bool rescale = __any_sync(0xffffffffu, (m_new - m_used) * scale_log2 > kRescaleThreshold);   // (true on the first step)
                    float alpha = 1.f;
                    if (rescale) {
                        alpha = exp2_approx((m_used - m_new) * scale_log2);   // 0 on the first step
                        m_used = m_new;
                        if (j > 0) rescale_o<D>(lane_addr + col_o, alpha);
                    }
                    const float ms = fmaf(m_used, scale_log2, m_new - m_new);   // (a NaN score makes the row NaN)
                    const float2 sc2 = make_float2(scale_log2, scale_log2), nms2 = make_float2(-ms, -ms);
                    float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t preg[32];                                  // 64 keys as bf16 pairs
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            float2 xy = __ffma2_rn(make_float2(__uint_as_float(sreg[2 * c + (k >> 4)][(2 * k) & 31]),
                                                               __uint_as_float(sreg[2 * c + (k >> 4)][(2 * k + 1) & 31])),
                                                   sc2, nms2);
                            // one pair in eight goes to the FMA pipe instead of the special-function unit
                            if ((k & 7) == 7) {
                                xy = exp2_poly2<true>(xy);
                            } else {
                                xy.x = exp2_approx(xy.x);
                                xy.y = exp2_approx(xy.y);
                            }
                            // (the sum takes the weights as they are; P V takes them in bf16, each off by at most 2^-8 of itself)
                            sum2 = __fadd2_rn(sum2, xy);
                            preg[k] = pack_bf16x2(xy.x, xy.y);
                        }
                        tmem_st_32x32b_x32(lane_addr + col_p + c * 32, preg);
                    }
                    l = l * alpha + (sum2.x + sum2.y);
                    tmem_st_wait();
                    if (j == n_steps - 1 && kv_len < n_steps * kTileN) {
                        // Rows past the unit's last key belong to nobody it serves (the next prompt's, or none): 0 * V must be 0.
                        // Both tiles' groups clear them (the same zeros) before they hand their own P over: a tile that waited
                        // for the other's hand-over could find it two phases on.
                        const uint32_t ev = e0 + (uint32_t)kv_seq_v(j, n_steps), s = ev % kSlots;
                        if (!wait_or_abort(&kv_full[s], ev / kSlots & 1u, abort_flag, wait_limit_ns)) { ok = false; break; }
                        uint8_t *v_tile = smem + Cfg::kOffK + s * Cfg::kKvTileBytes;
                        const int past = kv_len - tok0;
                        for (int idx = r; idx < (kTileN - past) * (D / 8); idx += 128) {
                            const int key = past + idx / (D / 8), ch = idx % (D / 8);
                            *(uint4 *)(v_tile + (ch >> 3) * (kTileN * 128) + key * 128 + ((ch & 7) << 4)) = make_uint4(0, 0, 0, 0);
                        }
                        fence_proxy_async_smem();
                    }
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[x]);
                }
                if (ok) ok = wait_or_abort(&pv_done[x], (n + n_steps - 1) & 1u, abort_flag, wait_limit_ns);
                if (!ok) break;
                tcgen05_fence_after();
                uint32_t oreg[D / 32][32];
#pragma unroll
                for (int c = 0; c < D / 32; ++c) tmem_ld_32x32b_x32(lane_addr + col_o + c * 32, oreg[c]);
                tmem_ld_wait();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&o_empty[x]);             // (the next unit's products may begin)
                const float inv = 1.f / l;
                // 64 columns of the warp's rows at a time: 16-byte pieces of row r at piece ^ (r & 7), then out as whole rows
                uint8_t *rows = smem + Cfg::kOffStage + warp * Cfg::kStageBytes;
                __nv_bfloat16 *to = out + ((size_t)(tile.row0 + (warp & 3) * 32 + (lane >> 3)) * Hq + q_head) * D + (lane & 7) * 8;
                const int rows_left = tile.rows - (warp & 3) * 32;
#pragma unroll
                for (int half = 0; half < D / 64; ++half) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const uint32_t *o = &oreg[2 * half + c / 4][c % 4 * 8];
                        uint4 v;
                        v.x = pack_bf16x2(__uint_as_float(o[0]) * inv, __uint_as_float(o[1]) * inv);
                        v.y = pack_bf16x2(__uint_as_float(o[2]) * inv, __uint_as_float(o[3]) * inv);
                        v.z = pack_bf16x2(__uint_as_float(o[4]) * inv, __uint_as_float(o[5]) * inv);
                        v.w = pack_bf16x2(__uint_as_float(o[6]) * inv, __uint_as_float(o[7]) * inv);
                        *(uint4 *)(rows + lane * 128 + ((c ^ (lane & 7)) << 4)) = v;
                    }
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < 32; k += 4) {
                        const int row = k + (lane >> 3);
                        if (row < rows_left)
                            *(uint4 *)(to + (size_t)k * Hq * D + half * 64) = *(const uint4 *)(rows + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
                    }
                    __syncwarp();
                }
                if (r < tile.rows && lse_out)
                    lse_out[(size_t)(tile.row0 + r) * Hq + q_head] = (m_used * scale_log2 + log2f(l)) * 0.6931471805599453f;
                n += n_steps;
                e0 += 2 * n_steps;
            }
            if (!ok) {
                record_status(status, AP_ERR_TIMEOUT);
                *abort_flag = 1;
            }
        }
    }

    tcgen05_fence_before();
    __syncthreads();
    if (*abort_flag) {
        // Given up: what is under way still writes shared and tensor memory, and ends before they are given back.
        volatile int none = 0;
        if (warp == kMmaWarp || (warp == kMmaWarp + 1 && kTiles == 2)) {
            uint64_t *mine = &drained[warp - kMmaWarp];
            umma_commit(elect_one(), mine);
            (void)wait_or_abort(mine, 0, &none, kDrainNs);
        } else if (warp == kProducerWarp && lane == 0) {
            const uint32_t entries = issued[0], units = issued[1];
            for (uint32_t e = entries < (uint32_t)kSlots ? 0 : entries - kSlots; e < entries; ++e)
                (void)wait_or_abort(&kv_full[e % kSlots], e / kSlots & 1u, &none, kDrainNs);
            if (units > 0) (void)wait_or_abort(q_full, (units - 1) & 1u, &none, kDrainNs);
        }
        __syncthreads();
    }
    if (warp == kMmaWarp) tmem_dealloc(tmem, Cols::kTmemCols);
}

// ---------------------------------------------------------- short prompts --
//
// A block takes some blocks of 16 rows of a prompt for one kv head, as many as make kShortWarps items of (16 rows, q head), and
// each warp an item at a time (mma.sync m16n8k16: a 128-row tile of the tensor cores would be empty for the most part, and a
// unit's prologue and epilogue cost 5 us).  K and V up to the last of the rows stand in shared memory, with each warp's
// first Q all in flight together.  All scores of a row are in registers, so the softmax takes one pass.
constexpr int kShortWarps = 4;

template <int D>
struct ShortSmem {
    static constexpr int kStride = D * 2 + 16;                        // bytes of a row: 8 rows of an ldmatrix in 8 bank groups
    alignas(16) uint8_t q[kShortWarps][16 * kStride];                 // a warp's rows; then its results on their way out
    alignas(16) uint8_t k[kShortRows * kStride], v[kShortRows * kStride];
};

// 16 bytes global -> shared, asynchronous; zeros (and `from` is not read) where `there` is false
__device__ __forceinline__ void copy16_or_zero(void *to, const void *from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(there ? 16 : 0) : "memory");
}

// kBlocks: blocks an SM that registers are kept for, by the units there are for an SM.  More of them hide more, and each is slower:
// up to 2 units, 2 blocks (16 prompts of 1 to 64 tokens, 1.8 units an SM: 4.8 us, with 3 blocks 5.3, with 4 5.5); up to 4 units,
// 3 (64 prompts at 8 / 8 heads, 3.5 units: 5.8, with 2 6.8, with 4 6.5); else 4 (64 prompts of 64 tokens: 26.4, with 3 29.2; 200 of
// 1 to 64: 25.6, with 3 28.3).
template <int D, int kBlocks>
__global__ void __launch_bounds__(32 * kShortWarps, kBlocks)
prompt_short_kernel(const ShortPrompt *__restrict__ prompts, const uint16_t *q, const uint16_t *k, const uint16_t *v, uint16_t *out,
                    float *lse_out, int Hq, int Hkv, int64_t qs, int64_t ks, int64_t vs, float scale_log2) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    ShortSmem<D> &sm = *(ShortSmem<D> *)smem_raw;
    constexpr int kStride = ShortSmem<D>::kStride, kChunks = D / 8;
    const ShortPrompt p = prompts[blockIdx.x / Hkv];
    const int kv_head = (int)blockIdx.x % Hkv, G = Hq / Hkv;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int keys = p.block1 * 16;                                   // rows of K and V that the block's rows see
    griddep_launch_dependents();
    griddep_wait();
    uint8_t *mine = sm.q[warp];
    auto load_q = [&](int item) {
        const int row0 = (p.block1 - 1 - item / G) * 16, head = kv_head * G + item % G;
        for (int i = lane; i < 16 * kChunks; i += 32) {
            const int row = i / kChunks, ch = i % kChunks;
            const bool there = row0 + row < p.rows;
            copy16_or_zero(mine + row * kStride + ch * 16, q + (p.start + (int64_t)(there ? row0 + row : 0)) * qs + head * D + ch * 8, there);
        }
    };
    const int items = (p.block1 - p.block0) * G;
    if (warp < items) load_q(warp);
    for (int i = threadIdx.x; i < keys * kChunks; i += 32 * kShortWarps) {
        const int row = i / kChunks, ch = i % kChunks;
        const bool there = row < p.rows;                              // (rows past the prompt: zeros, whatever the next one holds)
        const int64_t at = p.start + (int64_t)(there ? row : 0);
        copy16_or_zero(sm.k + row * kStride + ch * 16, k + at * ks + kv_head * D + ch * 8, there);
        copy16_or_zero(sm.v + row * kStride + ch * 16, v + at * vs + kv_head * D + ch * 8, there);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    const uint32_t q_addr = smem_u32(mine) + (lane & 15) * kStride + (lane >> 4) * 16;
    const uint32_t k_addr = smem_u32(sm.k) + ((lane & 7) + (lane >> 4) * 8) * kStride + ((lane >> 3) & 1) * 16;
    const uint32_t v_addr = smem_u32(sm.v) + (lane & 15) * kStride + (lane >> 4) * 16;
    for (int item = warp; item < items; item += kShortWarps) {
        // (the later blocks, with more keys, first)
        const int rb = p.block1 - 1 - item / G, head = kv_head * G + item % G;
        const int row0 = rb * 16;
        if (item != warp) {
            load_q(item);
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
        }
        uint32_t qf[D / 16][4];
#pragma unroll
        for (int c = 0; c < D / 16; ++c) ldmatrix_x4(qf[c], q_addr + c * 32);
        // S: blocks of 16 keys up to the rows' own
        float s[kShortRows / 8][4];
#pragma unroll
        for (int kb = 0; kb < kShortRows / 16; ++kb) {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[2 * kb][e] = s[2 * kb + 1][e] = 0.f;
            if (kb <= rb) {
#pragma unroll
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t kf[4];
                    ldmatrix_x4(kf, k_addr + kb * 16 * kStride + c * 32);
                    mma_bf16_16816(s[2 * kb], qf[c][0], qf[c][1], qf[c][2], qf[c][3], kf[0], kf[1]);
                    mma_bf16_16816(s[2 * kb + 1], qf[c][0], qf[c][1], qf[c][2], qf[c][3], kf[2], kf[3]);
                }
            }
        }
        // a lane holds rows lane / 4 and lane / 4 + 8, keys 8 n + 2 (lane % 4) and the next
        const int r0 = row0 + (lane >> 2), key0 = 2 * (lane & 3);
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < kShortRows / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (8 * n + key0 + (e & 1) > r0 + 8 * (e >> 1)) s[n][e] = -INFINITY;
                m[e >> 1] = prefill::max2(m[e >> 1], s[n][e]);
            }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            m[h] = prefill::max2(m[h], __shfl_xor_sync(0xffffffffu, m[h], 1));
            m[h] = prefill::max2(m[h], __shfl_xor_sync(0xffffffffu, m[h], 2));
        }
        float o[D / 8][4];
#pragma unroll
        for (int n = 0; n < D / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.f;
#pragma unroll
        for (int kb = 0; kb < kShortRows / 16; ++kb) {
            if (kb > rb) continue;
            uint32_t pf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {                               // (rows lane / 4, + 8) x (keys 0-7, 8-15) of the block
                float w[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int h = i & 1;
                    w[e] = exp2_approx((s[2 * kb + (i >> 1)][2 * h + e] - m[h]) * scale_log2);
                    l[h] += w[e];
                }
                pf[i] = pack_bf16x2(w[0], w[1]);                        // (off by at most 2^-8 of itself; the sum takes it as it is)
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c) {
                uint32_t vf[4];
                ldmatrix_x4_trans(vf, v_addr + kb * 16 * kStride + c * 32);
                mma_bf16_16816(o[2 * c], pf[0], pf[1], pf[2], pf[3], vf[0], vf[1]);
                mma_bf16_16816(o[2 * c + 1], pf[0], pf[1], pf[2], pf[3], vf[2], vf[3]);
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
            l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
            const int row = r0 + 8 * h;
            if (lse_out && (lane & 3) == 0 && row < p.rows)
                lse_out[(p.start + (int64_t)row) * Hq + head] = (m[h] * scale_log2 + log2f(l[h])) * 0.6931471805599453f;
            const float inv = 1.f / l[h];
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
                *(uint32_t *)(mine + ((lane >> 2) + 8 * h) * kStride + n * 16 + (lane & 3) * 4) =
                    pack_bf16x2(o[n][2 * h] * inv, o[n][2 * h + 1] * inv);
        }
        __syncwarp();
        for (int i = lane; i < 16 * kChunks; i += 32) {
            const int row = i / kChunks, ch = i % kChunks;
            if (row0 + row < p.rows)
                *(uint4 *)(out + ((p.start + (int64_t)(row0 + row)) * Hq + head) * D + ch * 8) = *(const uint4 *)(mine + row * kStride + ch * 16);
        }
        __syncwarp();
    }
}

template <int D>
cudaError_t launch_prompt_t(ap_kv_pool *pool, const ap_prompt_plan *plan, const void *q, const void *k, const void *v,
                            void *out, float *lse, const ap_prompt_strides &st, cudaStream_t stream) {
    using Cfg = PromptCfg<D>;
    static bool configured[64] = {};
    const int dev = pool->desc.device & 63;
    if (!configured[dev]) {
        cudaError_t e = cudaFuncSetAttribute(prompt_tcgen05_kernel<D, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(prompt_tcgen05_kernel<D, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg::kSmemBytes);
        for (auto kernel : {prompt_short_kernel<D, 2>, prompt_short_kernel<D, 3>, prompt_short_kernel<D, 4>})
            if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(ShortSmem<D>));
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    const int Hq = plan->num_q_heads, Hkv = pool->desc.num_kv_heads;
    const float scale_log2 = plan->scale * 1.4426950408889634f;
    cudaError_t e = cudaSuccess;
    if (plan->info.tiles > 0) {
        CUtensorMap q_map, k_map, v_map;
        if (encode_rows_tensor_map(&q_map, q, plan->info.n_rows, Hq, D, st.q_row_stride) != AP_OK ||
            encode_rows_tensor_map(&k_map, k, plan->info.n_rows, Hkv, D, st.k_row_stride) != AP_OK ||
            encode_rows_tensor_map(&v_map, v, plan->info.n_rows, Hkv, D, st.v_row_stride) != AP_OK)
            return cudaErrorInvalidValue;
        for (int t = 2; t >= 1 && e == cudaSuccess; --t) {
            const PromptLists &l = plan->lists[t - 1];
            if (l.blocks == 0) continue;
            TimedScope ts(pool, AP_KERNEL_PREFILL, stream);
            e = launch_overlapped(t == 2 ? prompt_tcgen05_kernel<D, 2> : prompt_tcgen05_kernel<D, 1>, (unsigned)l.blocks,
                                  (unsigned)kPrefillThreads, (size_t)Cfg::kSmemBytes, stream, q_map, k_map, v_map, l.tiles, l.begin,
                                  (__nv_bfloat16 *)out, lse, Hq, scale_log2, pool->status_dev, pool->wait_limit_ns);
        }
    }
    if (e == cudaSuccess && plan->info.short_units > 0) {
        TimedScope ts(pool, AP_KERNEL_PREFILL, stream);
        const int64_t units = plan->info.short_units, sms = pool->sm_count;
        e = launch_overlapped(units <= 2 * sms ? prompt_short_kernel<D, 2> : units <= 4 * sms ? prompt_short_kernel<D, 3> : prompt_short_kernel<D, 4>,
                              (unsigned)units, 32u * kShortWarps, sizeof(ShortSmem<D>), stream, plan->d_short, (const uint16_t *)q, (const uint16_t *)k,
                              (const uint16_t *)v, (uint16_t *)out, lse, Hq, Hkv, st.q_row_stride, st.k_row_stride, st.v_row_stride, scale_log2);
    }
    return e != cudaSuccess ? e : cudaGetLastError();
}

// Units to blocks, one block an SM: the longest first, each to the block with the least to do.  A unit takes its steps and
// about two more (results out, first softmax).
void deal_out(std::vector<PromptTile> &tiles, int sms, std::vector<PromptTile> *dealt, std::vector<int32_t> *begin) {
    if (tiles.empty()) return;
    auto steps = [](const PromptTile &t) { return (t.row0 - t.start + t.rows + kTileN - 1) / kTileN; };
    std::stable_sort(tiles.begin(), tiles.end(), [&](const PromptTile &x, const PromptTile &y) { return steps(x) > steps(y); });
    const size_t blocks = std::min<size_t>(tiles.size(), (size_t)std::max(1, sms));
    std::vector<std::pair<int64_t, int32_t>> load;       // (steps so far, block), the least on top
    for (size_t i = 0; i < blocks; ++i) load.push_back({0, (int32_t)i});
    std::vector<int32_t> of(tiles.size()), count(blocks, 0);
    auto more = std::greater<std::pair<int64_t, int32_t>>();
    std::make_heap(load.begin(), load.end(), more);
    for (size_t i = 0; i < tiles.size(); ++i) {
        std::pop_heap(load.begin(), load.end(), more);
        of[i] = load.back().second;
        ++count[(size_t)of[i]];
        load.back().first += steps(tiles[i]) + kUnitSteps;
        std::push_heap(load.begin(), load.end(), more);
    }
    begin->assign(blocks + 1, 0);
    for (size_t i = 0; i < blocks; ++i) (*begin)[i + 1] = (*begin)[i] + count[i];
    std::vector<int32_t> next(begin->begin(), begin->end() - 1);
    dealt->resize(tiles.size());
    for (size_t i = 0; i < tiles.size(); ++i) (*dealt)[(size_t)next[(size_t)of[i]]++] = tiles[i];
}

int plan_create(ap_prompt_plan **out, ap_kv_pool *pool, const ap_prompt_desc *b, void *stream) {
    if (!out) return AP_ERR_INVALID_ARG;
    *out = nullptr;
    if (!pool || !b || b->batch < 0 || b->num_q_heads <= 0 || (b->batch > 0 && !b->lens)) return AP_ERR_INVALID_ARG;
    const int Hkv = pool->desc.num_kv_heads, Hq = b->num_q_heads, d = pool->desc.head_dim;
    if (Hq % Hkv != 0) return AP_ERR_INVALID_ARG;
    const int G = Hq / Hkv;
    if (G > 8) return AP_ERR_UNSUPPORTED;
    const int short_blocks = std::max(1, kShortWarps / G);                    // blocks of 16 rows of a unit
    int64_t rows = 0, pairs = 0, tiles_n = 0, shorts_n = 0, few = 0;
    for (int s = 0; s < b->batch; ++s) {
        const int32_t n = b->lens[s];
        if (n < 0) return AP_ERR_INVALID_ARG;
        rows += n;
        pairs += (int64_t)n * ((int64_t)n + 1) / 2;
        if (n > kShortRows) tiles_n += ((int64_t)n + kTileM - 1) / kTileM * Hkv * ((G + 1) / 2);
        else if (n > 0) shorts_n += ((n + 15) / 16 + short_blocks - 1) / short_blocks, few += (int64_t)Hkv * ((G + 1) / 2);
    }
    const int32_t short_rows = tiles_n > 0 && few * 4 <= (int64_t)kFewUnits * pool->sm_count ? 0 : kShortRows;
    // (row numbers of a last tile's keys, past the end of the batch, stay within 32 bits)
    if (rows > (int64_t)1 << 30 || tiles_n > (int64_t)1 << 27 || shorts_n * Hkv >= (int64_t)1 << 31) return AP_ERR_UNSUPPORTED;
    std::vector<PromptTile> tiles[2];                    // units of one tile, of two
    std::vector<ShortPrompt> shorts;
    shorts.reserve((size_t)shorts_n);
    int32_t start = 0;
    for (int s = 0; s < b->batch; ++s) {
        const int32_t n = b->lens[s];
        if (n > short_rows) {
            for (int32_t t0 = 0; t0 < n; t0 += kTileM)
                for (int kv = 0; kv < Hkv; ++kv)
                    for (int g = 0; g < G; g += 2) {
                        const bool two = g + 1 < G;
                        tiles[two].push_back({start + t0, std::min(kTileM, n - t0), start, kv * G + g, two ? kv * G + g + 1 : -1, kv, {0, 0}});
                    }
        } else if (n > 0) {
            const int blocks = (n + 15) / 16;
            for (int b1 = blocks; b1 > 0; b1 -= short_blocks) shorts.push_back({start, n, std::max(0, b1 - short_blocks), b1});
        }
        start += n;
    }
    std::stable_sort(shorts.begin(), shorts.end(), [](const ShortPrompt &x, const ShortPrompt &y) { return x.block1 > y.block1; });
    std::vector<PromptTile> dealt[2];
    std::vector<int32_t> begin[2];
    for (int t = 0; t < 2; ++t) deal_out(tiles[t], pool->sm_count, &dealt[t], &begin[t]);

    ap_prompt_plan *plan = new (std::nothrow) ap_prompt_plan();
    if (!plan) return AP_ERR_CUDA;
    size_t ints = shorts.size() * (sizeof(ShortPrompt) / 4), at[2];
    for (int t = 0; t < 2; ++t) {
        at[t] = ints;                                    // the units, then where each block's begin
        ints += (dealt[t].size() * (sizeof(PromptTile) / 4) + begin[t].size() + 7) / 8 * 8;
    }
    if (pool->desc.device >= 0 && ints > 0) {
        DeviceGuard guard(pool->desc.device);
        if (!guard.ok) { delete plan; return AP_ERR_CUDA; }
        const int rc = acquire_plan_buffer(pool->plan_buffers, ints, &plan->buf);
        if (rc != AP_OK) { delete plan; return rc; }
        if (!shorts.empty()) std::memcpy(plan->buf.host, shorts.data(), shorts.size() * sizeof(ShortPrompt));
        plan->d_short = (const ShortPrompt *)plan->buf.dev;
        for (int t = 0; t < 2; ++t) {
            if (dealt[t].empty()) continue;
            const size_t tile_ints = dealt[t].size() * (sizeof(PromptTile) / 4);
            std::memcpy(plan->buf.host + at[t], dealt[t].data(), tile_ints * 4);
            std::memcpy(plan->buf.host + at[t] + tile_ints, begin[t].data(), begin[t].size() * 4);
            plan->lists[t] = {(const PromptTile *)(plan->buf.dev + at[t]), plan->buf.dev + at[t] + tile_ints, (int)begin[t].size() - 1};
        }
        cudaStream_t st = (cudaStream_t)stream;
        if (cudaMemcpyAsync(plan->buf.dev, plan->buf.host, ints * 4, cudaMemcpyHostToDevice, st) != cudaSuccess ||
            cudaEventRecord(plan->buf.uploaded, st) != cudaSuccess) {
            (void)cudaGetLastError();
            give_back_plan_buffer(pool->plan_buffers, plan->buf);
            delete plan;
            return AP_ERR_CUDA;
        }
    }
    plan->pool = pool;
    plan->num_q_heads = Hq;
    plan->scale = b->softmax_scale > 0.f ? b->softmax_scale : 1.0f / std::sqrt((float)d);
    plan->info.n_rows = rows;
    plan->info.pairs = pairs;
    plan->info.tiles = (int64_t)(dealt[0].size() + dealt[1].size());
    plan->info.short_units = (int64_t)shorts.size() * Hkv;
    plan->info.launches = (dealt[0].empty() ? 0 : 1) + (dealt[1].empty() ? 0 : 1) + (shorts.empty() ? 0 : 1);
    *out = plan;
    return AP_OK;
}

}  // namespace

cudaError_t launch_prompt(ap_kv_pool *pool, const ap_prompt_plan *plan, const void *q, const void *k, const void *v,
                          void *out, float *lse, const ap_prompt_strides &strides, cudaStream_t stream) {
    if (pool->desc.head_dim == 128) return launch_prompt_t<128>(pool, plan, q, k, v, out, lse, strides, stream);
    return launch_prompt_t<64>(pool, plan, q, k, v, out, lse, strides, stream);
}

}  // namespace ap

using namespace ap;

extern "C" {

int ap_prompt_plan_create(ap_prompt_plan **out, ap_kv_pool *pool, const ap_prompt_desc *prompts, void *stream) {
    try {
        return plan_create(out, pool, prompts, stream);
    } catch (const std::bad_alloc &) {
        return AP_ERR_CUDA;
    }
}

int ap_prompt_plan_destroy(ap_prompt_plan *plan) {
    if (!plan) return AP_ERR_INVALID_ARG;
    if (plan->buf.dev) give_back_plan_buffer(plan->pool->plan_buffers, plan->buf);
    delete plan;
    return AP_OK;
}

int ap_prompt_plan_get_info(const ap_prompt_plan *plan, ap_prompt_info *info) {
    if (!plan || !info) return AP_ERR_INVALID_ARG;
    *info = plan->info;
    return AP_OK;
}

int ap_prompt_attention(ap_kv_pool *pool, const ap_prompt_plan *plan, const void *q, const void *k, const void *v, void *out,
                        float *lse, const ap_prompt_strides *strides, void *stream) {
    if (!pool || !plan || plan->pool != pool || !strides) return AP_ERR_INVALID_ARG;
    const int64_t d = pool->desc.head_dim, Hq = plan->num_q_heads, Hkv = pool->desc.num_kv_heads, n = plan->info.n_rows;
    ap_prompt_strides st = *strides;
    if (st.q_row_stride == 0) st.q_row_stride = Hq * d;
    if (st.k_row_stride == 0) st.k_row_stride = Hkv * d;
    if (st.v_row_stride == 0) st.v_row_stride = Hkv * d;
    const int64_t far = (int64_t)1 << 32;
    if (st.q_row_stride < Hq * d || st.k_row_stride < Hkv * d || st.v_row_stride < Hkv * d ||
        (st.q_row_stride | st.k_row_stride | st.v_row_stride) % 8 || st.q_row_stride > far || st.k_row_stride > far || st.v_row_stride > far)
        return AP_ERR_INVALID_ARG;
    if (pool->desc.device < 0) return AP_ERR_CUDA;
    if (n == 0) return AP_OK;
    if (!q || !k || !v || !out || (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)out) & 15u) || ((uintptr_t)lse & 3u))
        return AP_ERR_INVALID_ARG;
    auto meets = [&](const void *p, int64_t stride, int64_t cols, const void *o, int64_t bytes) {
        const uintptr_t a = (uintptr_t)p, e = a + (uintptr_t)((n - 1) * stride + cols) * 2, o0 = (uintptr_t)o;
        return o && a < o0 + (uintptr_t)bytes && o0 < e;
    };
    for (int i = 0; i < 2; ++i) {
        const void *o = i ? (const void *)lse : out;
        const int64_t bytes = i ? n * Hq * 4 : n * Hq * d * 2;
        if (meets(q, st.q_row_stride, Hq * d, o, bytes) || meets(k, st.k_row_stride, Hkv * d, o, bytes) ||
            meets(v, st.v_row_stride, Hkv * d, o, bytes))
            return AP_ERR_INVALID_ARG;
    }
    if (lse && (uintptr_t)lse < (uintptr_t)out + (uintptr_t)(n * Hq * d * 2) && (uintptr_t)out < (uintptr_t)lse + (uintptr_t)(n * Hq * 4))
        return AP_ERR_INVALID_ARG;
    DeviceGuard guard(pool->desc.device);
    if (!guard.ok) return AP_ERR_CUDA;
    if (launch_prompt(pool, plan, q, k, v, out, lse, st, (cudaStream_t)stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return AP_ERR_CUDA;
    }
    return AP_OK;
}

}  // extern "C"
