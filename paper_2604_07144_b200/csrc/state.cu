// Host side of the layers with a state of fixed size per sequence: pool, planner, entry points.  Every entry point
// validates on the host and returns a status.
#include <algorithm>
#include <cstring>
#include <new>

#include "host_util.h"
#include "layers.h"

using namespace ap;

namespace {

// The scan's cut along time.  A warp walks its rows one after the other, so few long sequences leave SMs idle.  Cut into
// pieces, all but the first and the last are walked twice (once for the state behind them, once for their rows) and there
// are two launches.  It pays below kCutBelow warps an SM (6 x 1024 rows of 4096 channels, 10.4 warps an SM: 198 us cut, 209
// not), with pieces for kResident warps an SM, two rounds of those that are there together (8192 rows of 4096 channels: 314
// us; 16: 327, 24: 328, 32: 326).  Measured with sequences of one length: the rule counts sequences, whatever their rows, so a
// long one beside a few short ones is not cut (8192 rows of 4096 channels alone 319 us, beside seven of 2 rows 887).  Nor do the
// constants know what folding costs, a round a piece before: it shows where few channels make many pieces (64 channels: 8192 rows,
// 128 pieces, 55 us; 65536 rows, 1024 pieces, 444).
constexpr int kCutBelow = 12, kResident = 28, kLeastPiece = 64;

struct Cut {
    int32_t piece;       // rows of a piece, 0: no sequence is cut
};

Cut choose_cut(int sms, int blocks_c, int64_t chunk_seqs, int64_t chunk_rows) {
    const int64_t warps = chunk_seqs * blocks_c;
    if (warps >= kCutBelow * (int64_t)sms) return {0};
    // pieces for as many warps as are resident together (a launch leaves one piece of each sequence out)
    const int64_t rows = std::max<int64_t>(kLeastPiece, chunk_rows * blocks_c / (kResident * (int64_t)sms + warps));
    return {(int32_t)std::min<int64_t>(1 << 30, (rows + kScanTile - 1) / kScanTile * kScanTile)};
}

// Rows of a unit of the convolution.  A thread's start (weights, the rows before) costs as much as several rows: 8 x 1024 rows
// of 8192 channels take 49.7 us in runs of 32 or 64, 52.2 in runs of 16.  Shorter runs make kConvBlocks blocks an SM for few rows.
constexpr int kConvBlocks = 14;
int32_t conv_run(int sms, int blocks_c, int64_t rows) {
    int32_t run = 32;
    while (run > 4 && rows * blocks_c < (int64_t)kConvBlocks * sms * run) run /= 2;
    return run;
}

bool same_shape(const ap_state_desc &a, const ap_state_desc &b) {
    return a.num_slots == b.num_slots && a.channels == b.channels && a.state_dim == b.state_dim && a.conv_width == b.conv_width &&
           (a.device == b.device || (a.device < 0 && b.device < 0));
}

bool positive(const ap_state_desc *d) { return d && d->num_slots > 0 && d->channels > 0 && d->state_dim > 0 && d->conv_width > 0; }

bool supported(const ap_state_desc *d) {
    return d->channels % 8 == 0 && d->channels <= 1 << 20 && d->conv_width >= 2 && d->conv_width <= 4 &&
           (d->state_dim == 8 || d->state_dim == 16 || d->state_dim == 32 || d->state_dim == 64);
}

// Rows of `cols` numbers of `size` bytes, `stride` numbers apart: a tensor of a call.
struct Rows {
    const void *p;
    int64_t stride, cols;
    int size;
};

// Whether two tensors of n rows share a byte.  Rows of the same stride may lie between one another (slices of one
// projection's output); otherwise what lies between two rows counts as theirs.
bool overlap(const Rows &a, const Rows &b, int64_t n) {
    if (!a.p || !b.p || n <= 0) return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    const uintptr_t a1 = a0 + (uintptr_t)((n - 1) * a.stride + a.cols) * a.size, b1 = b0 + (uintptr_t)((n - 1) * b.stride + b.cols) * b.size;
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.stride * a.size != b.stride * b.size) return true;
    const uintptr_t s = (uintptr_t)(a.stride * a.size);
    const uintptr_t off = b0 >= a0 ? (b0 - a0) % s : (s - (a0 - b0) % s) % s;      // where b's rows begin within a's
    return off < (uintptr_t)a.cols * a.size || off + (uintptr_t)b.cols * b.size > s;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// stride 0: contiguous.  False: not one that the kernels take.
bool take_stride(int64_t given, int64_t cols, int64_t *out) {
    *out = given ? given : cols;
    return *out >= cols && *out % 8 == 0 && *out <= (int64_t)1 << 32;
}

int plan_create(ap_state_plan **out, ap_state_pool *pool, const ap_state_batch *b, void *stream) {
    if (!out) return AP_ERR_INVALID_ARG;
    *out = nullptr;
    if (!pool || !b || b->batch < 0) return AP_ERR_INVALID_ARG;
    if (b->batch > 0 && (!b->q_lens || !b->ctx_lens || !b->slots)) return AP_ERR_INVALID_ARG;
    const ap_state_desc &d = pool->desc;
    std::vector<uint8_t> taken((size_t)d.num_slots, 0);
    int64_t n_new = 0, chunk_rows = 0, singles = 0, chunk_seqs = 0;
    for (int s = 0; s < b->batch; ++s) {
        const int32_t ql = b->q_lens[s], cl = b->ctx_lens[s];
        if (ql < 0 || cl < 0 || ql > cl) return AP_ERR_INVALID_ARG;
        if (ql == 0) continue;
        if (b->slots[s] < 0 || b->slots[s] >= d.num_slots || taken[(size_t)b->slots[s]]) return AP_ERR_INVALID_ARG;
        taken[(size_t)b->slots[s]] = 1;
        n_new += ql;
        if (ql == 1) ++singles; else { ++chunk_seqs; chunk_rows += ql; }
    }
    if (n_new > (int64_t)1 << 30) return AP_ERR_UNSUPPORTED;

    const int blocks_c = (d.channels + scan_warp_channels(d.state_dim) - 1) / scan_warp_channels(d.state_dim);
    const Cut cut = choose_cut(pool->sm_count, blocks_c, chunk_seqs, chunk_rows);
    const int conv_blocks_c = (d.channels / 4 + kConvThreads - 1) / kConvThreads;
    const int32_t run = conv_run(pool->sm_count, conv_blocks_c, n_new);
    std::vector<StateUnit> conv, first, second, single;
    int64_t row = 0, segments = 0, split_seqs = 0;
    for (int s = 0; s < b->batch; ++s) {
        const int32_t ql = b->q_lens[s];
        if (ql == 0) continue;
        const int32_t kept = b->ctx_lens[s] > ql ? kUnitKept : 0;
        auto unit = [&](int32_t t0, int32_t rows, int32_t flags) {
            return StateUnit{(int32_t)(row + t0), rows, b->slots[s], flags | kept | (t0 == 0 ? kUnitFirst : 0) | (t0 + rows == ql ? kUnitLast : 0),
                             0, 0, ql, 0};
        };
        for (int32_t t0 = 0; t0 < ql; t0 += std::min(run, ql - t0)) conv.push_back(unit(t0, std::min(run, ql - t0), 0));
        if (ql == 1) {
            single.push_back(unit(0, 1, 0));
        } else if (cut.piece == 0 || ql < 2 * cut.piece) {
            first.push_back(unit(0, ql, 0));
        } else {
            const int32_t pieces = ql / cut.piece;                  // (the last takes the rest)
            for (int32_t i = 0; i < pieces; ++i) {
                const int32_t t0 = i * cut.piece;
                StateUnit u = unit(t0, i + 1 < pieces ? cut.piece : ql - t0, 0);
                u.seg_first = (int32_t)segments;
                u.seg = i;
                if (i > 0) second.push_back(u);
                if (i + 1 < pieces) {
                    if (i > 0) u.flags |= kUnitStateOnly;
                    first.push_back(u);
                }
            }
            segments += pieces;
            ++split_seqs;
        }
        row += ql;
    }
    // the longest first: blocks are handed out in order
    auto longer = [](const StateUnit &x, const StateUnit &y) { return x.rows > y.rows; };
    std::stable_sort(first.begin(), first.end(), longer);
    std::stable_sort(second.begin(), second.end(), longer);
    const int64_t most = (int64_t)std::max(first.size(), second.size()) * blocks_c + (int64_t)single.size() * (d.channels / 8);
    if (most >= (int64_t)1 << 31 || (int64_t)conv.size() * conv_blocks_c >= (int64_t)1 << 31) return AP_ERR_UNSUPPORTED;

    ap_state_plan *plan = new (std::nothrow) ap_state_plan();
    if (!plan) return AP_ERR_CUDA;
    const std::vector<StateUnit> *lists[4] = {&conv, &first, &second, &single};
    size_t ints = 0;
    for (auto *l : lists) ints += l->size() * (sizeof(StateUnit) / 4);
    if (d.device >= 0 && ints > 0) {
        DeviceGuard guard(d.device);
        if (!guard.ok) { delete plan; return AP_ERR_CUDA; }
        const int rc = acquire_plan_buffer(pool->plan_buffers, ints, &plan->buf);
        if (rc != AP_OK) { delete plan; return rc; }
        const StateUnit **at[4] = {&plan->d_conv, &plan->d_first, &plan->d_second, &plan->d_single};
        size_t o = 0;
        for (int i = 0; i < 4; ++i) {
            if (!lists[i]->empty()) std::memcpy(plan->buf.host + o, lists[i]->data(), lists[i]->size() * sizeof(StateUnit));
            *at[i] = (const StateUnit *)(plan->buf.dev + o);
            o += lists[i]->size() * (sizeof(StateUnit) / 4);
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
    plan->desc = d;
    plan->n_conv = (int)conv.size();
    plan->n_first = (int)first.size();
    plan->n_second = (int)second.size();
    plan->n_single = (int)single.size();
    plan->workspace_bytes = segments ? align_up((size_t)segments * d.channels * d.state_dim * sizeof(float), 256) +
                                           align_up((size_t)segments * d.channels * sizeof(float), 256)
                                     : 0;
    plan->info.n_new = n_new;
    plan->info.single_rows = singles;
    plan->info.chunk_seqs = chunk_seqs;
    plan->info.split_seqs = split_seqs;
    plan->info.segments = segments;
    plan->info.launches_scan = first.empty() ? (single.empty() ? 0 : 1) : second.empty() ? 1 : 2;
    *out = plan;
    return AP_OK;
}

}  // namespace

extern "C" {

size_t ap_state_pool_conv_bytes(const ap_state_desc *d) {
    if (!positive(d) || !supported(d)) return 0;
    return (size_t)d->num_slots * (size_t)(d->conv_width - 1) * (size_t)d->channels * 2u;
}

size_t ap_state_pool_scan_bytes(const ap_state_desc *d) {
    if (!positive(d) || !supported(d)) return 0;
    return (size_t)d->num_slots * (size_t)d->channels * (size_t)d->state_dim * 4u;
}

int ap_state_pool_create(ap_state_pool **out, const ap_state_desc *desc) {
    if (!out) return AP_ERR_INVALID_ARG;
    *out = nullptr;
    if (!positive(desc)) return AP_ERR_INVALID_ARG;
    if (!supported(desc)) return AP_ERR_UNSUPPORTED;
    if (!aligned16(desc->conv_base) || !aligned16(desc->scan_base)) return AP_ERR_INVALID_ARG;
    if (desc->device < 0 && (desc->conv_base || desc->scan_base)) return AP_ERR_INVALID_ARG;
    if (desc->conv_base && desc->scan_base) {              // (planes that share a byte)
        const uintptr_t c = (uintptr_t)desc->conv_base, s = (uintptr_t)desc->scan_base;
        if (c < s + ap_state_pool_scan_bytes(desc) && s < c + ap_state_pool_conv_bytes(desc)) return AP_ERR_INVALID_ARG;
    }
    ap_state_pool *p = new (std::nothrow) ap_state_pool();
    if (!p) return AP_ERR_CUDA;
    p->desc = *desc;
    p->sm_count = 148;
    if (desc->device >= 0) {
        DeviceGuard guard(desc->device);
        bool ok = guard.ok && cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, desc->device) == cudaSuccess;
        const bool allocate = !desc->conv_base && !desc->scan_base;
        auto plane = [&](void **base, bool *owns, size_t bytes) {
            if (!ok || !allocate) return;
            *owns = true;
            ok = cudaMalloc(base, bytes) == cudaSuccess && cudaMemset(*base, 0, bytes) == cudaSuccess;
        };
        plane(&p->desc.conv_base, &p->owns_conv, ap_state_pool_conv_bytes(desc));
        plane(&p->desc.scan_base, &p->owns_scan, ap_state_pool_scan_bytes(desc));
        // (the zeros are there before a stream that does not wait for the default one can read or write the slots)
        if (ok && allocate) ok = cudaStreamSynchronize(0) == cudaSuccess;
        if (!ok) {
            (void)cudaGetLastError();
            ap_state_pool_destroy(p);
            return AP_ERR_CUDA;
        }
    }
    *out = p;
    return AP_OK;
}

int ap_state_pool_destroy(ap_state_pool *pool) {
    if (!pool) return AP_ERR_INVALID_ARG;
    if (pool->desc.device >= 0) {
        DeviceGuard guard(pool->desc.device);
        if (guard.ok) (void)cudaDeviceSynchronize();
        for (auto &b : pool->plan_buffers) release_plan_buffer(b);
        if (pool->owns_conv && pool->desc.conv_base) (void)cudaFree(pool->desc.conv_base);
        if (pool->owns_scan && pool->desc.scan_base) (void)cudaFree(pool->desc.scan_base);
        (void)cudaGetLastError();
    }
    delete pool;
    return AP_OK;
}

void *ap_state_pool_conv_base(const ap_state_pool *pool) { return pool ? pool->desc.conv_base : nullptr; }
void *ap_state_pool_scan_base(const ap_state_pool *pool) { return pool ? pool->desc.scan_base : nullptr; }

int ap_state_plan_create(ap_state_plan **out, ap_state_pool *pool, const ap_state_batch *batch, void *stream) {
    try {
        return plan_create(out, pool, batch, stream);
    } catch (const std::bad_alloc &) {
        return AP_ERR_CUDA;
    }
}

int ap_state_plan_destroy(ap_state_plan *plan) {
    if (!plan) return AP_ERR_INVALID_ARG;
    if (plan->buf.dev) give_back_plan_buffer(plan->pool->plan_buffers, plan->buf);
    delete plan;
    return AP_OK;
}

int ap_state_plan_get_info(const ap_state_plan *plan, ap_state_info *info) {
    if (!plan || !info) return AP_ERR_INVALID_ARG;
    *info = plan->info;
    return AP_OK;
}

size_t ap_state_plan_workspace_bytes(const ap_state_plan *plan) { return plan ? plan->workspace_bytes : 0; }

int ap_conv_iteration(ap_state_pool *pool, const ap_state_plan *plan, const ap_conv_desc *conv, void *stream) {
    if (!pool || !plan || !conv || !same_shape(pool->desc, plan->desc)) return AP_ERR_INVALID_ARG;
    const int64_t D = pool->desc.channels, n = plan->info.n_new;
    ap_conv_desc c = *conv;
    if ((c.silu != 0 && c.silu != 1) || !take_stride(conv->x_row_stride, D, &c.x_row_stride) ||
        !take_stride(conv->out_row_stride, D, &c.out_row_stride))
        return AP_ERR_INVALID_ARG;
    if (pool->desc.device < 0) return AP_ERR_CUDA;
    if (n == 0) return AP_OK;
    if (!pool->desc.conv_base) return AP_ERR_INVALID_ARG;
    const void *x = c.x, *weight = c.weight, *bias = c.bias, *out = c.out;
    if (!x || !weight || !out || !aligned16(x) || !aligned16(weight) || !aligned16(bias) || !aligned16(out)) return AP_ERR_INVALID_ARG;
    const Rows o{out, c.out_row_stride, D, 2};
    const int64_t slots = pool->desc.num_slots, w = pool->desc.conv_width;
    auto flat = [](const void *p, int64_t count, int size) { return Rows{p, count, count, size}; };
    auto meets = [&](const Rows &r) {                      // (one long row against out's rows)
        const uintptr_t r0 = (uintptr_t)r.p, r1 = r0 + (uintptr_t)r.cols * r.size;
        const uintptr_t o0 = (uintptr_t)out, o1 = o0 + (uintptr_t)((n - 1) * o.stride + D) * 2;
        return r.p && r0 < o1 && o0 < r1;
    };
    const Rows plane = flat(pool->desc.conv_base, slots * (w - 1) * D, 2);
    if (overlap(o, Rows{x, c.x_row_stride, D, 2}, n) || meets(flat(weight, D * w, 2)) || meets(flat(bias, D, 2)) || meets(plane) ||
        overlap(plane, Rows{x, (n - 1) * c.x_row_stride + D, (n - 1) * c.x_row_stride + D, 2}, 1) ||
        overlap(plane, flat(weight, D * w, 2), 1) || overlap(plane, flat(bias, D, 2), 1))
        return AP_ERR_INVALID_ARG;
    DeviceGuard guard(pool->desc.device);
    if (!guard.ok) return AP_ERR_CUDA;
    if (launch_conv(pool, plan, c, (cudaStream_t)stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return AP_ERR_CUDA;
    }
    return AP_OK;
}

int ap_scan_iteration(ap_state_pool *pool, const ap_state_plan *plan, const ap_scan_desc *scan, void *workspace,
                      size_t workspace_bytes, void *stream) {
    if (!pool || !plan || !scan || !same_shape(pool->desc, plan->desc)) return AP_ERR_INVALID_ARG;
    const int64_t D = pool->desc.channels, N = pool->desc.state_dim, n = plan->info.n_new;
    ScanArgs g{};
    if ((scan->softplus != 0 && scan->softplus != 1) || !take_stride(scan->x_row_stride, D, &g.xs) ||
        !take_stride(scan->dt_row_stride, D, &g.dts) || !take_stride(scan->b_row_stride, N, &g.bs) ||
        !take_stride(scan->c_row_stride, N, &g.cs) || !take_stride(scan->z_row_stride, D, &g.zs) ||
        !take_stride(scan->out_row_stride, D, &g.os))
        return AP_ERR_INVALID_ARG;
    if (pool->desc.device < 0) return AP_ERR_CUDA;
    if (n == 0) return AP_OK;
    if (!pool->desc.scan_base) return AP_ERR_INVALID_ARG;
    const void *x = scan->x, *dt = scan->dt, *b = scan->b, *c = scan->c, *z = scan->z, *out = scan->out;
    const float *a = scan->a, *d_skip = scan->d_skip, *dt_bias = scan->dt_bias;
    if (!x || !dt || !a || !b || !c || !out) return AP_ERR_INVALID_ARG;
    for (const void *p : {x, dt, b, c, z, out, (const void *)a, (const void *)d_skip, (const void *)dt_bias})
        if (!aligned16(p)) return AP_ERR_INVALID_ARG;
    if (plan->workspace_bytes > 0) {
        if (!workspace || workspace_bytes < plan->workspace_bytes) return AP_ERR_WORKSPACE_TOO_SMALL;
        if ((uintptr_t)workspace & 255u) return AP_ERR_INVALID_ARG;
    }
    const Rows o{out, g.os, D, 2};
    const uintptr_t o0 = (uintptr_t)out, o1 = o0 + (uintptr_t)((n - 1) * g.os + D) * 2;
    auto meets = [&](const void *p, int64_t bytes) { return p && (uintptr_t)p < o1 && o0 < (uintptr_t)p + (uintptr_t)bytes; };
    if (overlap(o, Rows{x, g.xs, D, 2}, n) || overlap(o, Rows{dt, g.dts, D, 2}, n) || overlap(o, Rows{b, g.bs, N, 2}, n) ||
        overlap(o, Rows{c, g.cs, N, 2}, n) || overlap(o, Rows{z, g.zs, D, 2}, n) || meets(a, D * N * 4) || meets(d_skip, D * 4) ||
        meets(dt_bias, D * 4) || meets(pool->desc.scan_base, (int64_t)pool->desc.num_slots * D * N * 4) ||
        meets(plan->workspace_bytes ? workspace : nullptr, (int64_t)plan->workspace_bytes))
        return AP_ERR_INVALID_ARG;
    // nor does what the call keeps for itself overlap an input
    const int64_t planes = (int64_t)pool->desc.num_slots * D * N;
    const Rows slots{pool->desc.scan_base, planes, planes, 4};
    const Rows pieces{plan->workspace_bytes ? workspace : nullptr, (int64_t)plan->workspace_bytes, (int64_t)plan->workspace_bytes, 1};
    if (overlap(slots, pieces, 1)) return AP_ERR_INVALID_ARG;
    for (const Rows &kept : {slots, pieces}) {
        auto in = [&](const void *p, int64_t stride, int64_t cols, int size) {
            const int64_t all = (n - 1) * stride + cols;
            return overlap(kept, Rows{p, all, all, size}, 1);
        };
        if (in(x, g.xs, D, 2) || in(dt, g.dts, D, 2) || in(z, g.zs, D, 2) || in(b, g.bs, N, 2) || in(c, g.cs, N, 2) ||
            in(a, 0, D * N, 4) || in(d_skip, 0, D, 4) || in(dt_bias, 0, D, 4))
            return AP_ERR_INVALID_ARG;
    }
    g.x = (const uint16_t *)x, g.dt = (const uint16_t *)dt, g.b = (const uint16_t *)b, g.c = (const uint16_t *)c;
    g.z = (const uint16_t *)z, g.a = a, g.d_skip = d_skip, g.dt_bias = dt_bias, g.out = (uint16_t *)out;
    g.state = (float *)pool->desc.scan_base;
    g.seg_state = (float *)workspace;
    g.seg_dt = workspace ? (float *)((char *)workspace + align_up((size_t)plan->info.segments * D * N * sizeof(float), 256)) : nullptr;
    g.channels = (int)D;
    g.softplus = scan->softplus;
    DeviceGuard guard(pool->desc.device);
    if (!guard.ok) return AP_ERR_CUDA;
    if (launch_scan(pool, plan, g, (cudaStream_t)stream) != cudaSuccess) {
        (void)cudaGetLastError();
        return AP_ERR_CUDA;
    }
    return AP_OK;
}

}  // extern "C"
