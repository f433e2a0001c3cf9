// Appending to, reading back from and widening a 4-bit pool (the format is described in kv4.cuh).  All
// three are single passes over their data, bound by HBM: 8000 rows at 8 heads of 128, appended and read back
// (84 MB), 16.2 us (5.2 TB/s; 16.6 us in a loop of seconds); widening 1290 pages of 8 heads (107 MB read and written) 15.5 us.
#include "internal.h"
#include "kv4.cuh"
#include "ptx.cuh"

namespace ap {

namespace {

using ptx::load16;
using ptx::load4;
using ptx::load8;

// A thread has elements 32 g + 8 t .. + 7 of every group g of one head row, for its t: the words of a row that
// are stored next to one another (16 bytes at d = 128).  The four lanes of a quad have the row's four t.
__device__ __forceinline__ void row_and_head(int64_t rh, int num_kv_heads, int64_t &row, int &head) {
    if (rh < (int64_t)1 << 32) {                         // (a 64-bit division takes as long as the rest of the thread)
        row = (uint32_t)rh / (uint32_t)num_kv_heads;
        head = (int)((uint32_t)rh % (uint32_t)num_kv_heads);
    } else {
        row = rh / num_kv_heads;
        head = (int)(rh % num_kv_heads);
    }
}

// One thread quantises its slice of a K row and of the V row; a quad shares its groups' maxima by shuffle and its
// first lane stores the steps.  All loads go out first: 2 d / 32 of 16 bytes a thread.
template <int D>
__global__ void __launch_bounds__(128) kv4_append_kernel(uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                                                         const uint4 *__restrict__ k_new, const uint4 *__restrict__ v_new,
                                                         const int32_t *__restrict__ append_dst, int64_t n_slices,
                                                         int num_kv_heads, int num_pages, int *status) {
    using T = kv4::Tile<D>;
    constexpr int NG = T::kGroups;
    const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t i = idx < n_slices ? idx : n_slices - 1;      // the shuffles need whole warps; the rest stores nothing
    const int t = (int)(i & 3);
    int64_t row;
    int g;
    row_and_head(i >> 2, num_kv_heads, row, g);
    const int32_t dst = __ldg(append_dst + row);                // plan data: uploaded before any kernel of the step
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    const int64_t vec = (i >> 2) * (D / 8) + t;
    uint4 k[NG], v[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        k[j] = load16(k_new + vec + 4 * j);
        v[j] = load16(v_new + vec + 4 * j);
    }
    uint32_t kw[NG], vw[NG], ks[NG], vs[NG];
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        float a, b;
        kw[j] = kv4::quantise8(k[j], a);
        vw[j] = kv4::quantise8(v[j], b);
        ks[j] = __float_as_uint(a) >> 16;
        vs[j] = __float_as_uint(b) >> 16;
    }
    const int32_t page = dst >> 4, slot = dst & 15;
    if (idx >= n_slices) return;
    if (page < 0 || page >= num_pages) {
        ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        return;
    }
    const int64_t tile = ((int64_t)page * num_kv_heads + g) * T::kBytes;
    const int words = slot * T::kRowBytes + 4 * NG * t, steps = T::kCodeBytes + 2 * NG * slot;
    if constexpr (NG == 4) {
        *reinterpret_cast<uint4 *>(k_pool + tile + words) = make_uint4(kw[0], kw[1], kw[2], kw[3]);
        *reinterpret_cast<uint4 *>(v_pool + tile + words) = make_uint4(vw[0], vw[1], vw[2], vw[3]);
        if (t == 0) {
            *reinterpret_cast<uint2 *>(k_pool + tile + steps) = make_uint2(ks[0] | ks[1] << 16, ks[2] | ks[3] << 16);
            *reinterpret_cast<uint2 *>(v_pool + tile + steps) = make_uint2(vs[0] | vs[1] << 16, vs[2] | vs[3] << 16);
        }
    } else {
        *reinterpret_cast<uint2 *>(k_pool + tile + words) = make_uint2(kw[0], kw[1]);
        *reinterpret_cast<uint2 *>(v_pool + tile + words) = make_uint2(vw[0], vw[1]);
        if (t == 0) {
            *reinterpret_cast<uint32_t *>(k_pool + tile + steps) = ks[0] | ks[1] << 16;
            *reinterpret_cast<uint32_t *>(v_pool + tile + steps) = vs[0] | vs[1] << 16;
        }
    }
}

// A slice's words and steps -> its d / 32 vectors of eight bf16 values.
template <int D>
__device__ __forceinline__ void read_slice(const uint8_t *row_words, const uint8_t *row_steps, uint4 (&out)[kv4::Tile<D>::kGroups]) {
    constexpr int NG = kv4::Tile<D>::kGroups;
    uint32_t w[NG], s[NG / 2];
    if constexpr (NG == 4) {
        const uint4 a = load16(row_words);
        const uint2 b = load8(row_steps);
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
        s[0] = b.x; s[1] = b.y;
    } else {
        const uint2 a = load8(row_words);
        w[0] = a.x; w[1] = a.y;
        s[0] = load4(row_steps);
    }
#pragma unroll
    for (int j = 0; j < NG; ++j) out[j] = kv4::dequantise8(w[j], (uint16_t)(j & 1 ? s[j / 2] >> 16 : s[j / 2] & 0xFFFFu));
}

// Reads the plan's new rows back, [N_new][Hkv][d] bf16: the values that a 4-bit pool stands for.
template <int D>
__global__ void __launch_bounds__(128) kv4_read_new_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                                                           uint4 *__restrict__ k_out, uint4 *__restrict__ v_out,
                                                           const int32_t *__restrict__ append_dst, int64_t n_slices,
                                                           int num_kv_heads, int num_pages, int *status) {
    using T = kv4::Tile<D>;
    constexpr int NG = T::kGroups;
    const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t i = idx < n_slices ? idx : n_slices - 1;
    const int t = (int)(i & 3);
    int64_t row;
    int g;
    row_and_head(i >> 2, num_kv_heads, row, g);
    const int32_t dst = __ldg(append_dst + row);
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    if (idx >= n_slices) return;
    const int32_t page = dst >> 4, slot = dst & 15;
    if (page < 0 || page >= num_pages) {
        ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        return;
    }
    const int64_t tile = ((int64_t)page * num_kv_heads + g) * T::kBytes, vec = (i >> 2) * (D / 8) + t;
    const int words = slot * T::kRowBytes + 4 * NG * t, steps = T::kCodeBytes + 2 * NG * slot;
    uint4 k[NG], v[NG];
    read_slice<D>(k_pool + tile + words, k_pool + tile + steps, k);
    read_slice<D>(v_pool + tile + words, v_pool + tile + steps, v);
#pragma unroll
    for (int j = 0; j < NG; ++j) {
        k_out[vec + 4 * j] = k[j];
        v_out[vec + 4 * j] = v[j];
    }
}

// The same of a bf16 pool: the values it holds.  One thread per eight elements and plane.
__global__ void __launch_bounds__(256) kv_read_new_kernel(const uint4 *__restrict__ k_pool, const uint4 *__restrict__ v_pool,
                                                          uint4 *__restrict__ k_out, uint4 *__restrict__ v_out,
                                                          const int32_t *__restrict__ append_dst, int64_t n_vec, int num_kv_heads,
                                                          int chunks, int num_pages, int *status) {
    const int64_t v = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    if (v >= n_vec) return;
    const int c = (int)(v % chunks);
    const int64_t rh = v / chunks;
    const int g = (int)(rh % num_kv_heads);
    const int32_t dst = __ldg(append_dst + rh / num_kv_heads);
    const int32_t page = dst >> 4, slot = dst & 15;
    if (page < 0 || page >= num_pages) {
        ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        return;
    }
    const int64_t o = (((int64_t)page * num_kv_heads + g) * kPageSize + slot) * chunks + c;
    k_out[v] = load16(k_pool + o);
    v_out[v] = load16(v_pool + o);
}

// Widens the listed pages to bf16 pages of the same layout as a bf16 pool's, page after page in the list's
// order: what the prefill kernel's TMA and tensor cores read.  A block takes one page of one plane: it reads
// Hkv tiles in a row and writes Hkv bf16 tiles in a row.
template <int D>
__global__ void __launch_bounds__(256) kv4_widen_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                                                        uint4 *__restrict__ k_out, uint4 *__restrict__ v_out,
                                                        const int32_t *__restrict__ pages, int num_kv_heads, int num_pages,
                                                        int *status) {
    using T = kv4::Tile<D>;
    constexpr int kChunks = D / 8;
    const int at = blockIdx.x >> 1;
    const bool is_v = blockIdx.x & 1;
    int32_t page = __ldg(pages + at);
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    if (page < 0 || page >= num_pages) {
        if (threadIdx.x == 0) ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        page = 0;
    }
    const uint8_t *src = (is_v ? v_pool : k_pool) + (int64_t)page * num_kv_heads * T::kBytes;
    uint4 *dst = (is_v ? v_out : k_out) + (int64_t)at * num_kv_heads * kPageSize * kChunks;
    const int n = num_kv_heads * kPageSize * 4;                  // slices of rows, a thread one at a time
    for (int i = threadIdx.x; i < n; i += 256) {
        const int t = i & 3, row = i >> 2, slot = row % kPageSize;
        const uint8_t *tile = src + (row / kPageSize) * T::kBytes;
        uint4 x[T::kGroups];
        read_slice<D>(tile + slot * T::kRowBytes + 4 * T::kGroups * t, tile + T::kCodeBytes + 2 * T::kGroups * slot, x);
#pragma unroll
        for (int j = 0; j < T::kGroups; ++j) dst[row * kChunks + 4 * j + t] = x[j];
    }
}

template <int D>
cudaError_t append_t(const ap_kv_pool *pool, const ap_plan *plan, const void *k_new, const void *v_new, cudaStream_t stream) {
    const int64_t n = plan->info.n_new * pool->desc.num_kv_heads * 4;
    return launch_overlapped(kv4_append_kernel<D>, (unsigned)((n + 127) / 128), 128u, 0, stream, (uint8_t *)pool->desc.k_base,
                             (uint8_t *)pool->desc.v_base, (const uint4 *)k_new, (const uint4 *)v_new, plan->d_append_dst, n,
                             pool->desc.num_kv_heads, pool->desc.num_pages, pool->status_dev);
}

template <int D>
cudaError_t read_t(const ap_kv_pool *pool, const ap_plan *plan, void *k, void *v, cudaStream_t stream) {
    const int64_t n = plan->info.n_new * pool->desc.num_kv_heads * 4;
    return launch_overlapped(kv4_read_new_kernel<D>, (unsigned)((n + 127) / 128), 128u, 0, stream,
                             (const uint8_t *)pool->desc.k_base, (const uint8_t *)pool->desc.v_base, (uint4 *)k, (uint4 *)v,
                             plan->d_append_dst, n, pool->desc.num_kv_heads, pool->desc.num_pages, pool->status_dev);
}

template <int D>
cudaError_t widen_t(const ap_kv_pool *pool, const ap_plan *plan, void *k, void *v, cudaStream_t stream) {
    return launch_overlapped(kv4_widen_kernel<D>, (unsigned)(2 * plan->n_wide_pages), 256u, 0, stream,
                             (const uint8_t *)pool->desc.k_base, (const uint8_t *)pool->desc.v_base, (uint4 *)k, (uint4 *)v,
                             plan->d_wide_pages, pool->desc.num_kv_heads, pool->desc.num_pages, pool->status_dev);
}

}  // namespace

cudaError_t launch_kv4_append(const ap_kv_pool *pool, const ap_plan *plan, const void *k_new, const void *v_new,
                              cudaStream_t stream) {
    const cudaError_t e = pool->desc.head_dim == 128 ? append_t<128>(pool, plan, k_new, v_new, stream)
                                                     : append_t<64>(pool, plan, k_new, v_new, stream);
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv_read_new(const ap_kv_pool *pool, const ap_plan *plan, void *k, void *v, cudaStream_t stream) {
    cudaError_t e;
    if (pool->four_bit) {
        e = pool->desc.head_dim == 128 ? read_t<128>(pool, plan, k, v, stream) : read_t<64>(pool, plan, k, v, stream);
    } else {
        const int chunks = pool->desc.head_dim / 8;
        const int64_t n_vec = plan->info.n_new * pool->desc.num_kv_heads * chunks;
        e = launch_overlapped(kv_read_new_kernel, (unsigned)((n_vec + 255) / 256), 256u, 0, stream, (const uint4 *)pool->desc.k_base,
                              (const uint4 *)pool->desc.v_base, (uint4 *)k, (uint4 *)v, plan->d_append_dst, n_vec,
                              pool->desc.num_kv_heads, chunks, pool->desc.num_pages, pool->status_dev);
    }
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv4_widen(const ap_kv_pool *pool, const ap_plan *plan, void *k, void *v, cudaStream_t stream) {
    const cudaError_t e = pool->desc.head_dim == 128 ? widen_t<128>(pool, plan, k, v, stream) : widen_t<64>(pool, plan, k, v, stream);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ap
