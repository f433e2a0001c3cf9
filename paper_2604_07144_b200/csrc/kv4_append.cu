// Appending to, reading back from and widening a 4-bit pool (the format is described in kv4.cuh).  All
// three are single passes over their data, bound by HBM.
#include "internal.h"
#include "kv4.cuh"
#include "ptx.cuh"

namespace ap {

namespace {

// One thread quantises eight elements of K and the matching eight of V; the four lanes of a quad share the
// groups' maxima by shuffle.  Each 16-byte load is followed by one 4-byte store.
template <int D>
__global__ void __launch_bounds__(256) kv4_append_kernel(uint8_t *__restrict__ k_pool, uint8_t *__restrict__ v_pool,
                                                         const uint4 *__restrict__ k_new, const uint4 *__restrict__ v_new,
                                                         const int32_t *__restrict__ append_dst, int64_t n_vec,
                                                         int num_kv_heads, int num_pages, int *status) {
    using T = kv4::Tile<D>;
    constexpr int kChunks = D / 8;
    const int64_t idx = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    const int64_t v = idx < n_vec ? idx : n_vec - 1;      // the shuffles need whole warps; the rest stores nothing
    const int c = (int)(v % kChunks);
    const int64_t rh = v / kChunks;
    const int g = (int)(rh % num_kv_heads);
    const int32_t dst = __ldg(append_dst + rh / num_kv_heads);   // plan data: uploaded before any kernel of the step
    ptx::griddep_launch_dependents();
    ptx::griddep_wait();
    float ks, vs;
    const uint32_t kw = kv4::quantise8(__ldg(k_new + v), ks);
    const uint32_t vw = kv4::quantise8(__ldg(v_new + v), vs);
    const int32_t page = dst >> 4, slot = dst & 15;
    if (idx >= n_vec) return;
    if (page < 0 || page >= num_pages) {
        ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        return;
    }
    const int64_t tile = ((int64_t)page * num_kv_heads + g) * T::kBytes;
    const int word = slot * T::kRowBytes + 4 * kv4::stored_word<D>(c);
    *reinterpret_cast<uint32_t *>(k_pool + tile + word) = kw;
    *reinterpret_cast<uint32_t *>(v_pool + tile + word) = vw;
    if ((c & 3) == 0) {
        const int step = T::kCodeBytes + 2 * (slot * T::kGroups + (c >> 2));
        *reinterpret_cast<uint16_t *>(k_pool + tile + step) = (uint16_t)(__float_as_uint(ks) >> 16);
        *reinterpret_cast<uint16_t *>(v_pool + tile + step) = (uint16_t)(__float_as_uint(vs) >> 16);
    }
}

// Reads the plan's new rows back, [N_new][Hkv][d] bf16: of a 4-bit pool the values it stands for, of a bf16
// pool the values it holds.  One thread per eight elements and plane.
template <int D, bool kFour>
__global__ void __launch_bounds__(256) kv_read_new_kernel(const uint8_t *__restrict__ k_pool, const uint8_t *__restrict__ v_pool,
                                                          uint4 *__restrict__ k_out, uint4 *__restrict__ v_out,
                                                          const int32_t *__restrict__ append_dst, int64_t n_vec,
                                                          int num_kv_heads, int num_pages, int *status) {
    using T = kv4::Tile<D>;
    constexpr int kChunks = D / 8;
    const int64_t v = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    ptx::griddep_launch_dependents();
    if (v >= n_vec) {
        ptx::griddep_wait();
        return;
    }
    const int c = (int)(v % kChunks);
    const int64_t rh = v / kChunks;
    const int g = (int)(rh % num_kv_heads);
    const int32_t dst = __ldg(append_dst + rh / num_kv_heads);
    ptx::griddep_wait();
    const int32_t page = dst >> 4, slot = dst & 15;
    if (page < 0 || page >= num_pages) {
        ptx::record_status(status, AP_ERR_BAD_BLOCK_TABLE);
        return;
    }
    const int64_t tile = (int64_t)page * num_kv_heads + g;
    if constexpr (kFour) {
        const uint8_t *k = k_pool + tile * T::kBytes, *vv = v_pool + tile * T::kBytes;
        const int word = slot * T::kRowBytes + 4 * kv4::stored_word<D>(c);
        const int step = T::kCodeBytes + 2 * (slot * T::kGroups + (c >> 2));
        k_out[v] = kv4::dequantise8(*reinterpret_cast<const uint32_t *>(k + word), *reinterpret_cast<const uint16_t *>(k + step));
        v_out[v] = kv4::dequantise8(*reinterpret_cast<const uint32_t *>(vv + word), *reinterpret_cast<const uint16_t *>(vv + step));
    } else {
        const int64_t o = (tile * kPageSize + slot) * kChunks + c;
        k_out[v] = reinterpret_cast<const uint4 *>(k_pool)[o];
        v_out[v] = reinterpret_cast<const uint4 *>(v_pool)[o];
    }
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
    const int n = num_kv_heads * kPageSize * kChunks;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int c = i % kChunks, row = i / kChunks;
        const uint8_t *tile = src + (row / kPageSize) * T::kBytes;
        const int slot = row % kPageSize;
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t *>(tile + slot * T::kRowBytes) + kv4::stored_word<D>(c));
        const uint16_t s = __ldg(reinterpret_cast<const uint16_t *>(tile + T::kCodeBytes) + slot * T::kGroups + (c >> 2));
        dst[i] = kv4::dequantise8(w, s);
    }
}

template <int D>
cudaError_t append_t(const ap_kv_pool *pool, const ap_plan *plan, const void *k_new, const void *v_new, cudaStream_t stream) {
    const int64_t n_vec = plan->info.n_new * pool->desc.num_kv_heads * (D / 8);
    return launch_overlapped(kv4_append_kernel<D>, (unsigned)((n_vec + 255) / 256), 256u, 0, stream, (uint8_t *)pool->desc.k_base,
                             (uint8_t *)pool->desc.v_base, (const uint4 *)k_new, (const uint4 *)v_new, plan->d_append_dst, n_vec,
                             pool->desc.num_kv_heads, pool->desc.num_pages, pool->status_dev);
}

template <int D, bool kFour>
cudaError_t read_t(const ap_kv_pool *pool, const ap_plan *plan, void *k, void *v, cudaStream_t stream) {
    const int64_t n_vec = plan->info.n_new * pool->desc.num_kv_heads * (D / 8);
    return launch_overlapped(kv_read_new_kernel<D, kFour>, (unsigned)((n_vec + 255) / 256), 256u, 0, stream,
                             (const uint8_t *)pool->desc.k_base, (const uint8_t *)pool->desc.v_base, (uint4 *)k, (uint4 *)v,
                             plan->d_append_dst, n_vec, pool->desc.num_kv_heads, pool->desc.num_pages, pool->status_dev);
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
    if (pool->four_bit)
        e = pool->desc.head_dim == 128 ? read_t<128, true>(pool, plan, k, v, stream) : read_t<64, true>(pool, plan, k, v, stream);
    else
        e = pool->desc.head_dim == 128 ? read_t<128, false>(pool, plan, k, v, stream) : read_t<64, false>(pool, plan, k, v, stream);
    return e != cudaSuccess ? e : cudaGetLastError();
}

cudaError_t launch_kv4_widen(const ap_kv_pool *pool, const ap_plan *plan, void *k, void *v, cudaStream_t stream) {
    const cudaError_t e = pool->desc.head_dim == 128 ? widen_t<128>(pool, plan, k, v, stream) : widen_t<64>(pool, plan, k, v, stream);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace ap
