// Prefill-chunk attention kernel (tcgen05 / tensor memory) and its launcher; the device code is in
// prefill_tcgen05.cuh.
#include "prefill_tcgen05.cuh"

namespace ap {

namespace {

using namespace prefill;

template <int D, bool kWin>
__global__ void __launch_bounds__(kPrefillThreads, 1)
prefill_tcgen05_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                       const __grid_constant__ CUtensorMap v_map, const PrefillTile *__restrict__ tiles,
                       const int32_t *__restrict__ bt_flat, __nv_bfloat16 *__restrict__ out,
                       float *__restrict__ lse_out, int Hq, int Hkv, int num_pages, float scale_log2, int *status,
                       uint64_t wait_limit_ns, int window, int sinks) {
    prefill_unit<D, kWin>(q_map, k_map, v_map, tiles, bt_flat, out, lse_out, Hq, Hkv, num_pages, scale_log2, status, wait_limit_ns,
                    (int)blockIdx.x, window, sinks);
}

template <int D, bool kWin>
cudaError_t launch_prefill_t(const ap_kv_pool *pool, const ap_plan *plan, const void *q, void *out, float *lse,
                             const CUtensorMap &k_map, const CUtensorMap &v_map, int num_pages, cudaStream_t stream) {
    using Cfg = PrefillCfg<D>;
    static bool configured[64] = {};
    const int dev = pool->desc.device & 63;
    if (!configured[dev]) {
        cudaError_t e = cudaFuncSetAttribute(prefill_tcgen05_kernel<D, kWin>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             Cfg::kSmemBytes);
        if (e != cudaSuccess) return e;
        configured[dev] = true;
    }
    CUtensorMap q_map;
    if (encode_q_tensor_map(&q_map, q, plan->info.n_new, plan->num_q_heads, D) != AP_OK) return cudaErrorInvalidValue;
    const float scale_log2 = plan->scale * 1.4426950408889634f;
    cudaError_t e = launch_overlapped(
        prefill_tcgen05_kernel<D, kWin>, (unsigned)plan->info.prefill_tiles, (unsigned)kPrefillThreads,
        (size_t)Cfg::kSmemBytes, stream, q_map, k_map, v_map, plan->d_tiles, plan->d_bt_flat,
        (__nv_bfloat16 *)out, lse, plan->num_q_heads, pool->desc.num_kv_heads, num_pages, scale_log2,
        pool->status_dev, pool->wait_limit_ns, plan->window > 0 ? plan->window : 1 << 30, plan->sinks);
    return e != cudaSuccess ? e : cudaGetLastError();
}

}  // namespace

cudaError_t launch_prefill(const ap_kv_pool *pool, const ap_plan *plan, const void *q, void *out, float *lse,
                           const CUtensorMap &k_map, const CUtensorMap &v_map, int num_pages, cudaStream_t stream) {
    // A plan without a window keeps a kernel without the window's tests.  (On a 4-bit pool it takes the windowed one, with
    // a window that no context fills, for its finer exponential.)
    if (plan->window > 0 || pool->four_bit) {
        if (pool->desc.head_dim == 128) return launch_prefill_t<128, true>(pool, plan, q, out, lse, k_map, v_map, num_pages, stream);
        return launch_prefill_t<64, true>(pool, plan, q, out, lse, k_map, v_map, num_pages, stream);
    }
    if (pool->desc.head_dim == 128) return launch_prefill_t<128, false>(pool, plan, q, out, lse, k_map, v_map, num_pages, stream);
    return launch_prefill_t<64, false>(pool, plan, q, out, lse, k_map, v_map, num_pages, stream);
}

}  // namespace ap
