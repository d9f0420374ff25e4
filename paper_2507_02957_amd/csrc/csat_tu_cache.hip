// Translation unit of the 8-bit key/value cache: store, attention over it, eviction.
#include "csat_cache.h"
#include "csat_launch.h"

namespace csat {

hipError_t cache_store_launch(bool bf16, const StoreArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)((long long)a.B * a.reach * a.Hkv));
    if (bf16) hipLaunchKernelGGL(cache_store_kernel<bf16_t>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(cache_store_kernel<float>, grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

hipError_t cache_attention_launch(bool bf16, const CachedArgs& a, hipStream_t st) {
    auto launch = [&](auto kernel, int lds_bytes) -> hipError_t {
        if (lds_bytes > 64 * 1024) {
            const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
            if (e != hipSuccess) return e;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)a.B * a.shares * a.tiles * a.Hkv)), dim3(256), lds_bytes, st, a);
        return hipGetLastError();
    };
#define CSAT_CACHED(DC_) (bf16 ? launch(cache_attention_kernel<bf16_t, DC_>, cached_lds_bytes<DC_>(a.d)) : launch(cache_attention_kernel<float, DC_>, cached_lds_bytes<DC_>(a.d)))
    if (a.d <= 64) return CSAT_CACHED(1);
    if (a.d <= 128) return CSAT_CACHED(2);
    return CSAT_CACHED(4);
#undef CSAT_CACHED
}

hipError_t cache_join_launch(bool bf16, const JoinArgs& j, const CachedArgs& a, hipStream_t st) {
    const long long o_blocks = (long long)a.B * a.max_q * a.Hq, w_blocks = a.scores ? (long long)a.B * a.Hkv * ((a.c.max_len + 1023) / 1024) : 0;
    const dim3 grid((unsigned)(o_blocks + w_blocks));
    if (bf16) hipLaunchKernelGGL(cache_join_kernel<bf16_t>, grid, dim3(256), 0, st, j, a, (int)o_blocks);
    else hipLaunchKernelGGL(cache_join_kernel<float>, grid, dim3(256), 0, st, j, a, (int)o_blocks);
    return hipGetLastError();
}

hipError_t cache_evict_launch(const EvictArgs& a, int blocks, hipStream_t st) {
    hipLaunchKernelGGL(cache_select_kernel, dim3((unsigned)(a.B * a.Hkv)), dim3(kSelectThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(cache_gather_kernel, dim3((unsigned)((long long)a.B * blocks * a.Hkv)), dim3(256), 0, st, a, blocks);
    return hipGetLastError();
}

}  // namespace csat
