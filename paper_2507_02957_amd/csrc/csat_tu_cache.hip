// Translation unit of the 8-bit key/value cache: store, attention over it, eviction.
#include "csat_cache.h"
#include "csat_launch.h"

namespace csat {

template <typename K, typename... A>
static hipError_t launch(K kernel, dim3 grid, int threads, int lds_bytes, hipStream_t st, A... args) {
    if (lds_bytes > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds_bytes, st, args...);
    return hipGetLastError();
}

hipError_t cache_store_launch(bool bf16, const StoreArgs& a, hipStream_t st) {
    const int items = (a.d * a.c.page / 16 + 255) / 256, lds_bytes = store_lds_bytes(a.d, a.c.page);
    const dim3 grid((unsigned)(a.Hkv * a.reach), (unsigned)a.B);
#define CSAT_STORE(NI_) (bf16 ? launch(cache_store_kernel<bf16_t, NI_>, grid, 256, lds_bytes, st, a) : launch(cache_store_kernel<float, NI_>, grid, 256, lds_bytes, st, a))
    return items <= 1 ? CSAT_STORE(1) : items <= 2 ? CSAT_STORE(2) : items <= 4 ? CSAT_STORE(4) : CSAT_STORE(8);
#undef CSAT_STORE
}

constexpr int kMostBlocks = (1 << 22) - 1;      // of the grid's x; what needs more takes several launches

hipError_t cache_attention_launch(bool bf16, const CachedArgs& all, hipStream_t st) {
    CachedArgs a = all;
    const int most = kMostBlocks / a.Hkv;
    for (int n; a.first_tile < a.tiles; a.first_tile += n) {
        n = a.tiles - a.first_tile < most ? a.tiles - a.first_tile : most;
        const dim3 grid((unsigned)(a.Hkv * n), (unsigned)a.shares, (unsigned)a.B);
#define CSAT_CACHED(T_, DC_, RT_) launch(cache_attention_kernel<T_, DC_, RT_>, grid, 256, cached_lds_bytes<DC_, RT_>(a.d), st, a)
        const hipError_t e = !bf16 ? (a.d <= 64 ? CSAT_CACHED(float, 1, 1) : a.d <= 128 ? CSAT_CACHED(float, 2, 1) : CSAT_CACHED(float, 4, 1))
                             : a.row_tiles == 2 ? (a.d <= 64 ? CSAT_CACHED(bf16_t, 1, 2) : CSAT_CACHED(bf16_t, 2, 2))
                                                : (a.d <= 64 ? CSAT_CACHED(bf16_t, 1, 1) : a.d <= 128 ? CSAT_CACHED(bf16_t, 2, 1) : CSAT_CACHED(bf16_t, 4, 1));
#undef CSAT_CACHED
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t cache_join_launch(bool bf16, const JoinArgs& j, const CachedArgs& a, hipStream_t st) {
    const int o_blocks = join_blocks_per_sequence(a.max_q, a.Hq, a.shares), all = o_blocks + (a.scores ? a.Hkv * ((a.c.max_len + 1023) / 1024) : 0);
    for (int first = 0, n; first < all; first += n) {
        n = all - first < kMostBlocks ? all - first : kMostBlocks;
        const dim3 grid((unsigned)n, (unsigned)a.B);
        const hipError_t e = bf16 ? launch(cache_join_kernel<bf16_t>, grid, 256, 0, st, j, a, o_blocks, first) : launch(cache_join_kernel<float>, grid, 256, 0, st, j, a, o_blocks, first);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t cache_evict_launch(const EvictArgs& a, int blocks, hipStream_t st) {
    const hipError_t e = launch(cache_select_kernel, dim3((unsigned)(a.B * a.Hkv)), kSelectThreads, 0, st, a);
    if (e != hipSuccess) return e;
    const int items = (a.d * a.from.page / 16 + 255) / 256, lds_bytes = gather_pages(a.d, a.from.page) * gather_page_bytes(a.d, a.from.page);
    const dim3 grid((unsigned)(a.Hkv * 2 * blocks), (unsigned)a.B);
#define CSAT_GATHER(NI_) launch(cache_gather_kernel<NI_>, grid, 256, lds_bytes, st, a)
    return items <= 1 ? CSAT_GATHER(1) : items <= 2 ? CSAT_GATHER(2) : items <= 4 ? CSAT_GATHER(4) : CSAT_GATHER(8);
#undef CSAT_GATHER
}

}  // namespace csat
