// Translation unit of the exact attention over packed sequences for one element type: compile with -DCSAT_TU_BF16=<0|1>.
#include "csat_prompt.h"
#include "csat_launch.h"

#ifndef CSAT_TU_BF16
#error "compile with -DCSAT_TU_BF16=<0|1>"
#endif

namespace csat {

#if CSAT_TU_BF16
typedef bf16_t T;
#define CSAT_TU_FN(name) name##_bf16
#else
typedef float T;
#define CSAT_TU_FN(name) name##_f32
#endif

hipError_t CSAT_TU_FN(prompt_launch)(const PromptArgs& a, bool split, hipStream_t st) {
    auto launch = [&](auto kernel, int threads, int lds_bytes) -> hipError_t {
        if (lds_bytes > 64 * 1024) {
            const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds_bytes);
            if (e != hipSuccess) return e;
        }
        // (the grid's y holds 65535 tiles; the last ones, the longest, first)
        PromptArgs part = a;
        for (int n; part.tiles > 0; part.tiles -= n) {
            n = part.tiles < 65535 ? part.tiles : 65535;
            hipLaunchKernelGGL(kernel, dim3((unsigned)(a.B * a.Hkv / a.pair_groups), (unsigned)n, (unsigned)(a.shares > 1 ? a.shares : a.pair_groups)), dim3(threads), lds_bytes, st, part);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    };
#if CSAT_TU_BF16
#define CSAT_PROMPT(DT_) (split ? launch(prompt_split_kernel<T, DT_>, 64 * prompt_split_waves<T, DT_>(), prompt_split_lds<T, DT_>()) \
                                : launch(prompt_kernel<DT_>, 64 * kPromptWaves, prompt_lds<DT_>()))
#else
#define CSAT_PROMPT(DT_) launch(prompt_split_kernel<T, DT_>, 64 * prompt_split_waves<T, DT_>(), prompt_split_lds<T, DT_>())
#endif
    if (a.d <= 64) return CSAT_PROMPT(2);
    if (a.d <= 96) return CSAT_PROMPT(3);
    if (a.d <= 128) return CSAT_PROMPT(4);
    return CSAT_PROMPT(8);
#undef CSAT_PROMPT
}

hipError_t CSAT_TU_FN(attention_join_launch)(const JoinArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(attention_join_kernel<T>, dim3((unsigned)join_blocks_per_sequence(a.max_q, a.Hq, a.shares), (unsigned)a.B), dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace csat
