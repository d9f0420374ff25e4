// Exact attention over packed sequences: O = softmax(scale Q K^T) V per sequence and head, causal or not, several query
// heads to a key head.
//
// Mathematics: one pass over the keys.  A row keeps a reference ref (its running maximum, moved only when a score
// exceeds it by more than 2^8), the sum of its weights e = 2^(s sl + off), off = -ref sl, sl = scale log2(e), and the
// unnormalised output; moving the reference multiplies both by 2^(off' - off), the same rounded offsets that the weights
// were formed with, so the change of reference itself rounds nothing but the product.
// With bf16 tensors the weights go into the second product rounded to bf16, half a step of the output's own type, for one
// matrix instruction in place of two or three; scores, exponentials, sums and outputs are float, and the sum is of the weights as
// they were before the rounding.
//
// Rows: the rows of one key head are the (row, head of the group) pairs, row / G first, so that a workgroup's keys serve all
// heads of the group.  Everything is computed transposed (S^T = K Q^T, O^T = V^T P^T): a query row sits in one lane pair
// and the scores' accumulator layout is the B operand of the second product (K-slot order 4h + {0..3}, 8 + 4h + {0..3}
// in lane half h; V^T comes from the transposing LDS load in the same order).
#pragma once
#include "csat_gemm_f32.h"      // split3
#include "csat_kernels.h"

namespace csat {

// Query heads to a key head; the rows of a key head are its (token, head of the group) pairs.
struct Group {
    int size, shift;               // shift >= 0: size is that power of two
    __host__ __device__ Group(int n = 1) : size(n), shift(-1) {
        for (int k = 0; k < 31; ++k)
            if (n == 1 << k) shift = k;
    }
    __device__ __forceinline__ int token(int r) const { return shift >= 0 ? r >> shift : r / size; }
};

struct PromptArgs {
    const void *Q, *K, *V;
    void* O;
    float* lse;
    const int *q_off, *k_off;
    long long q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
    int B, Hq, Hkv, d, n_q, n_k, max_q, causal;
    Group G;
    float sl;                      // scale log2(e)
    int tiles;                     // row tiles per sequence and key head, up to the end of this launch's
    int pair_groups;               // (sequence, key head) pairs / the grid's x
    int shares;                    // > 1: workgroups that split a row tile's keys, joined by attention_join_kernel
    float* part;                   // [shares][n_q Hq][d] unnormalised outputs, then [shares][n_q Hq][2]: offset, sum
};

constexpr int kPromptWaves = 4;
template <int DT> constexpr int prompt_lds() { return 2 * 2 * 64 * DT * 32 * 2 + 32 * DT * 12 + 16; }      // K and V twice; three keys a column, a word

// One sequence's rows: clamped to the tensors whatever the offsets say.
struct PackedSpan {
    int first, count;
    __device__ __forceinline__ PackedSpan(const int* off, int b, int total) {
        int f = off[b], e = off[b + 1];
        f = f < 0 ? 0 : f > total ? total : f;
        e = e < f ? f : e > total ? total : e;
        first = f;
        count = e - f;
    }
};

// Infinities and NaN in V where some row does not see their key: a weight of 0 times one of them is NaN.  They are taken out
// of the staged tile (only a step with a masked key is looked through) and noted per column, the lowest key of each kind; at
// the end a row that sees that key, as rows see a leading part of the keys, gets what the sum would have been.
struct OddColumn { int nan, pinf, ninf; };
constexpr int kNoKey = 0x7fffffff;
template <typename T> __device__ __forceinline__ uint32_t odd_values(const uint4& w);      // bit e: value e of the piece
template <> __device__ __forceinline__ uint32_t odd_values<bf16_t>(const uint4& w) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = (&w.x)[i];
        m |= ((x & 0x7f80u) == 0x7f80u ? 1u : 0u) << (2 * i) | ((x & 0x7f800000u) == 0x7f800000u ? 1u : 0u) << (2 * i + 1);
    }
    return m;
}
template <> __device__ __forceinline__ uint32_t odd_values<float>(const uint4& w) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) m |= (((&w.x)[i] & 0x7f800000u) == 0x7f800000u ? 1u : 0u) << i;
    return m;
}
template <typename T>
__device__ __forceinline__ void take_odd(uint4* piece, int key, OddColumn* col, int* any) {
    const uint4 w = *piece;
    const uint32_t m = odd_values<T>(w);
    if (m == 0) return;
    *any = 1;
    T* const x = (T*)piece;
    for (int e = 0; e < Elem<T>::per_chunk; ++e) {
        if (!((m >> e) & 1)) continue;
        const float v = Elem<T>::load(x + e);
        atomicMin(v != v ? &col[e].nan : v > 0.f ? &col[e].pinf : &col[e].ninf, key);
        Elem<T>::store(x + e, 0.f);
    }
}
__device__ __forceinline__ float with_odd(float finite, const OddColumn& c, int limit) {
    const bool p = c.pinf < limit, n = c.ninf < limit;
    if (c.nan < limit || (p && n)) return __uint_as_float(0x7fc00000u);
    return p ? finite + INFINITY : n ? finite - INFINITY : finite;
}

// 16 bytes of memory per lane, base + off, to LDS at `at` + 16 lane.  In assembly, so that the compiler, which cannot tell the half
// that is written from the half that is read, does not wait for it before every LDS read: who calls it waits (vmcnt) himself.
__device__ __forceinline__ void stage16(uint32_t at, const char* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" :: "s"(at), "v"(off), "s"(base) : "memory", "m0");
}

__device__ __forceinline__ float pair_max(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

// Swizzles of the staged tiles: 16-byte piece c of row `row` lies at piece c ^ swizzle, C pieces a row, so that 16 rows' pieces of
// K (one fragment read), or 4 rows' 64 bytes of V (half a transposing read; float: 2 rows 4 apart), cover the 64 banks once.
template <int C> __device__ __forceinline__ int swizzle_k(int row) { return C % 16 == 0 ? row & 15 : C % 8 == 0 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <typename T, int C> __device__ __forceinline__ int swizzle_v(int row) {
    if (sizeof(T) == 4) return C % 16 == 0 ? 8 * ((row >> 2) & 1) : 0;
    return C % 16 == 0 ? 4 * (row & 3) : C % 8 == 0 ? 4 * ((row >> 1) & 1) : 0;
}

// Outputs are accumulated before they are divided by the sum, with weights of up to 2^8, so that finite values of V above 2^120 / keys
// may pass the largest float where their mean does not.  Whoever finds outputs at the end whose squares do not add up to a float
// (one of 2^64 or more, or not finite) goes over the keys once more with weights that are smaller by `headroom` powers of two: then
// all together come to half the largest |v| at most, and weights that this makes 0 are below 2^-87 of the row's largest.
__device__ __forceinline__ float headroom(int keys) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint((float)(41 - __builtin_clz(keys | 1))))); }

// What a wavefront accumulates for 32 rows, and what becomes of a tile's scores.
template <int DT>
struct PromptAcc {
    f32x16 o[DT];
    float ref, off, sum;                  // reference score, what a weight's exponent takes off for it, this lane's share of the row's sum
    float down;                           // powers of two that all weights are smaller by (see headroom)
    int lim;                              // keys that the lane's row sees
    __device__ __forceinline__ void clear(float smaller) {
        ref = -INFINITY; off = 0.f; sum = 0.f; down = smaller;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[t][v] = 0.f;
    }
    // scores of KT x 32 keys from key0 on -> weights, what was accumulated brought to their reference
    template <int KT>
    __device__ __forceinline__ void weights(f32x16 (&s)[KT], int key0, bool masked, float sl, int lh) {
        if (masked) {
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (key0 + 32 * u + 8 * (v >> 2) + 4 * lh + (v & 3) >= lim) s[u][v] = -INFINITY;
        }
        float mx = s[0][0];
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[u][v]);
        mx = pair_max(mx);
        if (__builtin_amdgcn_ballot_w64((mx - ref) * sl > 8.f) != 0) {      // (both lanes of a pair agree; -inf against -inf is no)
            // before a row's first score there is nothing to rescale, and no offset that means anything
            const float nm = fmaxf(mx, ref), to = nm == -INFINITY ? 0.f : -nm * sl - down;
            const float f = ref == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(to - off);
            ref = nm;
            off = to;
            sum *= f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[dt][v] *= f;
        }
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                s[u][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][v], sl, off));
                sum += s[u][v];
            }
    }
};

// 32 rows against KT x 32 keys in LDS, on the matrix instruction of the tensors' type.
template <typename T, int DT, int KT>
struct PromptRows : PromptAcc<DT> {
    using PromptAcc<DT>::o;
    static constexpr bool BF = sizeof(T) == 2;
    static constexpr int D = 32 * DT, EPC = Elem<T>::per_chunk, C = D / EPC, NK = C / 2;      // 16-byte pieces of a row, pairs of them
    uint4 qf[NK];

    // row r of key head hk's rows
    __device__ __forceinline__ void init(const PromptArgs& a, int first, int hk, int r, int limit, float down, int lane) {
        const int lh = lane >> 5, dc = a.d / EPC;
        this->clear(down);
        this->lim = limit;
        const int token = a.G.token(r);
        const T* q = (const T*)a.Q + (long long)(first + token) * a.q_token + (long long)(hk * a.G.size + r - token * a.G.size) * a.q_head;
        if (dc == C) {
#pragma unroll
            for (int g = 0; g < NK; ++g) qf[g] = *(const uint4*)(q + (2 * g + lh) * EPC);
        } else {
#pragma unroll
            for (int g = 0; g < NK; ++g) {
                const int c = 2 * g + lh;
                qf[g] = c < dc ? *(const uint4*)(q + c * EPC) : uint4{0u, 0u, 0u, 0u};
            }
        }
    }

    // keys key0 .., K's tile at LDS address sk, V's at sv; masked: some row does not see all of them.  k_read() is called when K's
    // tile has been read, v_needed() before V's is.
    template <typename KRead, typename VNeeded>
    __device__ __forceinline__ void step(uint32_t sk, uint32_t sv, int key0, bool masked, float sl, int lane, KRead k_read, VNeeded v_needed) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
        typedef __attribute__((address_space(3))) const u32x4* lds_u32x4;
        typedef __attribute__((address_space(3))) const float* lds_float;
        const int li = lane & 31, lh = lane >> 5;
        f32x16 s[KT];
#pragma unroll
        for (int u = 0; u < KT; ++u)
#pragma unroll
            for (int v = 0; v < 16; ++v) s[u][v] = 0.f;
#pragma unroll
        for (int g = 0; g < NK; ++g)
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                const u32x4 kf = *(lds_u32x4)(uintptr_t)(sk + (uint32_t)(((32 * u + li) * C + ((2 * g + lh) ^ swizzle_k<C>(li))) * 16));
                mfma_group<T>(__builtin_bit_cast(uint4, kf), qf[g], s[u]);
            }
        k_read();
        this->template weights<KT>(s, key0, masked, sl, lh);
        v_needed();
        // O^T += V^T P^T
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if constexpr (BF) {
                const int l = lane & 15;
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2) {
                    const f32x16& e = s[u];
                    const uint4 pf = uint4{f2bf_pk(e[8 * h2], e[8 * h2 + 1]), f2bf_pk(e[8 * h2 + 2], e[8 * h2 + 3]),
                                           f2bf_pk(e[8 * h2 + 4], e[8 * h2 + 5]), f2bf_pk(e[8 * h2 + 6], e[8 * h2 + 7])};
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        // rows 32 u + 16 h2 + 4 lh + {0..3} and the same + 8, columns 32 dt + 16 (lane / 16 % 2) + {0..15}
                        const int row = 4 * lh + (l >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((l & 3) >> 1);
                        const uint32_t at0 = sv + (uint32_t)((row * C + (c ^ swizzle_v<T, C>(row))) * 16 + (l & 1) * 8);
                        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at0 + (32 * u + 16 * h2) * C * 16));
                        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at0 + (32 * u + 16 * h2 + 8) * C * 16));
                        const uint2 w0 = __builtin_bit_cast(uint2, v0), w1 = __builtin_bit_cast(uint2, v1);
                        mfma_group<T>(uint4{w0.x, w0.y, w1.x, w1.y}, pf, o[dt]);
                    }
                }
            } else {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int row = 4 * lh + (v & 3), c = 8 * dt + (li >> 2);
                        const uint32_t at = sv + (uint32_t)((row * C + (c ^ swizzle_v<T, C>(row))) * 16 + (li & 3) * 4);
                        const float x = *(lds_float)(uintptr_t)(at + (32 * u + 8 * (v >> 2)) * C * 16);
                        o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[u][v], o[dt], 0, 0, 0);
                    }
            }
        }
    }
};

// ... float rows on the bf16 instruction: six products of the operands' three parts (csat_gemm_f32.h) in 6/16 of the float
// instruction's time.  The parts say a value down to 2^-133.  Infinities, and values of V below 2^-109, show in what is accumulated (not
// finite, or not zero and below 2^-90): the workgroup then starts again with the float instruction.  Scores do not show it: values of Q
// and K below 2^-109 count as multiples of 2^-133 (looking the queries over took 0.4 us of the smallest call's 10.6, 4 % of long ones).
template <int DT>
struct PromptRowsParts : PromptAcc<DT> {
    using PromptAcc<DT>::o;
    static constexpr int D = 32 * DT, C = D / 4, NB = D / 16;
    uint4 qp[NB][3];
    __device__ __forceinline__ static void parts(const float (&x)[8], uint4 (&p)[3]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) split3(x[2 * i], x[2 * i + 1], (&p[0].x)[i], (&p[1].x)[i], (&p[2].x)[i]);
    }
    __device__ __forceinline__ static void products(const uint4 (&x)[3], const uint4 (&y)[3], f32x16& acc) {      // small ones first
        mfma_group<bf16_t>(x[1], y[1], acc);
        mfma_group<bf16_t>(x[0], y[2], acc);
        mfma_group<bf16_t>(x[2], y[0], acc);
        mfma_group<bf16_t>(x[0], y[1], acc);
        mfma_group<bf16_t>(x[1], y[0], acc);
        mfma_group<bf16_t>(x[0], y[0], acc);
    }
    __device__ __forceinline__ void init(const PromptArgs& a, int first, int hk, int r, int limit, float down, int lane) {
        const int lh = lane >> 5;
        this->clear(down);
        this->lim = limit;
        const int token = a.G.token(r);
        const float* q = (const float*)a.Q + (long long)(first + token) * a.q_token + (long long)(hk * a.G.size + r - token * a.G.size) * a.q_head;
#pragma unroll
        for (int g = 0; g < NB; ++g) {
            const int f = 16 * g + 8 * lh;
            float x[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (f < a.d) {
                const float4 x0 = *(const float4*)(q + f), x1 = *(const float4*)(q + f + 4);
                x[0] = x0.x; x[1] = x0.y; x[2] = x0.z; x[3] = x0.w; x[4] = x1.x; x[5] = x1.y; x[6] = x1.z; x[7] = x1.w;
            }
            parts(x, qp[g]);
        }
    }
    template <typename KRead, typename VNeeded>
    __device__ __forceinline__ void step(uint32_t sk, uint32_t sv, int key0, bool masked, float sl, int lane, KRead k_read, VNeeded v_needed) {
        typedef __attribute__((address_space(3))) const f32x4* lds_f32x4;
        typedef __attribute__((address_space(3))) const float* lds_float;
        const int li = lane & 31, lh = lane >> 5;
        f32x16 s[1];
#pragma unroll
        for (int v = 0; v < 16; ++v) s[0][v] = 0.f;
#pragma unroll
        for (int g = 0; g < NB; ++g) {
            float x[8];
            uint4 kp[3];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 w = *(lds_f32x4)(uintptr_t)(sk + (uint32_t)((li * C + ((4 * g + 2 * lh + h) ^ swizzle_k<C>(li))) * 16));
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * h + e] = w[e];
            }
            parts(x, kp);
            products(kp, qp[g], s[0]);
        }
        k_read();
        this->template weights<1>(s, key0, masked, sl, lh);
        v_needed();
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
            float x[8];
            uint4 pp[3], vp[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[0][8 * h2 + e];
            parts(x, pp);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int row = 4 * lh + (e & 3), c = 8 * dt + (li >> 2);
                    const uint32_t at = sv + (uint32_t)((row * C + (c ^ swizzle_v<float, C>(row))) * 16 + (li & 3) * 4);
                    x[e] = *(lds_float)(uintptr_t)(at + (16 * h2 + 8 * (e >> 2)) * C * 16);
                }
                parts(x, vp);
                products(vp, pp, o[dt]);
            }
        }
    }
};
template <int DT>
__device__ __forceinline__ bool has_large(const PromptAcc<DT>& a) {
    float squares[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) squares[v & 7] = __builtin_fmaf(a.o[dt][v], a.o[dt][v], squares[v & 7]);
    return !((squares[0] + squares[1]) + (squares[2] + squares[3]) + ((squares[4] + squares[5]) + (squares[6] + squares[7])) < INFINITY);
}
template <int DT>
__device__ __forceinline__ SplitSuspect magnitudes(const PromptAcc<DT>& a) {
    SplitSuspect t;
    t.add(a.sum);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int v = 0; v < 16; ++v) t.add(a.o[dt][v]);
    return t;
}

// A sequence's keys in steps of KEYS: a step's pieces go from memory straight into LDS, piece q of the tile at its place there;
// thread `tid` of THREADS brings the pieces q = THREADS p + tid from the places that the swizzles send there (token strides are
// below 2^24 elements, so 32 bits hold them within a step).  Rows behind the sequence's last one are that one again
// (masked); columns behind d are left out (zeroed beforehand).
template <typename T, int C, int KEYS, int THREADS>
struct PromptKeys {
    static constexpr int PIECES = KEYS * C / THREADS, TILE = KEYS * C * 16;
    static_assert(KEYS * C % THREADS == 0, "a step's pieces are dealt out evenly");
    const char *kb, *vb;
    uint32_t k_row, v_row;
    uint32_t ko[PIECES], vo[PIECES];
    int nk, dc;
    __device__ __forceinline__ PromptKeys(const PromptArgs& a, int first, int count, int hk, int tid) : nk(count), dc(a.d / Elem<T>::per_chunk) {
        kb = (const char*)a.K + ((long long)first * a.k_token + (long long)hk * a.k_head) * (long long)sizeof(T);
        vb = (const char*)a.V + ((long long)first * a.v_token + (long long)hk * a.v_head) * (long long)sizeof(T);
        k_row = (uint32_t)a.k_token * (uint32_t)sizeof(T);
        v_row = (uint32_t)a.v_token * (uint32_t)sizeof(T);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int q = p * THREADS + tid, row = q / C, c = q % C;
            ko[p] = (uint32_t)row * k_row + 16u * (uint32_t)(c ^ swizzle_k<C>(row));
            vo[p] = (uint32_t)row * v_row + 16u * (uint32_t)(c ^ swizzle_v<T, C>(row));
        }
    }
    // step t's tile of K, or of V, to LDS address `at`, PIECES requests of every wavefront; `wave`: which 64 of the threads it is
    template <bool IS_V>
    __device__ __forceinline__ void load(int t, uint32_t at, int wave, int tid) const {
        const uint32_t step_row = IS_V ? v_row : k_row;
        const uint32_t (&off)[PIECES] = IS_V ? vo : ko;
        const char* const from = (IS_V ? vb : kb) + (long long)t * KEYS * step_row;
        at += wave * 1024;
        if (dc == C && (t + 1) * KEYS <= nk) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) stage16(at + p * THREADS * 16, from, off[p]);
            return;
        }
        const int left = nk - 1 - t * KEYS;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {           // (a wavefront's 64 pieces are whole rows: some of its lanes have a column below d)
            const int q = p * THREADS + tid, row = q / C, c = q % C, over = row > left ? row - left : 0;
            if ((c ^ (IS_V ? swizzle_v<T, C>(row) : swizzle_k<C>(row))) < dc) stage16(at + p * THREADS * 16, from, off[p] - (uint32_t)over * step_row);
        }
    }
    // both, V's tile behind K's
    __device__ __forceinline__ void load_both(int t, uint32_t at, int wave, int tid) const {
        load<false>(t, at, wave, tid);
        load<true>(t, at + TILE, wave, tid);
    }
    // zeros where load() leaves out the columns behind d, of `tiles` tiles from `to` (K and V in turn)
    __device__ __forceinline__ void clear(uint4* to, int tiles, int tid) const {
        for (int u = 0; u < tiles; ++u)
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int q = p * THREADS + tid, row = q / C, c = q % C;
                if ((c ^ (u & 1 ? swizzle_v<T, C>(row) : swizzle_k<C>(row))) >= dc) to[u * KEYS * C + q] = uint4{0u, 0u, 0u, 0u};
            }
    }
    // the odd values of V's staged tile (see take_odd)
    __device__ __forceinline__ void look_over(int t, uint4* sv, int tid, OddColumn* oddc, int* any_odd) const {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int q = p * THREADS + tid, row = q / C, c = q % C ^ swizzle_v<T, C>(row);
            take_odd<T>(sv + q, t * KEYS + row, oddc + c * Elem<T>::per_chunk, any_odd);
        }
    }
};
// This wavefront's pieces are there, but for the N that it asked for last (vmcnt(N)).
template <int N = 0> __device__ __forceinline__ void wait_staged() {
    static_assert(N < 64, "vmcnt has six bits");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | (N >> 4) << 14);
    asm volatile("" ::: "memory");
}

// Which rows a workgroup has.  The grid's y is a row tile, the last ones, which see most keys, first.  x is a (sequence, key head)
// pair, z a share of its keys; or, for many tiles, x one of eight pairs and z which eight, so that an XCD, which takes every
// eighth workgroup, works through the tiles of one pair before the next and finds its keys in its L2.
template <int ROWS>
struct PromptPlace {
    int share, b, hk, r_base, rows, r_end, lo, hi, q_first, q_count, k_first, nk, causal;
    Group G;
    __device__ __forceinline__ explicit PromptPlace(const PromptArgs& a) : share(0), causal(a.causal), G(a.G) {
        int pair = blockIdx.x;
        if (a.shares > 1) share = blockIdx.z;
        else pair += gridDim.x * blockIdx.z;
        b = pair / a.Hkv;
        hk = pair - b * a.Hkv;
        const PackedSpan qs(a.q_off, b, a.n_q), ks(a.k_off, b, a.n_k);
        q_first = __builtin_amdgcn_readfirstlane(qs.first); q_count = __builtin_amdgcn_readfirstlane(qs.count);
        k_first = __builtin_amdgcn_readfirstlane(ks.first); nk = __builtin_amdgcn_readfirstlane(ks.count);
        rows = (q_count < a.max_q ? q_count : a.max_q) * G.size;
        r_base = (a.tiles - 1 - (int)blockIdx.y) * ROWS;
        r_end = r_base + ROWS < rows ? r_base + ROWS : rows;
        lo = r_base < rows ? limit(r_base) : 0;
        hi = r_base < rows ? limit(r_end - 1) : 0;
    }
    // this workgroup's steps of the keys, KEYS each
    template <int KEYS>
    __device__ __forceinline__ void steps(int shares, int* t0, int* t1) const {
        const int n = (hi + KEYS - 1) / KEYS;
        *t0 = 0;
        *t1 = n;
        if (shares == 1) return;
        const int per = (int)((uint32_t)(n + shares - 1) / (uint32_t)shares);
        *t0 = share * per < n ? share * per : n;
        *t1 = *t0 + per < n ? *t0 + per : n;
    }
    __device__ __forceinline__ int limit(int r) const {      // keys that row r sees
        if (!causal) return nk;
        const int v = G.token(r) + nk - q_count + 1;
        return v < 0 ? 0 : v > nk ? nk : v;
    }
};

// The second pass for large outputs (headroom), next to never taken, starts from the kernel's arguments as they lie in memory, so that the
// first holds no registers for it (where it did, 96 heads x 274 rows, d 64, took 11.9 us and 32 x 300 11.0; 11.4 and 10.1 so; 11.2 and
// 9.9 without a second pass).
__device__ __forceinline__ void arguments_anew(PromptArgs* to) {
    typedef const uint64_t __attribute__((address_space(4)))* kernarg;
    kernarg from = (kernarg)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(from));
    union Words { PromptArgs a; uint64_t w[sizeof(PromptArgs) / 8]; __device__ Words() {} } u;
    static_assert(sizeof(PromptArgs) % 8 == 0, "whole words");
#pragma unroll
    for (size_t i = 0; i < sizeof(PromptArgs) / 8; ++i) u.w[i] = from[i];
    *to = u.a;
    auto global = [](auto& p) { p = (std::remove_reference_t<decltype(p)>)(const __attribute__((address_space(1))) char*)p; };      // (what a kernel's argument is known to be)
    global(to->Q); global(to->K); global(to->V); global(to->O); global(to->lse); global(to->q_off); global(to->k_off); global(to->part);
}

// Long sequences, bf16: four wavefronts of 32 rows each go over the same keys, 64 at a time, which they stage together, the next step's
// while one is worked on.  Two wavefronts per SIMD fill each other's waits between products (32 a step), exponentials (32 at a
// quarter of the rate) and fragment reads (32 KB a step, at 128 bytes a cycle and CU just below the products' time).
// Measured: 16384 tokens causal, 16 heads over 4 key heads, d 128, 1.03 to 1.06 ms = 1040 to 1070 TFLOP/s of visible pairs, where a library's
// product of two 16384 x 16384 matrices reaches 1400; matrix units busy 43 % of the cycles at 2.4 GHz, vector instructions 40 %, no bank
// conflicts.  With the tiles in staging registers (244 instead of 211) 1.35 ms; with the odd values' products in the loop (410
// registers, one wavefront per SIMD) 2.14.  129 to 256 features have one wavefront per SIMD, whose waits nothing fills: 4 x 2048, 8 heads,
// d 256, 120 us, 570 TFLOP/s.
// One pass over the keys; true: outputs are too large for it (see headroom), and `again` has to be.
template <int DT>
__device__ __forceinline__ bool prompt_pass(const PromptArgs& a, int tid, bool again) {
    typedef bf16_t T;
    typedef PromptRows<T, DT, 2> Rows;
    constexpr int C = Rows::C, D = Rows::D, KEYS = 64, THREADS = 64 * kPromptWaves;
    typedef PromptKeys<T, C, KEYS, THREADS> Keys;
    extern __shared__ uint4 lds[];                  // K tile, V tile; the same once more; then the columns' odd values
    OddColumn* const oddc = (OddColumn*)(lds + 4 * KEYS * C);
    int* const any_odd = (int*)(oddc + D);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;
    const int lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PromptPlace<32 * kPromptWaves> at(a);
    if (at.r_base >= at.rows) return false;
    const int w_base = at.r_base + wave * 32;
    const bool active = w_base < at.rows;
    const int w_end = w_base + 32 < at.rows ? w_base + 32 : at.rows;
    const int w_lo = active ? at.limit(w_base) : 0, w_hi = active ? at.limit(w_end - 1) : 0;
    int t0, t1;
    at.steps<KEYS>(a.shares, &t0, &t1);
    const Keys keys(a, at.k_first, at.nk, at.hk, tid);
    int* const any_large = any_odd + 1;
    Rows rows;
    const bool ok = w_base + li < at.rows;
    const int r = ok ? w_base + li : at.rows - 1;
    if (t0 < t1) keys.load_both(t0, lds0 + (t0 & 1) * 2 * Keys::TILE, wave, tid);
    if (!again) {
        if (keys.dc < C) keys.clear(lds, 4, tid);
        for (int i = tid; i < D; i += THREADS) oddc[i] = OddColumn{kNoKey, kNoKey, kNoKey};
        if (tid == 0) *any_odd = *any_large = 0;
    }
    rows.init(a, at.q_first, at.hk, r, at.limit(r), again ? headroom(at.nk) : 0.f, lane);
    for (int t = t0; t < t1; ++t) {
        const uint32_t sk = lds0 + (t & 1) * 2 * Keys::TILE;
        wait_staged();
        __syncthreads();                             // everybody's pieces are there; the other half of the LDS has been read
        if (t + 1 < t1) keys.load_both(t + 1, lds0 + ((t + 1) & 1) * 2 * Keys::TILE, wave, tid);
        if ((t + 1) * KEYS > at.lo) {                // some row of the workgroup does not see all of the step's keys
            keys.look_over(t, lds + (t & 1) * 2 * KEYS * C + KEYS * C, tid, oddc, any_odd);
            __syncthreads();
        }
        if (t * KEYS >= w_hi) continue;              // (uniform over the wavefront: none of its rows sees these keys)
        rows.step(sk, sk + Keys::TILE, t * KEYS, (t + 1) * KEYS > w_lo, a.sl, lane, [] {}, [] {});
    }
    if (!again && has_large(rows)) *any_large = 1;   // (set up before the first step's barrier)
    __syncthreads();                                 // (the last steps' odd values are noted)
    if (!again && __builtin_expect(*any_large, 0)) return true;
    if (!active) return false;

    const float total = pair_sum(rows.sum);
    const int token = a.G.token(r), head = at.hk * a.G.size + r - token * a.G.size;
    const long long row = at.q_first + token;
    f32x16 (&o)[DT] = rows.o;
    if (*any_odd) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[dt][v] = with_odd(o[dt][v], oddc[32 * dt + 8 * (v >> 2) + 4 * lh + (v & 3)], rows.lim);
    }
    if (a.shares > 1) {
        const long long all = (long long)a.n_q * a.Hq, p0 = (long long)at.share * all + row * a.Hq + head;
        if (!ok) return false;
        float* p = a.part + p0 * a.d;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int col = 32 * dt + 8 * g + 4 * lh;
                if (col < a.d) *(float4*)(p + col) = float4{o[dt][4 * g], o[dt][4 * g + 1], o[dt][4 * g + 2], o[dt][4 * g + 3]};
            }
        if (lh == 0) ((float2*)(a.part + (long long)a.shares * all * a.d))[p0] = float2{total == 0.f ? INFINITY : rows.off, total};
        return false;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;      // (a row that saw nothing is 0)
    if (a.lse && ok && lh == 0) a.lse[(long long)head * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - rows.off);
    T* out = (T*)a.O + row * a.o_token + (long long)head * a.o_head;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
        for (int v = 0; v < 16; ++v) o[dt][v] *= inv;
        // lane (i, h) holds columns 8 g + 4 h .. + 3 of its row: the pair exchanges so that each lane stores 16 bytes
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            const uint32_t a0 = f2bf_pk(o[dt][4 * g], o[dt][4 * g + 1]), a1 = f2bf_pk(o[dt][4 * g + 2], o[dt][4 * g + 3]);
            const uint32_t b0 = f2bf_pk(o[dt][4 * g + 4], o[dt][4 * g + 5]), b1 = f2bf_pk(o[dt][4 * g + 6], o[dt][4 * g + 7]);
            const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
            const auto s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            const int col = 32 * dt + 8 * (g + lh);
            if (ok && col < a.d) *(uint4*)(out + col) = uint4{s0[0], s1[0], s0[1], s1[1]};
        }
    }
    return false;
}
template <int DT>
__global__ __launch_bounds__(64 * kPromptWaves, DT <= 4 ? 2 : 1) void prompt_kernel(PromptArgs a) {
    if (__builtin_expect(!prompt_pass<DT>(a, threadIdx.x, false), 1)) return;
    PromptArgs anew;
    arguments_anew(&anew);
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    prompt_pass<DT>(anew, tid, true);
}

// Few rows, and float tensors of any length: a workgroup has 32 rows, and its wavefronts divide the keys, every W-th 32 of them
// each, in LDS of their own without a barrier, and join their rows at the end.  Float is bound by what a step issues (d 64: 48
// products of 32 cycles, 570 vector instructions, most of them splitting K, V and the weights); for bf16 it is the form
// that spreads little work over the chip.
template <typename T, int DT> constexpr int prompt_split_tile() { return 2 * 32 * 32 * DT * (int)sizeof(T); }      // K and V, 32 keys
// bf16: as many wavefronts as the LDS holds tiles for, up to 8, since a row tile's keys are a chain (2 key heads x 1024 x 4, d 128: 13.4
// against 15.9 us with 4, then; 13.8 now).  Float: 4, so that with up to 64 features two workgroups share a CU's vector units and one fills
// the other's start and end (a clip of 1600 tokens, 12 heads: 40 against 54 us with 8); from 65 on the registers leave one wavefront per
// SIMD (4 x 1024, 8 heads, d 128: 101 us, 85 TFLOP/s), and from 129 on the LDS two per CU, of 512 registers each and
// scratch (156 bytes a lane, 760 with the second pass; 4 x 300, 8 heads, d 256: 88 us, 17 TFLOP/s).
template <typename T, int DT> constexpr int prompt_split_waves() {
    const int most = sizeof(T) == 2 ? 8 : 4;
    return most * prompt_split_tile<T, DT>() <= 128 * 1024 ? most : most / 2;
}
// staging, or the joining rows (float), and per column three keys, a word, per wavefront and row an offset and a sum
template <typename T, int DT> constexpr int prompt_split_lds() {
    return prompt_split_waves<T, DT>() * (prompt_split_tile<T, DT>() + 32 * 8) + 32 * DT * 12 + 16;
}
template <typename T, int DT>
__device__ __forceinline__ bool prompt_split_pass(const PromptArgs& a, int tid, bool again) {      // (as prompt_pass)
    typedef PromptRows<T, DT, 1> Rows;
    constexpr int C = Rows::C, D = Rows::D, KEYS = 32, W = prompt_split_waves<T, DT>(), THREADS = 64 * W;
    typedef PromptKeys<T, C, KEYS, 64> Keys;
    static_assert(2 * Keys::TILE == prompt_split_tile<T, DT>() && 32 * D * 4 <= 2 * Keys::TILE, "a wavefront's rows fit its staging");
    extern __shared__ uint4 lds[];
    OddColumn* const oddc = (OddColumn*)(lds + W * 2 * KEYS * C);
    int* const any_odd = (int*)(oddc + D);
    int* const any_large = any_odd + 1;
    float2* const ml = (float2*)(any_odd + 4);
    const int lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const PromptPlace<32> at(a);
    if (at.r_base >= at.rows) return false;
    int t0, t1;
    at.steps<KEYS>(a.shares, &t0, &t1);
    const Keys keys(a, at.k_first, at.nk, at.hk, lane);
    uint4* const own = lds + wave * 2 * KEYS * C;
    const uint32_t sk = (uint32_t)(uintptr_t)(lds_ptr_t)own;
    if (!again) {
        if (keys.dc < C) keys.clear(own, 2, lane);
        for (int i = tid; i < D; i += THREADS) oddc[i] = OddColumn{kNoKey, kNoKey, kNoKey};
        if (tid == 0) *any_odd = *any_large = 0;
    }
    const int lane_row = at.r_base + li < at.rows ? at.r_base + li : at.rows - 1, lane_limit = at.limit(lane_row);
    PromptAcc<DT> acc;
    auto go = [&](auto rows, float down) {
        // K's tile is asked for again as soon as it has been read, V's too: each has the other's work to arrive in.  (A wavefront
        // has 64 lanes' part in every request, so PIECES requests are one tile.)
        if (t0 + wave < t1) keys.load_both(t0 + wave, sk, 0, lane);
        rows.init(a, at.q_first, at.hk, lane_row, lane_limit, down, lane);
        __syncthreads();                             // (the columns' odd values are set up)
        for (int t = t0 + wave; t < t1; t += W) {
            const bool masked = (t + 1) * KEYS > at.lo, more = t + W < t1;
            wait_staged<Keys::PIECES>();             // K's
            rows.step(sk, sk + Keys::TILE, t * KEYS, masked, a.sl, lane, [&] {
                __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the tile has been read
                if (more) keys.template load<false>(t + W, sk, 0, lane);
            }, [&] {
                if (more) wait_staged<Keys::PIECES>();
                else wait_staged();
                if (masked) keys.look_over(t, own + KEYS * C, lane, oddc, any_odd);
                __builtin_amdgcn_wave_barrier();
            });
            __builtin_amdgcn_s_waitcnt(0xc07f);
            __builtin_amdgcn_wave_barrier();
            if (more) keys.template load<true>(t + W, sk + Keys::TILE, 0, lane);
        }
        acc = rows;
    };
    if constexpr (Rows::BF || DT > 4) {              // (256 features in three parts do not fit the registers)
        go(Rows{}, again ? headroom(at.nk) : 0.f);
        if (!again && has_large(acc)) *any_large = 1;
    } else {
        go(PromptRowsParts<DT>{}, 0.f);
        const SplitSuspect seen = magnitudes(acc);
        const bool large = seen.high >= 2 * __float_as_uint(0x1p64f);
        if (__syncthreads_or(large || seen.any())) go(Rows{}, __syncthreads_or(large) ? headroom(at.nk) : 0.f);
    }
    // the wavefronts' parts of a row, brought to the smallest offset
    const float sum = pair_sum(acc.sum);
    if (lh == 0) ml[wave * 32 + li] = float2{sum == 0.f ? INFINITY : acc.off, sum};
    __syncthreads();                                 // (staging is free, odd values are noted)
    if (!again && __builtin_expect(*any_large, 0)) return true;
    float* const joint = (float*)lds;
    {
        float off = INFINITY;
#pragma unroll
        for (int w = 0; w < W; ++w) off = fminf(off, ml[w * 32 + li].x);
        const float f = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(off - acc.off);
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f32x16& o = acc.o[dt];
                *(float4*)(joint + (wave * 32 + li) * D + ((32 * dt + 8 * g + 4 * lh) ^ (4 * (li & 7)))) =
                    float4{f * o[4 * g], f * o[4 * g + 1], f * o[4 * g + 2], f * o[4 * g + 3]};
            }
    }
    __syncthreads();
    const int n = at.r_end - at.r_base, dq = a.d / 4;
    const bool odd = *any_odd != 0;
    for (int q = tid; q < n * dq; q += THREADS) {
        const int i = q / dq, c = q % dq * 4, r = at.r_base + i, token = a.G.token(r), head = at.hk * a.G.size + r - token * a.G.size;
        const long long row = at.q_first + token;
        float off = INFINITY, total = 0.f;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < W; ++w) off = fminf(off, ml[w * 32 + i].x);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float2 y = ml[w * 32 + i];
            if (y.y != 0.f) total += __builtin_amdgcn_exp2f(off - y.x) * y.y;
            const float4 z = *(const float4*)(joint + (w * 32 + i) * D + (c ^ (4 * (i & 7))));
            x[0] += z.x; x[1] += z.y; x[2] += z.z; x[3] += z.w;
        }
        if (odd) {
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = with_odd(x[e], oddc[c + e], at.limit(r));
        }
        if (a.shares > 1) {
            const long long all = (long long)a.n_q * a.Hq, p0 = (long long)at.share * all + row * a.Hq + head;
            *(float4*)(a.part + p0 * a.d + c) = float4{x[0], x[1], x[2], x[3]};
            if (c == 0) ((float2*)(a.part + (long long)a.shares * all * a.d))[p0] = float2{total == 0.f ? INFINITY : off, total};
            continue;
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        if (a.lse && c == 0) a.lse[(long long)head * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - off);
        T* out = (T*)a.O + row * a.o_token + (long long)head * a.o_head + c;
        if constexpr (Rows::BF) *(uint2*)out = uint2{f2bf_pk(x[0] * inv, x[1] * inv), f2bf_pk(x[2] * inv, x[3] * inv)};
        else *(float4*)out = float4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
    }
    return false;
}
template <typename T, int DT>
__global__ __launch_bounds__((64 * prompt_split_waves<T, DT>())) void prompt_split_kernel(PromptArgs a) {
    if (__builtin_expect(!prompt_split_pass<T, DT>(a, threadIdx.x, false), 1)) return;
    if constexpr (sizeof(T) == 2 || DT > 4) {        // (the others have been over their keys once more themselves)
        PromptArgs anew;
        arguments_anew(&anew);
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));
        prompt_split_pass<T, DT>(anew, tid, true);
    }
}

// Shares of a row's keys -> the row: offsets brought to the smallest, outputs and sums added, a workgroup's wavefronts every fourth
// share each and then in order.  One workgroup per row of many shares.
struct JoinArgs {
    const float* part;             // [shares][n_q Hq][d], then [shares][n_q Hq][2]: offset (+inf: nothing seen), sum
    void* O;
    float* lse;
    const int* q_off;
    long long o_token, o_head;
    int B, Hq, d, n_q, max_q, shares;
    const int* lengths;            // the sequences' keys, where a share is `share_keys` of them and a sequence has only those it needs; or null
    int share_keys, max_len;
};
__device__ __forceinline__ int shares_of(const int* lengths, int b, int share_keys, int max_len, int shares) {
    if (!lengths) return shares;
    const int L = lengths[b];
    return L <= 0 || L > max_len ? 1 : (L + share_keys - 1) / share_keys;
}

constexpr int kJoinAhead = 8;      // shares whose outputs a wavefront has in flight
template <typename T>
__device__ __forceinline__ void join_row(const JoinArgs& a, int b, int r) {
    __shared__ float4 outs[4][64];
    __shared__ float sums[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const PackedSpan qs(a.q_off, b, a.n_q);
    const int tok = r / a.Hq, head = r % a.Hq;
    if (tok >= (qs.count < a.max_q ? qs.count : a.max_q)) return;
    const int shares = shares_of(a.lengths, b, a.share_keys, a.max_len, a.shares);
    const long long row = qs.first + tok, all = (long long)a.n_q * a.Hq, at = row * a.Hq + head;
    const float2* ml = (const float2*)(a.part + (long long)a.shares * all * a.d) + at;
    const bool cols = 4 * lane < a.d;
    const float* const p = a.part + at * a.d + 4 * lane;
    float4 x[kJoinAhead];                            // a wavefront's next shares: asked for before their weights are known
    float2 y[kJoinAhead];
    auto ask = [&](int s0) {
#pragma unroll
        for (int i = 0; i < kJoinAhead; ++i) {
            const int s = s0 + 4 * i;
            y[i] = s < shares ? ml[(long long)s * all] : float2{INFINITY, 0.f};
            x[i] = s < shares && cols ? *(const float4*)(p + (long long)s * all * a.d) : float4{0.f, 0.f, 0.f, 0.f};
        }
    };
    ask(wave);
    float off = INFINITY, odd = 0.f;
    for (int s = lane; s < shares; s += 64) {
        const float v = ml[(long long)s * all].x;
        off = fminf(off, v);
        if (v != v) odd = v;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) off = fminf(off, __shfl_xor(off, s));
    if (__ballot(odd != odd) != 0) odd = __uint_as_float(0x7fc00000u);
    float total = odd;
    float4 o = float4{odd, odd, odd, odd};           // columns 4 lane .. + 3
    for (int s0 = wave; s0 < shares; s0 += 4 * kJoinAhead) {
        if (s0 != wave) ask(s0);
#pragma unroll
        for (int i = 0; i < kJoinAhead; ++i) {
            if (y[i].x == INFINITY) continue;
            const float f = __builtin_amdgcn_exp2f(off - y[i].x);
            total += f * y[i].y;
            o.x += f * x[i].x; o.y += f * x[i].y; o.z += f * x[i].z; o.w += f * x[i].w;
        }
    }
    outs[wave][lane] = o;
    if (lane == 0) sums[wave] = total;
    __syncthreads();
    if (wave != 0) return;
    total = sums[0] + sums[1] + sums[2] + sums[3];
#pragma unroll
    for (int w = 1; w < 4; ++w) {
        const float4 x = outs[w][lane];
        o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (a.lse && lane == 0) a.lse[(long long)head * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - off);
    if (!cols) return;
    T* out = (T*)a.O + row * a.o_token + (long long)head * a.o_head + 4 * lane;
    if constexpr (sizeof(T) == 2) *(uint2*)out = uint2{f2bf_pk(o.x * inv, o.y * inv), f2bf_pk(o.z * inv, o.w * inv)};
    else *(float4*)out = float4{o.x * inv, o.y * inv, o.z * inv, o.w * inv};
}
// ... of few shares: one wavefront per row.
constexpr int kJoinFew = 8;
template <typename T>
__device__ __forceinline__ void join_row_few(const JoinArgs& a, int b, int r) {
    const int lane = threadIdx.x & 63;
    const PackedSpan qs(a.q_off, b, a.n_q);
    const int tok = r / a.Hq, head = r % a.Hq;
    if (tok >= (qs.count < a.max_q ? qs.count : a.max_q)) return;
    const int shares = shares_of(a.lengths, b, a.share_keys, a.max_len, a.shares);
    const long long row = qs.first + tok, all = (long long)a.n_q * a.Hq, at = row * a.Hq + head;
    const float2* ml = (const float2*)(a.part + (long long)a.shares * all * a.d) + at;
    const bool cols = 4 * lane < a.d;
    const float* const p = a.part + at * a.d + 4 * lane;
    float4 x[kJoinFew];
    float2 y[kJoinFew];
    float off = INFINITY, total = 0.f;
#pragma unroll
    for (int s = 0; s < kJoinFew; ++s) {
        y[s] = s < shares ? ml[(long long)s * all] : float2{INFINITY, 0.f};
        x[s] = s < shares && cols ? *(const float4*)(p + (long long)s * all * a.d) : float4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int s = 0; s < kJoinFew; ++s) off = fminf(off, y[s].x);
    float4 o = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < kJoinFew; ++s) {
        if (y[s].x == INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(off - y[s].x);      // (an offset that is NaN stays one)
        total += f * y[s].y;
        o.x += f * x[s].x; o.y += f * x[s].y; o.z += f * x[s].z; o.w += f * x[s].w;
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (a.lse && lane == 0) a.lse[(long long)head * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - off);
    if (!cols) return;
    T* out = (T*)a.O + row * a.o_token + (long long)head * a.o_head + 4 * lane;
    if constexpr (sizeof(T) == 2) *(uint2*)out = uint2{f2bf_pk(o.x * inv, o.y * inv), f2bf_pk(o.z * inv, o.w * inv)};
    else *(float4*)out = float4{o.x * inv, o.y * inv, o.z * inv, o.w * inv};
}
// the workgroups that a sequence's rows need, and which a workgroup has
__host__ __device__ inline int join_blocks_per_sequence(int max_q, int Hq, int shares) { return shares <= kJoinFew ? (max_q * Hq + 3) / 4 : max_q * Hq; }
template <typename T>
__device__ __forceinline__ void join_block(const JoinArgs& a, int b, int block) {
    if (a.shares <= kJoinFew) join_row_few<T>(a, b, 4 * block + (threadIdx.x >> 6));
    else join_row<T>(a, b, block);
}
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(JoinArgs a) { join_block<T>(a, blockIdx.y, blockIdx.x); }

}  // namespace csat
