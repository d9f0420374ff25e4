// Exact attention over packed sequences: O = softmax(scale Q K^T) V per sequence and head, causal or not, several query
// heads to a key head.
//
// Mathematics: one pass over the keys.  A row keeps a reference ref (its running maximum, moved only when a score
// exceeds it by more than 2^8), the sum of its weights e = 2^(s sl + off), off = -ref sl, sl = scale log2(e), and the
// unnormalised output; moving the reference multiplies both by 2^(off' - off), the same rounded offsets that the weights
// were formed with, so the change of reference itself rounds nothing but the product.
//
// Rows: the rows of one key head are the (row, head of the group) pairs, row / G first, so that a workgroup's keys serve all
// heads of the group.  Everything is computed transposed (S^T = K Q^T, O^T = V^T P^T): a query row sits in one lane pair
// and the scores' accumulator layout is the B operand of the second product (K-slot order 4h + {0..3}, 8 + 4h + {0..3}
// in lane half h; V^T comes from the transposing LDS load in the same order).
#pragma once
#include "csat_kernels.h"

namespace csat {

struct PromptArgs {
    const void *Q, *K, *V;
    void* O;
    float* lse;
    const int *q_off, *k_off;
    long long q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;
    int B, Hq, Hkv, G, d, n_q, n_k, max_q, causal;
    float sl;                      // scale log2(e)
    int tiles;                     // row tiles per sequence and key head
    int shares;                    // > 1: workgroups that split a row tile's keys, joined by prompt_join_kernel
    float* part;                   // [shares][n_q Hq][d] unnormalised outputs, then [shares][n_q Hq][2]: offset, sum
};

constexpr int kPromptWaves = 4;
template <typename T> constexpr int prompt_key_tiles() { return sizeof(T) == 2 ? 2 : 1; }      // 32-key tiles per step
template <typename T, int DT> constexpr int prompt_lds_bytes() {
    return 2 * 2 * prompt_key_tiles<T>() * 32 * DT * 32 * (int)sizeof(T) + 32 * DT * 12 + 16;      // K and V twice; three keys a column, a word
}

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

template <typename T, int DT, int NT>
__global__ __launch_bounds__(64 * kPromptWaves, NT == 1 && DT <= 4 ? 2 : 1) void prompt_kernel(PromptArgs a) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    typedef __attribute__((address_space(3))) const u32x4* lds_u32x4;
    typedef __attribute__((address_space(3))) const float* lds_float;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KT = prompt_key_tiles<T>(), KEYS = 32 * KT, D = 32 * DT, THREADS = 64 * kPromptWaves;
    constexpr int EPC = Elem<T>::per_chunk, C = D / EPC, NK = C / 2;      // 16-byte pieces of a row, pairs of them
    constexpr int PIECES = KEYS * C / THREADS, TILE = KEYS * C * 16;
    static_assert(KEYS * C % THREADS == 0, "a step's pieces are dealt out evenly");
    extern __shared__ uint4 lds[];                  // K tile, V tile; the same once more; then the columns' odd values
    OddColumn* const oddc = (OddColumn*)(lds + 4 * KEYS * C);
    int* const any_odd = (int*)(oddc + D);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)lds;

    const int tid = threadIdx.x, lane = tid & 63, li = lane & 31, lh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the last row tiles, which see most keys, first; neighbouring workgroups take different heads, so an XCD's keep to a
    // share of the heads where their number is a multiple of eight
    const int P = a.B * a.Hkv;
    const int share = blockIdx.x / (P * a.tiles), id = blockIdx.x % (P * a.tiles);
    const int pair = id % P, tile = a.tiles - 1 - id / P;
    const int b = pair / a.Hkv, hk = pair % a.Hkv;
    const PackedSpan qs(a.q_off, b, a.n_q), ks(a.k_off, b, a.n_k);
    const int nk = ks.count, rows = (qs.count < a.max_q ? qs.count : a.max_q) * a.G;
    const int r_base = tile * (32 * NT * kPromptWaves);
    if (r_base >= rows) return;
    auto limit_of = [&](int r) {      // keys that row r sees
        if (!a.causal) return nk;
        const int v = r / a.G + nk - qs.count + 1;
        return v < 0 ? 0 : v > nk ? nk : v;
    };
    const int r_end = r_base + 32 * NT * kPromptWaves < rows ? r_base + 32 * NT * kPromptWaves : rows;
    const int lo = limit_of(r_base), hi = limit_of(r_end - 1);
    const int steps = (hi + KEYS - 1) / KEYS;
    const int t0 = (int)((long long)steps * share / a.shares), t1 = (int)((long long)steps * (share + 1) / a.shares);

    // this wavefront's rows
    const int w_base = r_base + wave * 32 * NT;
    const bool active = w_base < rows;
    const int w_end = w_base + 32 * NT < rows ? w_base + 32 * NT : rows;
    const int w_lo = active ? limit_of(w_base) : 0, w_hi = active ? limit_of(w_end - 1) : 0;
    int lim[NT];
    uint4 qf[NT][NK];
    const int dc = a.d / EPC;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int r = w_base + 32 * n + li;
        if (r >= rows) r = rows - 1;
        lim[n] = limit_of(r);
        const T* q = (const T*)a.Q + (long long)(qs.first + r / a.G) * a.q_token + (long long)(hk * a.G + r % a.G) * a.q_head;
#pragma unroll
        for (int g = 0; g < NK; ++g) {
            const int c = 2 * g + lh;
            qf[n][g] = c < dc ? *(const uint4*)(q + c * EPC) : uint4{0u, 0u, 0u, 0u};
        }
    }
    f32x16 o[NT][DT];
    float ref[NT], off[NT], sum[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        ref[n] = -INFINITY; off[n] = 0.f; sum[n] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[n][t][v] = 0.f;
    }
    for (int i = tid; i < D; i += THREADS) oddc[i] = OddColumn{kNoKey, kNoKey, kNoKey};
    if (tid == 0) *any_odd = 0;

    // A step's pieces go from memory straight into LDS, piece q of the tile at its place there; a thread's pieces q = 256 p + tid
    // come from the places that the swizzles send there (token strides are below 2^24 elements, so 32 bits hold them within a
    // step).  Rows behind the sequence's last one are that one again (masked); columns behind d are zeroed once and left out.
    const char* const kb = (const char*)a.K + ((long long)ks.first * a.k_token + (long long)hk * a.k_head) * (long long)sizeof(T);
    const char* const vb = (const char*)a.V + ((long long)ks.first * a.v_token + (long long)hk * a.v_head) * (long long)sizeof(T);
    const uint32_t k_row = (uint32_t)a.k_token * (uint32_t)sizeof(T), v_row = (uint32_t)a.v_token * (uint32_t)sizeof(T);
    uint32_t ko[PIECES], vo[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const int q = p * THREADS + tid, row = q / C, c = q % C;
        ko[p] = (uint32_t)row * k_row + 16u * (uint32_t)(c ^ swizzle_k<C>(row));
        vo[p] = (uint32_t)row * v_row + 16u * (uint32_t)(c ^ swizzle_v<T, C>(row));
    }
    if (dc < C)
        for (int i = tid; i < 4 * KEYS * C; i += THREADS) lds[i] = uint4{0u, 0u, 0u, 0u};
    auto load = [&](int t) {
        const char* const kt = kb + (long long)t * KEYS * k_row;
        const char* const vt = vb + (long long)t * KEYS * v_row;
        const uint32_t at = lds0 + (t & 1) * 2 * TILE + wave * 1024;
        if (dc == C && (t + 1) * KEYS <= nk) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) stage16(at + p * THREADS * 16, kt, ko[p]);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) stage16(at + TILE + p * THREADS * 16, vt, vo[p]);
            return;
        }
        const int left = nk - 1 - t * KEYS;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int q = p * THREADS + tid, row = q / C, c = q % C, over = row > left ? row - left : 0;
            if ((c ^ swizzle_k<C>(row)) < dc) stage16(at + p * THREADS * 16, kt, ko[p] - (uint32_t)over * k_row);
            if ((c ^ swizzle_v<T, C>(row)) < dc) stage16(at + TILE + p * THREADS * 16, vt, vo[p] - (uint32_t)over * v_row);
        }
    };
    __syncthreads();                                 // (the zeroed columns, and the columns' odd values are set up)
    if (t0 < t1) load(t0);
    for (int t = t0; t < t1; ++t) {
        const uint32_t sk = lds0 + (t & 1) * 2 * TILE, sv = sk + TILE;
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): this thread's pieces are there
        __syncthreads();                             // ... and everybody's; the other half of the LDS has been read
        if (t + 1 < t1) load(t + 1);
        if ((t + 1) * KEYS > lo) {                   // some row of the workgroup does not see all of the step's keys
            uint4* const wv = lds + (t & 1) * 2 * KEYS * C + KEYS * C;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const int q = p * THREADS + tid, row = q / C, c = q % C ^ swizzle_v<T, C>(row);
                take_odd<T>(wv + q, t * KEYS + row, oddc + c * EPC, any_odd);
            }
            __syncthreads();
        }
        if (t * KEYS >= w_hi) continue;              // (uniform over the wavefront: none of its rows sees these keys)

        f32x16 s[NT][KT];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) s[n][u][v] = 0.f;
#pragma unroll
        for (int g = 0; g < NK; ++g)
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                const u32x4 kf = *(lds_u32x4)(uintptr_t)(sk + (uint32_t)(((32 * u + li) * C + ((2 * g + lh) ^ swizzle_k<C>(li))) * 16));
#pragma unroll
                for (int n = 0; n < NT; ++n) mfma_group<T>(__builtin_bit_cast(uint4, kf), qf[n][g], s[n][u]);
            }
        if ((t + 1) * KEYS > w_lo) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int u = 0; u < KT; ++u)
#pragma unroll
                    for (int v = 0; v < 16; ++v)
                        if (t * KEYS + 32 * u + 8 * (v >> 2) + 4 * lh + (v & 3) >= lim[n]) s[n][u][v] = -INFINITY;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float mx = s[n][0][0];
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) mx = fmaxf(mx, s[n][u][v]);
            mx = pair_max(mx);
            if (__builtin_amdgcn_ballot_w64((mx - ref[n]) * a.sl > 8.f) != 0) {      // (both lanes of a pair agree; -inf against -inf is no)
                // before a row's first score there is nothing to rescale, and no offset that means anything
                const float nm = fmaxf(mx, ref[n]), to = nm == -INFINITY ? 0.f : -nm * a.sl;
                const float f = ref[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(to - off[n]);
                ref[n] = nm;
                off[n] = to;
                sum[n] *= f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int v = 0; v < 16; ++v) o[n][dt][v] *= f;
            }
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    s[n][u][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][u][v], a.sl, off[n]));
                    sum[n] += s[n][u][v];
                }
        }
        // O^T += V^T P^T
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            if constexpr (BF) {
                const int l = lane & 15;
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2) {
                    uint4 pf[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const f32x16& e = s[n][u];
                        pf[n] = uint4{f2bf_pk(e[8 * h2], e[8 * h2 + 1]), f2bf_pk(e[8 * h2 + 2], e[8 * h2 + 3]),
                                      f2bf_pk(e[8 * h2 + 4], e[8 * h2 + 5]), f2bf_pk(e[8 * h2 + 6], e[8 * h2 + 7])};
                    }
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        // rows 32 u + 16 h2 + 4 lh + {0..3} and the same + 8, columns 32 dt + 16 (lane / 16 % 2) + {0..15}
                        const int row = 4 * lh + (l >> 2), c = 4 * dt + 2 * ((lane >> 4) & 1) + ((l & 3) >> 1);
                        const uint32_t at0 = sv + (uint32_t)((row * C + (c ^ swizzle_v<T, C>(row))) * 16 + (l & 1) * 8);
                        const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at0 + (32 * u + 16 * h2) * C * 16));
                        const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(uintptr_t)(at0 + (32 * u + 16 * h2 + 8) * C * 16));
                        const uint2 w0 = __builtin_bit_cast(uint2, v0), w1 = __builtin_bit_cast(uint2, v1);
#pragma unroll
                        for (int n = 0; n < NT; ++n) mfma_group<T>(uint4{w0.x, w0.y, w1.x, w1.y}, pf[n], o[n][dt]);
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
#pragma unroll
                        for (int n = 0; n < NT; ++n) o[n][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[n][u][v], o[n][dt], 0, 0, 0);
                    }
            }
        }
    }
    __syncthreads();                                 // (the last steps' odd values are noted)
    if (!active) return;
    const bool odd = *any_odd != 0;

#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float total = pair_sum(sum[n]);
        const int r = w_base + 32 * n + li;
        const bool ok = r < rows;
        const int rr = ok ? r : rows - 1, head = hk * a.G + rr % a.G;
        const long long row = qs.first + rr / a.G;
        if (odd) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[n][dt][v] = with_odd(o[n][dt][v], oddc[32 * dt + 8 * (v >> 2) + 4 * lh + (v & 3)], lim[n]);
        }
        if (a.shares > 1) {
            const long long all = (long long)a.n_q * a.Hq, at = (long long)share * all + row * a.Hq + head;
            if (ok) {
                float* p = a.part + at * a.d;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int col = 32 * dt + 8 * g + 4 * lh;
                        if (col < a.d) *(float4*)(p + col) = float4{o[n][dt][4 * g], o[n][dt][4 * g + 1], o[n][dt][4 * g + 2], o[n][dt][4 * g + 3]};
                    }
                float2* ml = (float2*)(a.part + (long long)a.shares * all * a.d) + at;
                if (lh == 0) *ml = float2{total == 0.f ? INFINITY : off[n], total};
            }
            continue;
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;      // (a row that saw nothing is 0)
        if (a.lse && ok && lh == 0) a.lse[(long long)head * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - off[n]);
        T* out = (T*)a.O + row * a.o_token + (long long)head * a.o_head;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
            for (int v = 0; v < 16; ++v) o[n][dt][v] *= inv;
            if constexpr (BF) {
                // lane (i, h) holds columns 8 g + 4 h .. + 3 of its row: the pair exchanges so that each lane stores 16 bytes
#pragma unroll
                for (int g = 0; g < 4; g += 2) {
                    const uint32_t a0 = f2bf_pk(o[n][dt][4 * g], o[n][dt][4 * g + 1]), a1 = f2bf_pk(o[n][dt][4 * g + 2], o[n][dt][4 * g + 3]);
                    const uint32_t b0 = f2bf_pk(o[n][dt][4 * g + 4], o[n][dt][4 * g + 5]), b1 = f2bf_pk(o[n][dt][4 * g + 6], o[n][dt][4 * g + 7]);
                    const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
                    const auto s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
                    const int col = 32 * dt + 8 * (g + lh);
                    if (ok && col < a.d) *(uint4*)(out + col) = uint4{s0[0], s1[0], s0[1], s1[1]};
                }
            } else {
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int col = 32 * dt + 8 * g + 4 * lh;
                    if (ok && col < a.d) *(float4*)(out + col) = float4{o[n][dt][4 * g], o[n][dt][4 * g + 1], o[n][dt][4 * g + 2], o[n][dt][4 * g + 3]};
                }
            }
        }
    }
}

// Shares of a row's keys -> the row: offsets brought to the smallest, outputs and sums added, a workgroup's wavefronts every fourth
// share each and then in order.  One workgroup per row.
struct JoinArgs {
    const float* part;             // [shares][n_q Hq][d], then [shares][n_q Hq][2]: offset (+inf: nothing seen), sum
    void* O;
    float* lse;
    const int* q_off;
    long long o_token, o_head;
    int B, Hq, Hkv, G, d, n_q, max_q, shares;
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
    float off = INFINITY, odd = 0.f;
    for (int s = lane; s < shares; s += 64) {
        const float x = ml[(long long)s * all].x;
        off = fminf(off, x);
        if (x != x) odd = x;
    }
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        off = fminf(off, __shfl_xor(off, s));
        odd += __shfl_xor(odd, s);                   // (0, or NaN)
    }
    const bool cols = 4 * lane < a.d;
    const float* const p = a.part + at * a.d + 4 * lane;
    float total = odd;
    float4 o = float4{odd, odd, odd, odd};           // columns 4 lane .. + 3
    for (int s0 = wave; s0 < shares; s0 += 4 * kJoinAhead) {
        float4 x[kJoinAhead];
        float2 y[kJoinAhead];
#pragma unroll
        for (int i = 0; i < kJoinAhead; ++i) {
            const int s = s0 + 4 * i;
            y[i] = s < shares ? ml[(long long)s * all] : float2{INFINITY, 0.f};
            x[i] = s < shares && cols ? *(const float4*)(p + (long long)s * all * a.d) : float4{0.f, 0.f, 0.f, 0.f};
        }
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
template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(JoinArgs a) {
    const int per = a.max_q * a.Hq;
    join_row<T>(a, blockIdx.x / per, blockIdx.x % per);
}

}  // namespace csat
