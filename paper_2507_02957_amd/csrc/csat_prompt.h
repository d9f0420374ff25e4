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
template <typename T, int DT> constexpr int prompt_lds_bytes() { return 2 * 2 * prompt_key_tiles<T>() * 32 * DT * 32 * (int)sizeof(T); }

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

// Values of a 16-byte piece that are infinite or NaN.
template <typename T> __device__ __forceinline__ bool not_finite(const uint4& w);
template <> __device__ __forceinline__ bool not_finite<bf16_t>(const uint4& w) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t x = (&w.x)[i];
        any |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
    }
    return any;
}
template <> __device__ __forceinline__ bool not_finite<float>(const uint4& w) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) any |= ((&w.x)[i] & 0x7f800000u) == 0x7f800000u;
    return any;
}
// A fragment dword of bf16 pairs: what is finite; and 1.0 where it is NaN (kind 0), +inf (1), -inf (2).
__device__ __forceinline__ uint32_t finite_pair(uint32_t x) {
    return x & (((x & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u));
}
__device__ __forceinline__ uint32_t odd_pair(uint32_t x, int kind) {
    auto one = [&](uint32_t v) -> uint32_t {
        const bool is = kind == 0 ? (v & 0x7fffu) > 0x7f80u : v == (kind == 1 ? 0x7f80u : 0xff80u);
        return is ? 0x3f80u : 0u;
    };
    return one(x & 0xffffu) | (one(x >> 16) << 16);
}
__device__ __forceinline__ float odd_value(float finite, float nan, float pinf, float ninf) {
    if (nan > 0.f || (pinf > 0.f && ninf > 0.f)) return __uint_as_float(0x7fc00000u);
    return pinf > 0.f ? finite + INFINITY : ninf > 0.f ? finite - INFINITY : finite;
}

__device__ __forceinline__ float pair_max(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
}

template <typename T, int DT, int NT>
__global__ __launch_bounds__(64 * kPromptWaves) void prompt_kernel(PromptArgs a) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
    constexpr bool BF = sizeof(T) == 2;
    constexpr int KT = prompt_key_tiles<T>(), KEYS = 32 * KT, D = 32 * DT, THREADS = 64 * kPromptWaves;
    constexpr int EPC = Elem<T>::per_chunk, C = D / EPC, NK = C / 2;      // 16-byte pieces of a row, pairs of them
    constexpr int PIECES = KEYS * C / THREADS;
    static_assert(KEYS * C % THREADS == 0, "a step's pieces are dealt out evenly");
    // swizzles within a row: 8 rows (K, read 16 bytes per row) or 4 rows (V, read 32 bytes per row) fall into different banks
    constexpr int SWK = C % 8 == 0 ? 7 : 3, SWV = C % 8 == 0 ? 3 : 1;
    extern __shared__ uint4 lds[];
    uint4* const ldsK = lds;
    uint4* const ldsV = lds + 2 * KEYS * C;

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
    int lim[NT], tok[NT], head[NT];
    uint4 qf[NT][NK];
    const int dc = a.d / EPC;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        int r = w_base + 32 * n + li;
        if (r >= rows) r = rows - 1;
        tok[n] = r / a.G;
        head[n] = hk * a.G + r % a.G;
        lim[n] = limit_of(r);
        const T* q = (const T*)a.Q + (long long)(qs.first + tok[n]) * a.q_token + (long long)head[n] * a.q_head;
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

    const T* const kb = (const T*)a.K + (long long)ks.first * a.k_token + (long long)hk * a.k_head;
    const T* const vb = (const T*)a.V + (long long)ks.first * a.v_token + (long long)hk * a.v_head;
    uint4 kr[PIECES], vr[PIECES];
    auto load = [&](int t) {      // rows behind the sequence's last one as that one (masked), columns behind d as zeros
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int q = p * THREADS + tid, c = q % C;
            int row = t * KEYS + q / C;
            row = row < nk ? row : nk - 1;
            kr[p] = vr[p] = uint4{0u, 0u, 0u, 0u};
            if (c < dc) {
                kr[p] = *(const uint4*)(kb + (long long)row * a.k_token + c * EPC);
                vr[p] = *(const uint4*)(vb + (long long)row * a.v_token + c * EPC);
            }
        }
    };
    if (t0 < t1) load(t0);
    for (int t = t0; t < t1; ++t) {
        uint4* const sk = ldsK + (t & 1) * KEYS * C;
        uint4* const sv = ldsV + (t & 1) * KEYS * C;
        const bool masks = (t + 1) * KEYS > lo;      // some row of the workgroup does not see all of the step's keys
        bool odd = false;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const int q = p * THREADS + tid, row = q / C, c = q % C;
            sk[row * C + (c ^ (row & SWK))] = kr[p];
            sv[row * C + (c ^ (2 * (row & SWV)))] = vr[p];
            if (masks) odd |= not_finite<T>(vr[p]);
        }
        // (one barrier a step: the other half of the LDS was last read a step earlier)
        if (masks) odd = __syncthreads_or(odd) != 0;
        else __syncthreads();
        if (t + 1 < t1) load(t + 1);
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
                const uint4 kf = sk[(32 * u + li) * C + ((2 * g + lh) ^ (li & SWK))];
#pragma unroll
                for (int n = 0; n < NT; ++n) mfma_group<T>(kf, qf[n][g], s[n][u]);
            }
        const bool w_masks = (t + 1) * KEYS > w_lo;
        if (w_masks) {
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
        // O^T += V^T P^T.  A masked key's weight is 0, but 0 times an infinity or NaN is NaN: a step in which some row does not
        // see all keys and V holds such a value takes the finite part of V, and the others by what they are, for the rows
        // that see them (products with 1 for a visible key, 0 for a masked one).
        auto product = [&](auto oddc) {
            constexpr bool ODD = decltype(oddc)::value;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                f32x16 cnt[ODD ? NT : 1][3];
                if constexpr (ODD) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 3; ++k)
#pragma unroll
                            for (int v = 0; v < 16; ++v) cnt[n][k][v] = 0.f;
                }
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    if constexpr (BF) {
#pragma unroll
                        for (int h2 = 0; h2 < 2; ++h2) {
                            const int l = lane & 15;
                            const int row = 32 * u + 16 * h2 + 4 * lh + (l >> 2);
                            const int c = 4 * dt + 2 * ((lane >> 4) & 1) + ((l & 3) >> 1);
                            const char* p = (const char*)(sv + row * C + (c ^ (2 * (row & SWV)))) + (l & 1) * 8;
                            const char* p8 = (const char*)(sv + (row + 8) * C + (c ^ (2 * ((row + 8) & SWV)))) + (l & 1) * 8;
                            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p);
                            const s16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p8);
                            const uint2 w0 = __builtin_bit_cast(uint2, v0), w1 = __builtin_bit_cast(uint2, v1);
                            uint4 vf = uint4{w0.x, w0.y, w1.x, w1.y};
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                const f32x16& e = s[n][u];
                                const uint4 pf = uint4{f2bf_pk(e[8 * h2], e[8 * h2 + 1]), f2bf_pk(e[8 * h2 + 2], e[8 * h2 + 3]),
                                                       f2bf_pk(e[8 * h2 + 4], e[8 * h2 + 5]), f2bf_pk(e[8 * h2 + 6], e[8 * h2 + 7])};
                                if constexpr (ODD) {
                                    uint4 fin, ones;
#pragma unroll
                                    for (int i = 0; i < 4; ++i) {
                                        (&fin.x)[i] = finite_pair((&vf.x)[i]);
                                        const int key = t * KEYS + 32 * u + 16 * h2 + 8 * (i >> 1) + 4 * lh + 2 * (i & 1);
                                        (&ones.x)[i] = (key < lim[n] ? 0x3f80u : 0u) | (key + 1 < lim[n] ? 0x3f800000u : 0u);
                                    }
                                    mfma_group<T>(fin, pf, o[n][dt]);
#pragma unroll
                                    for (int k = 0; k < 3; ++k) {
                                        uint4 ind;
#pragma unroll
                                        for (int i = 0; i < 4; ++i) (&ind.x)[i] = odd_pair((&vf.x)[i], k);
                                        mfma_group<T>(ind, ones, cnt[n][k]);
                                    }
                                } else {
                                    mfma_group<T>(vf, pf, o[n][dt]);
                                }
                            }
                        }
                    } else {
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const int row = 32 * u + 8 * (v >> 2) + 4 * lh + (v & 3), col = 32 * dt + li;
                            const float x = ((const float*)(sv + row * C + ((col >> 2) ^ (2 * (row & SWV)))))[col & 3];
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                if constexpr (ODD) {
                                    const bool fin = fabsf(x) < INFINITY;
                                    const float one = t * KEYS + row < lim[n] ? 1.f : 0.f;
                                    o[n][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(fin ? x : 0.f, s[n][u][v], o[n][dt], 0, 0, 0);
                                    cnt[n][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x != x ? 1.f : 0.f, one, cnt[n][0], 0, 0, 0);
                                    cnt[n][1] = __builtin_amdgcn_mfma_f32_32x32x2f32(x == INFINITY ? 1.f : 0.f, one, cnt[n][1], 0, 0, 0);
                                    cnt[n][2] = __builtin_amdgcn_mfma_f32_32x32x2f32(x == -INFINITY ? 1.f : 0.f, one, cnt[n][2], 0, 0, 0);
                                } else {
                                    o[n][dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, s[n][u][v], o[n][dt], 0, 0, 0);
                                }
                            }
                        }
                    }
                }
                if constexpr (ODD) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int v = 0; v < 16; ++v) o[n][dt][v] = odd_value(o[n][dt][v], cnt[n][0][v], cnt[n][1][v], cnt[n][2][v]);
                }
            }
        };
        if (odd && w_masks) product(std::true_type{});
        else product(std::false_type{});
    }
    if (!active) return;

#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float total = pair_sum(sum[n]);
        const bool ok = w_base + 32 * n + li < rows;
        const long long row = qs.first + tok[n];
        if (a.shares > 1) {
            const long long all = (long long)a.n_q * a.Hq, at = (long long)share * all + row * a.Hq + head[n];
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
        if (a.lse && ok && lh == 0) a.lse[(long long)head[n] * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - off[n]);
        T* out = (T*)a.O + row * a.o_token + (long long)head[n] * a.o_head;
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

// Shares of a row's keys -> the row: offsets brought to the smallest, outputs and sums added in the order of the shares.
// One wavefront per row.
struct JoinArgs {
    const float* part;             // [shares][n_q Hq][d], then [shares][n_q Hq][2]: offset (+inf: nothing seen), sum
    void* O;
    float* lse;
    const int* q_off;
    long long o_token, o_head;
    int B, Hq, Hkv, G, d, n_q, max_q, shares;
};

template <typename T>
__global__ __launch_bounds__(256) void attention_join_kernel(JoinArgs a) {
    const int lane = threadIdx.x & 63;
    const int per = (a.max_q * a.Hq + 3) / 4;
    const int b = blockIdx.x / per, r = (blockIdx.x % per) * 4 + (threadIdx.x >> 6);
    const PackedSpan qs(a.q_off, b, a.n_q);
    const int tok = r / a.Hq, head = r % a.Hq;
    if (tok >= (qs.count < a.max_q ? qs.count : a.max_q)) return;
    const long long row = qs.first + tok, all = (long long)a.n_q * a.Hq, at = row * a.Hq + head;
    const float2* ml = (const float2*)(a.part + (long long)a.shares * all * a.d) + at;
    float off = INFINITY, bad = 0.f;
    for (int s = 0; s < a.shares; ++s) {
        const float x = ml[(long long)s * all].x;
        off = fminf(off, x);
        if (x != x) bad = x;
    }
    float total = bad, o[4] = {bad, bad, bad, bad};      // columns 4 lane .. + 3
    for (int s = 0; s < a.shares; ++s) {
        const float2 x = ml[(long long)s * all];
        if (x.x == INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(off - x.x);
        total += f * x.y;
        if (4 * lane < a.d) {
            const float4 p = *(const float4*)(a.part + ((long long)s * all + at) * a.d + 4 * lane);
            o[0] += f * p.x; o[1] += f * p.y; o[2] += f * p.z; o[3] += f * p.w;
        }
    }
    const float inv = total == 0.f ? 0.f : 1.f / total;
    if (a.lse && lane == 0) a.lse[(long long)head * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) - off);
    if (4 * lane >= a.d) return;
    T* out = (T*)a.O + row * a.o_token + (long long)head * a.o_head + 4 * lane;
    if constexpr (sizeof(T) == 2) *(uint2*)out = uint2{f2bf_pk(o[0] * inv, o[1] * inv), f2bf_pk(o[2] * inv, o[3] * inv)};
    else *(float4*)out = float4{o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
}

}  // namespace csat
