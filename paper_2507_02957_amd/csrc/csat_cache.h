// Key/value cache in 8 bits: store, attention over it, eviction.
//
// A block is one page of one head: `page` tokens of e4m3 codes under one scale 2^e.  With a power of two, x / scale and a
// code brought to another scale are exact before their one rounding to e4m3, so store and eviction have one right answer, bit
// for bit, and a code that keeps its scale keeps its bits.
//
// K lies [token][d] and V [d][token] within a block: what a lane of the attention's matrix instructions needs, 16 features
// of a token of K and 16 tokens of a feature of V, is 16 consecutive bytes of memory in either, so the attention reads
// the cache straight into registers, without LDS and without a transposition.
#pragma once
#include "csat_prompt.h"

namespace csat {

struct CacheView {
    uint8_t *K, *V;
    float *Ks, *Vs;
    const int* table;
    int* lengths;
    int pages, page, log_page, max_pages, max_len;
};

constexpr int kScaleMin = -118;
// 2^e, |e| <= 126
__device__ __forceinline__ float pow2f(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// smallest e >= kScaleMin with amax <= 448 * 2^e = 0.875 * 2^(e + 9), of a finite amax >= 0
__device__ __forceinline__ int scale_exponent(float amax) {
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 126 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0) - 9;      // amax = f 2^(u >> 23) - 126), f in [0.5, 1)
    return e < kScaleMin ? kScaleMin : e;                                                // (a subnormal amax is far below the least scale)
}
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23) - 127; }

__device__ __forceinline__ float finite_abs(float x) {
    const float v = fabsf(x);
    return v < INFINITY ? v : 0.f;
}
__device__ __forceinline__ float nan_if_odd(float x) { return fabsf(x) < INFINITY ? x : __uint_as_float(0x7fc00000u); }
// four floats (already divided by the scale) -> four codes, nearest, ties to even; codes_of: none of them infinite
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) { return codes_of(nan_if_odd(a), nan_if_odd(b), nan_if_odd(c), nan_if_odd(d)); }
__device__ __forceinline__ uint32_t rescale_codes(uint32_t w, float f) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return codes_of(lo[0] * f, lo[1] * f, hi[0] * f, hi[1] * f);
}

// ---- store

struct StoreArgs {
    CacheView c;
    const void *K, *V;
    const int* k_off;
    long long k_token, k_head, v_token, v_head;
    int B, Hkv, d, n_k, max_k, reach;      // reach: pages that one sequence's new tokens may touch
    int quad_magic;                        // 2^20 / (d / 4) + 1: a piece's row without a division
    __device__ __forceinline__ int by_row(int q) const { return (int)((uint32_t)q * (uint32_t)quad_magic >> 20); }      // q / (d / 4), q < 2^11
};

__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2) x = fmaxf(x, __shfl_xor(x, s));
    return x;
}

// 4 x 4 bytes: word i's byte j becomes word j's byte i
__device__ __forceinline__ void transpose_bytes(uint32_t (&w)[4]) {
    const uint32_t a0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), a1 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u);      // w0 w1 bytes 0, 1 in turn
    const uint32_t b0 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u), b1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(a1, a0, 0x05040100u);
    w[1] = __builtin_amdgcn_perm(a1, a0, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(b1, b0, 0x05040100u);
    w[3] = __builtin_amdgcn_perm(b1, b0, 0x07060302u);
}
// bytes of a word at slot s that lie in [lo, hi)
__device__ __forceinline__ uint32_t byte_mask(int s, int lo, int hi) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) m |= s + e >= lo && s + e < hi ? 0xffu << (8 * e) : 0u;
    return m;
}

// One workgroup per touched block (K and V of it).  A thread holds NI pieces of 4 tokens by 4 features of both, so memory is read
// once: largest finite magnitudes over the workgroup, the codes, K's rows straight to memory, V's 4 x 4 bytes turned and
// through LDS, from which they leave 16 tokens of a feature at a time, next to what older tokens the 16 hold.
// Bound by memory: (2 or 4) + 1 bytes a value in and out; 16910 tokens, 8 heads, d 128, bf16: 104 MB in 25 us, 4.1 TB/s of the 4.8
// that a copy reaches (50 us with two passes over memory and V's bytes gathered from it).  One token each of 64 sequences: 7.8 us,
// launch and latency.
constexpr int store_lds_bytes(int d, int page) { return d * (page + 4); }
template <typename T, int NI>
__global__ __launch_bounds__(256) void cache_store_kernel(StoreArgs a) {
    __shared__ float red[2][4];
    extern __shared__ uint4 turned[];                // [d][page + 4] codes of V
    const int tid = threadIdx.x;
    const int b = blockIdx.y, i = blockIdx.x / a.Hkv, hk = blockIdx.x - i * a.Hkv;
    const PackedSpan ks(a.k_off, b, a.n_k);
    const int n = ks.count < a.max_k ? ks.count : a.max_k;
    const int len = a.c.lengths[b];
    if (n <= 0 || len > a.c.max_len || len < ks.count) return;
    const int start = len - ks.count, end = start + n;      // (rows beyond max_k have their places too)
    const int page = a.c.page, first = start >> a.c.log_page, last = (end - 1) >> a.c.log_page;
    const int j = first + i;
    if (j > last) return;
    const int* const table = a.c.table + (long long)b * a.c.max_pages;
    const int lo = j == first ? start - j * page : 0, hi = j == last ? end - j * page : page;      // new slots
    const long long row0 = ks.first + ((long long)j * page - start);      // packed row of slot 0
    const T* K = (const T*)a.K + row0 * a.k_token + (long long)hk * a.k_head;
    const T* V = (const T*)a.V + row0 * a.v_token + (long long)hk * a.v_head;
    const int dq = a.d / 4, items = page / 4 * dq;
    typedef typename std::conditional<sizeof(T) == 2, uint2, float4>::type Four;
    // everything that memory has to say is asked for at once: the block's scales and, at the ends of the new tokens, what 16 slots hold
    const int id = table[j];
    bool bad = id < 0 || id >= a.c.pages;
    const long long block = (long long)(bad ? 0 : id) * a.Hkv + hk;
    const float ok = lo ? a.c.Ks[block] : 0.f, ov = lo ? a.c.Vs[block] : 0.f;
    uint8_t* const ck = a.c.K + block * page * a.d;
    uint8_t* const cv = a.c.V + block * page * a.d;
    const int lg = a.c.log_page - 4, groups = 1 << lg, pieces = a.d << lg;      // 16-token pieces of V's features
    uint4 was[NI];
#pragma unroll
    for (int p = 0; p < NI; ++p) {
        const int q = p * 256 + tid, g = (q & (groups - 1)) * 16;
        was[p] = q < pieces && g < hi && g + 16 > lo && (g < lo || g + 16 > hi) ? ((const uint4*)cv)[q] : uint4{0u, 0u, 0u, 0u};
    }
    Four xk[NI][4], xv[NI][4];
#pragma unroll
    for (int p = 0; p < NI; ++p) {
        const int q = p * 256 + tid, i4 = a.by_row(q), s = 4 * i4, f = 4 * (q - i4 * dq);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            xk[p][e] = xv[p][e] = Four{};
            if (q < items && s + e >= lo && s + e < hi) {
                xk[p][e] = *(const Four*)(K + (long long)(s + e) * a.k_token + f);
                xv[p][e] = *(const Four*)(V + (long long)(s + e) * a.v_token + f);
            }
        }
    }
    // a sequence with a page that does not exist is not stored to at all
    for (int t = first + tid; t <= last; t += 256) bad |= table[t] < 0 || table[t] >= a.c.pages;
    auto four = [](const Four& w, float* x) {
        if constexpr (sizeof(T) == 2) {
            x[0] = __uint_as_float(w.x << 16); x[1] = __uint_as_float(w.x & 0xffff0000u);
            x[2] = __uint_as_float(w.y << 16); x[3] = __uint_as_float(w.y & 0xffff0000u);
        } else {
            x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
        }
    };
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int p = 0; p < NI; ++p)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x[4];
            four(xk[p][e], x);
            mk = fmaxf(mk, fmaxf(fmaxf(finite_abs(x[0]), finite_abs(x[1])), fmaxf(finite_abs(x[2]), finite_abs(x[3]))));
            four(xv[p][e], x);
            mv = fmaxf(mv, fmaxf(fmaxf(finite_abs(x[0]), finite_abs(x[1])), fmaxf(finite_abs(x[2]), finite_abs(x[3]))));
        }
    mk = wave_max(mk);
    mv = wave_max(mv);
    if ((tid & 63) == 0) { red[0][tid >> 6] = mk; red[1][tid >> 6] = mv; }
    if (__syncthreads_or(bad)) return;
    mk = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    mv = fmaxf(fmaxf(red[1][0], red[1][1]), fmaxf(red[1][2], red[1][3]));
    const float sk = fmaxf(pow2f(scale_exponent(mk)), ok), sv = fmaxf(pow2f(scale_exponent(mv)), ov);
    const float ik = pow2f(-exponent_of(sk)), iv = pow2f(-exponent_of(sv));

    const int pitch = page + 4;
#pragma unroll
    for (int p = 0; p < NI; ++p) {
        const int q = p * 256 + tid, i4 = a.by_row(q), s = 4 * i4, f = 4 * (q - i4 * dq);
        if (q >= items || s + 4 <= lo || s >= hi) continue;
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x[4];
            four(xk[p][e], x);
            if (s + e >= lo && s + e < hi) *(uint32_t*)(ck + (long long)(s + e) * a.d + f) = to_codes(x[0] * ik, x[1] * ik, x[2] * ik, x[3] * ik);
            four(xv[p][e], x);
            w[e] = to_codes(x[0] * iv, x[1] * iv, x[2] * iv, x[3] * iv);
        }
        transpose_bytes(w);
#pragma unroll
        for (int e = 0; e < 4; ++e) *(uint32_t*)((uint8_t*)turned + (f + e) * pitch + s) = w[e];
    }
    if (lo && sk != ok) {
        const float f = ok * ik;
        for (int q = tid; q < lo * dq; q += 256) ((uint32_t*)ck)[q] = rescale_codes(((uint32_t*)ck)[q], f);
    }
    __syncthreads();
    if (tid == 0) { a.c.Ks[block] = sk; a.c.Vs[block] = sv; }      // (behind the barrier: every thread has read the old ones)
    const float fv = ov * iv;
#pragma unroll
    for (int p = 0; p < NI; ++p) {
        const int q = p * 256 + tid, g = (q & (groups - 1)) * 16, f = q >> lg;
        if (q >= pieces || g >= hi || (g + 16 <= lo && sv == ov)) continue;
        uint4 w;
#pragma unroll
        for (int k = 0; k < 4; ++k) (&w.x)[k] = *(const uint32_t*)((const uint8_t*)turned + f * pitch + g + 4 * k);
        if (g < lo || g + 16 > hi) {
            if (g + 16 <= lo) was[p] = ((const uint4*)cv)[q];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int s = g + 4 * k;
                const uint32_t in = byte_mask(s, lo, hi), old = byte_mask(s, 0, lo);
                uint32_t x = (&was[p].x)[k];
                if (old && sv != ov) x = (rescale_codes(x, fv) & old) | (x & ~old);
                (&w.x)[k] = ((&w.x)[k] & in) | (x & ~in);
            }
        }
        ((uint4*)cv)[q] = w;
    }
}

// ---- attention over the cache

struct CachedArgs {
    CacheView c;
    const void* Q;
    void* O;
    float* lse;
    const int* q_off;
    long long q_token, q_head, o_token, o_head;
    int B, Hq, Hkv, d, n_q, max_q, causal;
    Group G;
    float sl;                      // scale log2(e)
    int tiles, row_tiles;          // workgroups per sequence, key head and share, 16-row tiles in each
    int first_tile;                // of this launch
    int shares, share_tokens;      // the longest sequence's shares of share_tokens (a multiple of 64); a sequence has those it needs
    float* part;                   // [shares][n_q Hq][d], then [shares][n_q Hq][2] as in csat_prompt.h, or null: O and lse are written
    float* scores;                 // [B][Hkv][max_q G.size][score_ld] in units of log2, for the weights, or null
    int score_ld;
    float* W;                      // [B][Hkv][max_pages page]
    float decay;
};

__device__ __forceinline__ float quad_max(float x) {      // over lanes n, n + 16, n + 32, n + 48
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_max(fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])));
}
__device__ __forceinline__ float quad_sum(float x) {
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return pair_sum(__uint_as_float(sw[0]) + __uint_as_float(sw[1]));
}
// eight codes -> a bf16 fragment (every e4m3 value is a bf16 value)
__device__ __forceinline__ bf16x8 code_fragment(uint32_t lo, uint32_t hi) {
    uint4 w;
    w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
    w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
    w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
    w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
    return __builtin_bit_cast(bf16x8, w);
}
__device__ __forceinline__ uint32_t nan_codes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }      // a byte's top bit: it is NaN
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
    const uint32_t n = nan_codes(w);
    return w & ~((n - (n >> 7)) | n);
}

// A tile is 64 tokens by 16 rows.  S^T = K Q^T with 16 x 16 x 32 instructions: instruction row i of sub-tile s is token
// 16 (i / 4) + 4 s + i % 4, so that a lane's 16 scores are those of the 16 consecutive tokens 16 quad .. + 15 of one query
// row, and, as the B operand of O^T = V^T P^T, meet 16 consecutive bytes of V^T.  A wavefront takes every fourth tile of its
// share and keeps a running maximum and sum of its own; the four are joined through LDS at the end.
// Bound by memory: one sequence of 131072 tokens, 8 key heads, d 128: 268 MB in 51 us, 5.3 TB/s, and 6 for the join; 32 sequences of 700
// to 8100 tokens with weights: 287 MB and 18 of scores in 74 us, then 13 (a batch without weights 75 in all).
// RT tiles of 16 rows share what is read and converted (bf16, up to 128 features: the registers).
template <int DC, int RT> constexpr int cached_lds_bytes(int d) { return RT * (4 * 16 * (d + 4) * 4 + 4 * 16 * 8) + 64 * DC * 4; }
template <typename T, int DC, int RT>
__global__ __launch_bounds__(256, DC <= 2 ? 2 : 1) void cache_attention_kernel(CachedArgs a) {
    constexpr int NP = sizeof(T) == 2 ? 1 : 3;      // float queries and weights as three bf16 parts: 24 bits
    constexpr int DT = 4 * DC;
    constexpr int ROWS = 16 * RT;
    extern __shared__ float joint[];                // [4][ROWS][d + 4] outputs, then [4][ROWS][2]; a token per feature, of its first NaN
    const int tid = threadIdx.x, lane = tid & 63, li = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.z, share = blockIdx.y, tile = a.tiles == 1 ? 0 : blockIdx.x / a.Hkv, hk = blockIdx.x - tile * a.Hkv;
    const PackedSpan qs(a.q_off, b, a.n_q);
    const int rows = (qs.count < a.max_q ? qs.count : a.max_q) * a.G.size, r_base = ROWS * (a.first_tile + tile);
    if (r_base >= rows) return;
    int L = a.c.lengths[b];
    bool bad = L < 0 || L > a.c.max_len;
    if (bad) L = 0;
    auto limit_of = [&](int r) {
        if (!a.causal) return L;
        const int v = a.G.token(r) + L - qs.count + 1;
        return v < 0 ? 0 : v > L ? L : v;
    };
    const int r_last = r_base + ROWS < rows ? r_base + ROWS - 1 : rows - 1;
    const int lo = limit_of(r_base), hi = limit_of(r_last);
    const int s0 = share * a.share_tokens, s1 = s0 + a.share_tokens < hi ? s0 + a.share_tokens : hi;
    if (s0 >= L && share > 0) return;
    const int t0 = s0 / 64, t1 = (s1 + 63) / 64;     // (none where no row of the tile sees the share)
    // features 64 c + 16 quad + 8 h .. + 7 of the lane's rows
    bf16x8 qf[RT][NP][DC][2];
    int lim[RT];
#pragma unroll
    for (int m = 0; m < RT; ++m) {
        const int r = r_base + 16 * m + li < rows ? r_base + 16 * m + li : rows - 1;
        const int tok = a.G.token(r), head = hk * a.G.size + r - tok * a.G.size;
        lim[m] = limit_of(r);
        const T* q = (const T*)a.Q + (long long)(qs.first + tok) * a.q_token + (long long)head * a.q_head;
#pragma unroll
        for (int c = 0; c < DC; ++c)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int f = 64 * c + 16 * quad + 8 * h;
                if constexpr (NP == 1) {
                    qf[m][0][c][h] = __builtin_bit_cast(bf16x8, f < a.d ? *(const uint4*)(q + f) : uint4{0u, 0u, 0u, 0u});
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float x = f < a.d ? ((const float*)q)[f + e] : 0.f;
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            qf[m][p][c][h][e] = (__bf16)x;
                            x -= (float)qf[m][p][c][h][e];
                        }
                    }
                }
            }
    }
    const int pitch = a.d + 4;
    float2* const ml = (float2*)(joint + 4 * ROWS * pitch);
    int* const nan_at = (int*)(ml + 4 * ROWS);
    for (int i = tid; i < 64 * DC; i += 256) nan_at[i] = kNoKey;
    __syncthreads();
    f32x4 o[RT][DT];
    float ref[RT], sum[RT];

    const int page = a.c.page, lp = a.c.log_page, last_page = (L - 1) >> lp;
    const int* const table = a.c.table + (long long)b * a.c.max_pages;
    const long long head_bytes = (long long)page * a.d;
    auto page_of = [&](int t) {      // (a token behind the last: any page that exists, masked below)
        int i = t >> lp;
        i = i < last_page ? i : last_page;
        int id = table[i];
        if (id < 0 || id >= a.c.pages) { bad = true; id = 0; }
        return id;
    };
    // A step's loads are issued as soon as the registers of the step before are free (K behind its products, V behind its own), the
    // pages they need are looked up another step ahead: memory is never waited for from a standstill.
    uint4 kw[4][DC], vw[DT];
    float kscale, vscale;
    auto load_k = [&](int t, int kid, int vid) {
        const int kt = 64 * t + 16 * (li >> 2);
        const uint8_t* kp = a.c.K + ((long long)kid * a.Hkv + hk) * head_bytes + (long long)((kt & (page - 1)) + (li & 3)) * a.d + 16 * quad;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int c = 0; c < DC; ++c) kw[s][c] = 64 * c + 16 * quad < a.d ? *(const uint4*)(kp + (long long)(4 * s) * a.d + 64 * c) : uint4{0u, 0u, 0u, 0u};
        kscale = a.c.Ks[(long long)vid * a.Hkv + hk] * a.sl;
    };
    auto load_v = [&](int t, int vid) {
        const int vt = 64 * t + 16 * quad;
        const uint8_t* vp = a.c.V + ((long long)vid * a.Hkv + hk) * head_bytes + (long long)li * page + (vt & (page - 1));
#pragma unroll
        for (int u = 0; u < DT; ++u) vw[u] = 16 * u < a.d ? *(const uint4*)(vp + (long long)(16 * u) * page) : uint4{0u, 0u, 0u, 0u};
        vscale = a.c.Vs[(long long)vid * a.Hkv + hk];
    };
    float down = 0.f;                                // powers of two that all weights are smaller by (headroom, csat_prompt.h): references are larger
    for (;; down = headroom(L)) {
#pragma unroll
        for (int m = 0; m < RT; ++m) {
            ref[m] = -INFINITY;
            sum[m] = 0.f;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        int kid = 0, vid = 0, kid2 = 0, vid2 = 0;    // of the next step, of the one behind it
        int start = t0 + wave;
        asm volatile("" : "+s"(start));              // (so that a second pass keeps nothing in registers for its beginning)
        if (start < t1) {
            const int t = start;
            kid = page_of(64 * t + 16 * (li >> 2));
            vid = page_of(64 * t + 16 * quad);
            if (t + 4 < t1) { kid2 = page_of(64 * (t + 4) + 16 * (li >> 2)); vid2 = page_of(64 * (t + 4) + 16 * quad); }
            load_k(t, kid, vid);
            load_v(t, vid);
            kid = kid2; vid = vid2;
        }
        for (int t = start; t < t1; t += 4) {
            const int first = 64 * t, vt = first + 16 * quad;
            if (t + 8 < t1) { kid2 = page_of(64 * (t + 8) + 16 * (li >> 2)); vid2 = page_of(64 * (t + 8) + 16 * quad); }

            float e[RT][16];
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                f32x4 acc[RT];
#pragma unroll
                for (int m = 0; m < RT; ++m) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < DC; ++c) {
                    const bf16x8 k0 = code_fragment(kw[s][c].x, kw[s][c].y), k1 = code_fragment(kw[s][c].z, kw[s][c].w);
#pragma unroll
                    for (int m = 0; m < RT; ++m)
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[m][p][c][0], acc[m], 0, 0, 0);
                            acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[m][p][c][1], acc[m], 0, 0, 0);
                        }
                }
#pragma unroll
                for (int m = 0; m < RT; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) e[m][4 * s + i] = acc[m][i] * kscale;
            }
            __builtin_amdgcn_sched_barrier(0);
            if (t + 4 < t1) load_k(t + 4, kid, vid);
            __builtin_amdgcn_sched_barrier(0);
            const bool masks = first + 64 > lo;
            bf16x8 pf[RT][NP][2];
#pragma unroll
            for (int m = 0; m < RT; ++m) {
                const int r = r_base + 16 * m + li;
                if (masks) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (vt + i >= lim[m]) e[m][i] = -INFINITY;
                }
                if (a.scores && r < rows) {
                    float* p = a.scores + (((long long)b * a.Hkv + hk) * a.max_q * a.G.size + r) * a.score_ld + vt;
#pragma unroll
                    for (int i = 0; i < 16; i += 4) *(float4*)(p + i) = float4{e[m][i], e[m][i + 1], e[m][i + 2], e[m][i + 3]};
                }
                float mx = e[m][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) mx = fmaxf(mx, e[m][i]);
                mx = quad_max(mx);
                if (__builtin_amdgcn_ballot_w64(mx - ref[m] > 8.f - down) != 0) {
                    const float nm = fmaxf(mx + down, ref[m]);
                    const float f = ref[m] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ref[m] - nm);
                    ref[m] = nm;
                    sum[m] *= f;
#pragma unroll
                    for (int u = 0; u < DT; ++u) o[m][u] *= f;
                }
                const float base = ref[m] == -INFINITY ? 0.f : ref[m];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    e[m][i] = __builtin_amdgcn_exp2f(e[m][i] - base);
                    sum[m] += e[m][i];
                    e[m][i] *= vscale;
                }
                // weights of bf16 precision for bf16 tensors; the other parts for float ones
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float x = e[m][8 * h + i];
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            pf[m][p][h][i] = (__bf16)x;
                            x -= (float)pf[m][p][h][i];
                        }
                    }
            }
            if (masks) {      // NaN codes out of tokens that some row does not see (0 times NaN is NaN), the first of each feature noted
                uint32_t any = 0;
#pragma unroll
                for (int u = 0; u < DT; ++u) any |= nan_codes(vw[u].x) | nan_codes(vw[u].y) | nan_codes(vw[u].z) | nan_codes(vw[u].w);
                if (__builtin_amdgcn_ballot_w64(any != 0) != 0) {
#pragma unroll
                    for (int u = 0; u < DT; ++u) {
                        int at = 16;
#pragma unroll
                        for (int i = 3; i >= 0; --i) {
                            uint32_t& w = (&vw[u].x)[i];
                            const uint32_t n = nan_codes(w);
                            if (n) at = 4 * i + (__ffs(n) - 1) / 8;
                            w = without_nan(w);
                        }
                        if (at < 16) atomicMin(nan_at + 16 * u + li, vt + at);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < DT; ++u) {
                const bf16x8 v0 = code_fragment(vw[u].x, vw[u].y), v1 = code_fragment(vw[u].z, vw[u].w);
#pragma unroll
                for (int m = 0; m < RT; ++m)
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        o[m][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, pf[m][p][0], o[m][u], 0, 0, 0);
                        o[m][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, pf[m][p][1], o[m][u], 0, 0, 0);
                    }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (t + 4 < t1) load_v(t + 4, vid);
            kid = kid2; vid = vid2;
        }
        float squares = 0.f;
#pragma unroll
        for (int m = 0; m < RT; ++m)
#pragma unroll
            for (int u = 0; u < DT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) squares = __builtin_fmaf(o[m][u][i], o[m][u][i], squares);
        if (down != 0.f || __builtin_amdgcn_ballot_w64(!(squares < INFINITY)) == 0) break;
    }

    // (where a lane is, counted anew: nothing of it is held over the loop, whose registers are all taken with two row tiles)
    const int at_lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)), at_li = at_lane & 15, at_quad = at_lane >> 4;
    const int at_tid = 64 * wave + at_lane;
    // the wavefronts' parts of a row, brought to the largest reference
    const bool any_bad = __builtin_amdgcn_ballot_w64(bad) != 0;
#pragma unroll
    for (int m = 0; m < RT; ++m) {
        const float total = any_bad ? __uint_as_float(0x7fc00000u) : quad_sum(sum[m]);
#pragma unroll
        for (int u = 0; u < DT; ++u)
            if (16 * u < a.d) *(f32x4*)(joint + (wave * ROWS + 16 * m + at_li) * pitch + 16 * u + 4 * at_quad) = o[m][u];
        if (at_quad == 0) ml[wave * ROWS + 16 * m + at_li] = float2{ref[m], total};
    }
    __syncthreads();
    const int n_rows = rows - r_base < ROWS ? rows - r_base : ROWS, dq = a.d / 4;
    for (int q = at_tid; q < n_rows * dq; q += 256) {
        const int i = q / dq, f = q % dq * 4;
        float m = -INFINITY, total = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) m = fmaxf(m, ml[w * ROWS + i].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 y = ml[w * ROWS + i];
            if (y.y == 0.f) continue;
            const float k = y.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(y.x - m);      // (a sum that is NaN without a maximum stays)
            const float4 z = *(const float4*)(joint + (w * ROWS + i) * pitch + f);
            total += k * y.y;
            x[0] += k * z.x; x[1] += k * z.y; x[2] += k * z.z; x[3] += k * z.w;
        }
        const int rr = r_base + i, rt = a.G.token(rr), h = hk * a.G.size + rr - rt * a.G.size, seen = limit_of(rr);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (nan_at[f + e] < seen) x[e] = __uint_as_float(0x7fc00000u);
        const long long row = qs.first + rt;
        if (a.part) {
            const long long all = (long long)a.n_q * a.Hq, at = (long long)share * all + row * a.Hq + h;
            *(float4*)(a.part + at * a.d + f) = float4{x[0], x[1], x[2], x[3]};
            if (f == 0) ((float2*)(a.part + (long long)a.shares * all * a.d))[at] = float2{total == 0.f ? INFINITY : m == -INFINITY ? 0.f : -m, total};
            continue;
        }
        const float inv = total == 0.f ? 0.f : 1.f / total;
        if (a.lse && f == 0) a.lse[(long long)h * a.n_q + row] = total == 0.f ? -INFINITY : 0.69314718055994531f * (__log2f(total) + m);
        T* out = (T*)a.O + row * a.o_token + (long long)h * a.o_head + f;
        if constexpr (sizeof(T) == 2) *(uint2*)out = uint2{f2bf_pk(x[0] * inv, x[1] * inv), f2bf_pk(x[2] * inv, x[3] * inv)};
        else *(float4*)out = float4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv};
    }
}

// The second launch, y a sequence: its first o_blocks workgroups join the rows of O, the others form W = decay W + sum over rows of
// 2^(score - lse) for 1024 tokens of a key head, a thread four of them.  first_block: of this launch.
template <typename T>
__global__ __launch_bounds__(256) void cache_join_kernel(JoinArgs j, CachedArgs a, int o_blocks, int first_block) {
    constexpr int RB = 64;
    __shared__ float lse2[RB];
    __shared__ int limit[RB];
    const int b = blockIdx.y, block = first_block + blockIdx.x;
    if (block < o_blocks) {
        join_block<T>(j, b, block);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63;
    const int chunks = (a.c.max_len + 1023) / 1024, id = block - o_blocks, hk = id / chunks, chunk = id - hk * chunks;
    const int L = a.c.lengths[b], t = chunk * 1024 + 4 * tid;
    if (L < 0 || L > a.c.max_len || chunk * 1024 >= L) return;
    const PackedSpan qs(a.q_off, b, a.n_q);
    const int rows = (qs.count < a.max_q ? qs.count : a.max_q) * a.G.size;
    const long long all = (long long)a.n_q * a.Hq;
    const float2* ml = (const float2*)(a.part + (long long)a.shares * all * a.d);
    const int shares = shares_of(a.c.lengths, b, a.share_tokens, a.c.max_len, a.shares);
    float* const w = a.W + ((long long)b * a.Hkv + hk) * a.c.max_pages * a.c.page + t;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    // four rows' scores are asked for ahead of what they are weighed with
    const float* const scores = a.scores + ((long long)b * a.Hkv + hk) * a.max_q * a.G.size * a.score_ld + t;
    float4 y[4];
    auto ask = [&](int r) {
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = r + k < rows && t < L ? *(const float4*)(scores + (long long)(r + k) * a.score_ld) : float4{0.f, 0.f, 0.f, 0.f};
    };
    ask(0);
    for (int r0 = 0; r0 < rows; r0 += RB) {
        const int n = rows - r0 < RB ? rows - r0 : RB;
        __syncthreads();
        for (int i = tid >> 6; i < n; i += 4) {      // a wavefront a row
            const int r = r0 + i, tok = a.G.token(r);
            const long long at = (long long)(qs.first + tok) * a.Hq + hk * a.G.size + r - tok * a.G.size;
            const float2 z = lane < shares ? ml[(long long)lane * all + at] : float2{INFINITY, 0.f};      // (the first 64 shares)
            float off = z.x;
            for (int s = lane + 64; s < shares; s += 64) off = fminf(off, ml[(long long)s * all + at].x);
#pragma unroll
            for (int s = 1; s < 64; s *= 2) off = fminf(off, __shfl_xor(off, s));
            float total = z.x == INFINITY ? 0.f : __builtin_amdgcn_exp2f(off - z.x) * z.y;
            for (int s = lane + 64; s < shares; s += 64) {
                const float2 v = ml[(long long)s * all + at];
                if (v.x != INFINITY) total += __builtin_amdgcn_exp2f(off - v.x) * v.y;
            }
#pragma unroll
            for (int s = 1; s < 64; s *= 2) total += __shfl_xor(total, s);
            const int v = a.causal ? tok + L - qs.count + 1 : L;
            if (lane == 0) {
                lse2[i] = total == 0.f ? INFINITY : __log2f(total) - off;      // (nothing seen: weights 0)
                limit[i] = v < 0 ? 0 : v > L ? L : v;
            }
        }
        __syncthreads();
        for (int i = 0; i < n; i += 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float l = i + k < n ? lse2[i + k] : INFINITY;
                const int seen = i + k < n ? limit[i + k] : 0;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (t + e < seen) x[e] += __builtin_amdgcn_exp2f((&y[k].x)[e] - l);
            }
            ask(r0 + i + 4);
        }
    }
    if (t >= L) return;
    if (t + 4 <= L) {
        float4* const to = (float4*)w;
        const float4 was = a.decay == 0.f ? float4{0.f, 0.f, 0.f, 0.f} : *to;
        *to = float4{x[0] + a.decay * was.x, x[1] + a.decay * was.y, x[2] + a.decay * was.z, x[3] + a.decay * was.w};
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (t + e < L) w[e] = a.decay == 0.f ? x[e] : a.decay * w[e] + x[e];
}

// ---- eviction

struct EvictArgs {
    CacheView from, to;
    const float* W;
    float* W_to;
    int* kept;
    int B, Hkv, d, budget, recent;
    int row_magic;                 // 2^20 / (d / 16) + 1: a piece's row without a division
    __device__ __forceinline__ int by_row(int q) const { return (int)((uint32_t)q * (uint32_t)row_magic >> 20); }      // q / (d / 16), q < 2^11
};

constexpr int kSelectThreads = 1024;
// A key is a weight's bits in an order of whole numbers (NaN highest, -0 as 0).
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}
// Inclusive prefix sums over a wavefront.
__device__ __forceinline__ int wave_prefix(int x, int lane) {
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
        const int y = __shfl_up(x, s);
        if (lane >= s) x += y;
    }
    return x;
}
// Which tokens of a sequence and head stay, one workgroup each: the least key that does, digit by digit from the highest (11, 11 and
// 10 bits, counted in LDS), then one pass in slot order.  Keys are held in registers, kSelectKeys per thread, and read again
// for every digit only where the sequence is longer than that.  Bound by the chain of its steps: 128 of up to 8190 tokens 12.4 us, two of
// 1100 11 us (21.6 and 12.3 with the keys read for every digit and one wavefront summing the counts).
constexpr int kSelectKeys = 8;
static __global__ __launch_bounds__(kSelectThreads) void cache_select_kernel(EvictArgs a) {
    constexpr int BINS = 2048, WAVES = kSelectThreads / 64, CHUNK = kSelectThreads * kSelectKeys;
    __shared__ int bins[BINS];
    __shared__ int wsum[WAVES];
    __shared__ int above[kSelectKeys * WAVES], equal[kSelectKeys * WAVES];
    __shared__ int found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int hk = blockIdx.x % a.Hkv, b = blockIdx.x / a.Hkv;
    const int L = a.from.lengths[b], page = a.from.page;
    int* const kept = a.kept + ((long long)b * a.Hkv + hk) * a.budget;
    bool bad = L < 0 || L > a.from.max_len;
    const int keep = bad ? 0 : L < a.budget ? L : a.budget;
    const float* const w = a.W + ((long long)b * a.Hkv + hk) * a.from.max_pages * page;
    float* const w_to = a.W_to + ((long long)b * a.Hkv + hk) * a.to.max_pages * page;
    const int recent = keep < a.recent ? keep : a.recent, n = bad ? 0 : L - recent, k = keep - recent;      // k of the first n
    float x[kSelectKeys];
    auto load = [&](int c) {
#pragma unroll
        for (int r = 0; r < kSelectKeys; ++r) {
            const int i = c * CHUNK + r * kSelectThreads + tid;
            x[r] = i < n ? w[i] : 0.f;
        }
    };
    load(0);
    if (!bad) {
        for (int i = tid; i < (L + page - 1) / page; i += kSelectThreads) {
            const int id = a.from.table[(long long)b * a.from.max_pages + i];
            bad |= id < 0 || id >= a.from.pages;
        }
        for (int i = tid; i < (keep + page - 1) / page; i += kSelectThreads) {
            const int id = a.to.table[(long long)b * a.to.max_pages + i];
            bad |= id < 0 || id >= a.to.pages;
        }
    }
    for (int i = tid; i < BINS; i += kSelectThreads) bins[i] = 0;
    bad = __syncthreads_or(bad) != 0;
    if (tid == 0 && hk == 0) a.to.lengths[b] = bad ? -1 : keep;
    for (int i = (bad ? 0 : keep) + tid; i < a.budget; i += kSelectThreads) kept[i] = -1;
    if (bad) return;
    for (int i = tid; i < recent; i += kSelectThreads) {
        kept[k + i] = n + i;
        w_to[k + i] = w[n + i];
    }
    if (k <= 0) return;

    // the k-th largest key: its bits found so far, how many of the keys that have them are still to be taken
    const int chunks = (n + CHUNK - 1) / CHUNK;
    const bool all = k >= n;
    uint32_t prefix = 0;
    int need = k, low = 0;                           // (low: the bits not looked at, where all keys with the others' value are taken)
    if (!all) {
        int bits = 0;
        for (int pass = 0; pass < 3; ++pass) {
            const int width = pass < 2 ? 11 : 10, shift = 32 - bits - width;
            for (int c = 0; c < chunks; ++c) {
                if (chunks > 1) load(c);
#pragma unroll
                for (int r = 0; r < kSelectKeys; ++r) {
                    const uint32_t key = weight_key(x[r]);
                    if (c * CHUNK + r * kSelectThreads + tid < n && (bits == 0 || (key >> (32 - bits)) == prefix)) atomicAdd(&bins[(key >> shift) & ((1u << width) - 1u)], 1);
                }
            }
            __syncthreads();
            // from the highest bin down, two (one) a thread: the thread whose bins hold the place says where it is
            const int per = (1 << width) / kSelectThreads, top = (1 << width) - 1 - tid * per;
            const int c0 = bins[top], c1 = per == 2 ? bins[top - 1] : 0, mine = c0 + c1, up_to = wave_prefix(mine, lane);
            if (lane == 63) wsum[wave] = up_to;
            __syncthreads();
            int before = up_to - mine;
#pragma unroll
            for (int v = 0; v < WAVES; ++v) before += v < wave ? wsum[v] : 0;
            bins[top] = 0;
            if (per == 2) bins[top - 1] = 0;
            if (before < need && before + mine >= need) {
                const bool second = before + c0 < need;
                found[0] = second ? top - 1 : top;
                found[1] = need - before - (second ? c0 : 0);
                found[2] = second ? c1 : c0;
            }
            __syncthreads();
            prefix = (prefix << width) | (uint32_t)found[0];
            need = found[1];
            bits += width;
            low = 32 - bits;
            if (need == found[2]) break;
        }
    }
    // in slot order: keys above the k-th, and the first `need` of those equal to it
    int at_above = 0, at_equal = 0;
    const unsigned long long below = (1ull << lane) - 1ull;
    for (int c = 0; c < chunks; ++c) {
        if (chunks > 1) load(c);
        unsigned long long ma[kSelectKeys], me[kSelectKeys];
        if (c) __syncthreads();
#pragma unroll
        for (int r = 0; r < kSelectKeys; ++r) {
            const bool in = c * CHUNK + r * kSelectThreads + tid < n;
            const uint32_t key = weight_key(x[r]) >> low;
            ma[r] = __ballot(in && (all || key > prefix));
            me[r] = __ballot(in && !all && key == prefix);
            if (lane == 0) { above[r * WAVES + wave] = __popcll(ma[r]); equal[r * WAVES + wave] = __popcll(me[r]); }
        }
        __syncthreads();
        if (wave < 2) {      // exclusive sums over the kSelectKeys * WAVES = 128 counts
            int* const p = wave == 0 ? above : equal;
            const int x0 = p[2 * lane], x1 = p[2 * lane + 1], up_to = wave_prefix(x0 + x1, lane);
            p[2 * lane] = up_to - x0 - x1;
            p[2 * lane + 1] = up_to - x1;
            if (lane == 63) wsum[wave] = up_to;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kSelectKeys; ++r) {
            const int ra = at_above + above[r * WAVES + wave] + __popcll(ma[r] & below), re = at_equal + equal[r * WAVES + wave] + __popcll(me[r] & below);
            const bool is_above = (ma[r] >> lane) & 1, is_equal = (me[r] >> lane) & 1;
            if (is_above || (is_equal && re < need)) {
                const int p = ra + (re < need ? re : need);
                kept[p] = c * CHUNK + r * kSelectThreads + tid;
                w_to[p] = x[r];
            }
        }
        at_above += wsum[0];
        at_equal += wsum[1];
    }
}

// A workgroup per destination block and tensor: gathers its tokens' codes, each under its source's scale, and rounds them to
// the block's own.  K's rows come straight into registers.  V's tokens lie a byte each in lines that hold a page's other tokens
// too, so the source pages pass through LDS whole, two at a time (one where they are large), and a thread picks 16 tokens of
// a feature from there; the codes are held until the block's scale is known.  Bound by memory: what is kept once in and once
// out, and the rest of V's source pages: 112 615 tokens, 8 heads, d 128, cut to 65 536: 182 MB in and 134 out in 107 us, 2.9 TB/s;
// a workgroup of V takes 11 us, 4 of them the wait for its first source pages, and six fit a CU.
constexpr int gather_page_bytes(int d, int page) { return d * (page + 16); }
constexpr int gather_pages(int d, int page) { return 2 * gather_page_bytes(d, page) <= 40 * 1024 ? 2 : 1; }
__device__ __forceinline__ float largest_code(uint32_t w) {      // (the maximum passes over NaN)
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return fmaxf(fmaxf(fabsf(lo[0]), fabsf(lo[1])), fmaxf(fabsf(hi[0]), fabsf(hi[1])));
}
template <int NI>      // 16-byte pieces per thread; (six workgroups per CU: 109 us where five take 120, 112 k tokens cut to half)
__global__ __launch_bounds__(256, NI <= 2 ? 6 : NI == 4 ? 3 : 1) void cache_gather_kernel(EvictArgs a) {
    extern __shared__ uint4 staged[];
    __shared__ long long src_block[128];      // page * Hkv + head
    __shared__ int src_slot[128];             // K: slot in the source page; V: its byte among the staged rows of its round
    __shared__ int page_at[128 + 1];          // first token of each different source page
    __shared__ float src_scale[128];
    __shared__ float red[4];
    __shared__ int different, in_first;
    const int tid = threadIdx.x, lane = tid & 63, page = a.from.page, d = a.d;
    const int b = blockIdx.y, both = blockIdx.x / a.Hkv, hk = blockIdx.x - both * a.Hkv, is_v = both & 1, j = both >> 1;
    const int* const kept = a.kept + ((long long)b * a.Hkv + hk) * a.budget + (long long)j * page;
    const int* const table = a.from.table + (long long)b * a.from.max_pages;
    // (the slots are asked for before it is known how many there are: -1 behind them)
    const int t = tid < page && j * page + tid < a.budget ? kept[tid] : -1;
    const int keep = a.to.lengths[b], to_page = a.to.table[(long long)b * a.to.max_pages + j];
    if (j * page >= keep) return;             // (-1: nothing)
    const int n = keep - j * page < page ? keep - j * page : page;
    const long long size = (long long)page * d, dst = (long long)to_page * a.Hkv + hk;
    const int at_once = gather_pages(d, page), page_bytes = gather_page_bytes(d, page), pitch = page + 16;
    const int p0 = t >> a.from.log_page;
    float scale = 0.f;                        // (behind the last token: codes 0, which count for nothing)
    if (tid < n) {
        const long long block = (long long)table[p0] * a.Hkv + hk;
        src_block[tid] = block;
        src_slot[tid] = t & (page - 1);
        scale = (is_v ? a.from.Vs : a.from.Ks)[block];
    }
    uint4 w[NI];
    float most = 0.f;
    if (!is_v) {
        __syncthreads();
#pragma unroll
        for (int p = 0; p < NI; ++p) {
            const int q = p * 256 + tid, i = a.by_row(q), f = (q - i * (d / 16)) * 16;
            w[p] = i < n ? *(const uint4*)(a.from.K + src_block[i] * size + (long long)src_slot[i] * d + f) : uint4{0u, 0u, 0u, 0u};
        }
        if (tid < page) src_scale[tid] = scale;
        __syncthreads();
#pragma unroll
        for (int p = 0; p < NI; ++p) {
            const int i = a.by_row(p * 256 + tid);
            if (i < n) most = fmaxf(most, src_scale[i] * fmaxf(fmaxf(largest_code(w[p].x), largest_code(w[p].y)), fmaxf(largest_code(w[p].z), largest_code(w[p].w))));
        }
    } else {
        // tokens are in slot order: a new page begins where its number differs from the one before
        const int before = tid < n && tid > 0 ? kept[tid - 1] >> a.from.log_page : -1;
        const unsigned long long starts = __ballot(tid < n && p0 != before);
        if (tid == 0) in_first = __popcll(starts);
        __syncthreads();
        if (tid < n) {
            const int u = __popcll(starts & (lane == 63 ? ~0ull : (2ull << lane) - 1ull)) - 1 + (tid >= 64 ? in_first : 0);
            src_slot[tid] += u % at_once * page_bytes;
            if (p0 != before) page_at[u] = tid;
            if (tid == n - 1) { different = u + 1; page_at[u + 1] = n; }
        }
        __syncthreads();
        const int lg = a.from.log_page - 4, groups = 1 << lg, pieces = d << lg;      // 16-token groups of a feature
#pragma unroll
        for (int p = 0; p < NI; ++p) w[p] = uint4{0u, 0u, 0u, 0u};
        // a round's source pages are asked for while the round before is picked from
        uint4 x0[NI], x1[NI];
        auto page_of_round = [&](int u, uint4 (&x)[NI]) {
            const uint8_t* const src = a.from.V + src_block[page_at[u < different ? u : 0]] * size;
#pragma unroll
            for (int p = 0; p < NI; ++p) {
                const int q = p * 256 + tid;
                x[p] = q < pieces && u < different ? *(const uint4*)(src + q * 16) : uint4{0u, 0u, 0u, 0u};
            }
        };
        auto put = [&](int u, const uint4 (&x)[NI]) {
#pragma unroll
            for (int p = 0; p < NI; ++p) {
                const int q = p * 256 + tid, g = (q & (groups - 1)) * 16, f = q >> lg;
                if (q < pieces) *(uint4*)((uint8_t*)staged + u * page_bytes + f * pitch + g) = x[p];
            }
        };
        page_of_round(0, x0);
        if (at_once == 2) page_of_round(1, x1);
        for (int u0 = 0; u0 < different; u0 += at_once) {
            const int u1 = u0 + at_once < different ? u0 + at_once : different;
            if (u0) __syncthreads();
            put(0, x0);
            if (u1 - u0 == 2) put(1, x1);
            page_of_round(u1, x0);
            if (at_once == 2) page_of_round(u1 + 1, x1);
            if (u0 == 0 && tid < page) src_scale[tid] = scale;
            __syncthreads();
            const int i0 = page_at[u0], i1 = page_at[u1];
#pragma unroll
            for (int p = 0; p < NI; ++p) {
                const int q = p * 256 + tid, g = (q & (groups - 1)) * 16, f = q >> lg;
                if (q >= pieces || g >= i1 || g + 16 <= i0) continue;
                const uint8_t* const src = (const uint8_t*)staged + f * pitch;
                if (g >= i0 && g + 16 <= i1) {       // (most are: no token of the 16 in another round)
                    uint32_t c[16];
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const int4 at = *(const int4*)(src_slot + g + e);
#pragma unroll
                        for (int h = 0; h < 4; ++h) c[e + h] = src[(&at.x)[h]];
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 4) (&w[p].x)[e / 4] = c[e] | c[e + 1] << 8 | c[e + 2] << 16 | c[e + 3] << 24;
                    continue;
                }
#pragma unroll
                for (int e = 0; e < 16; e += 4) {
                    const int4 at = *(const int4*)(src_slot + g + e);
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (g + e + h >= i0 && g + e + h < i1) (&w[p].x)[e / 4] |= (uint32_t)src[(&at.x)[h]] << (8 * h);
                }
            }
        }
#pragma unroll
        for (int p = 0; p < NI; ++p) {
            const int g = ((p * 256 + tid) & (groups - 1)) * 16;
            if (g >= n) continue;
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const float4 s = *(const float4*)(src_scale + g + e);
                const uint32_t x = (&w[p].x)[e / 4];
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
                most = fmaxf(fmaxf(most, fmaxf(fabsf(lo[0]) * s.x, fabsf(lo[1]) * s.y)), fmaxf(fabsf(hi[0]) * s.z, fabsf(hi[1]) * s.w));
            }
        }
    }
    most = wave_max(most);
    if (lane == 0) red[tid >> 6] = most;
    __syncthreads();
    const int ex = scale_exponent(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
    if (tid == 0) (is_v ? a.to.Vs : a.to.Ks)[dst] = pow2f(ex);
    const float inv = pow2f(-ex);
    if (!is_v) {
#pragma unroll
        for (int p = 0; p < NI; ++p) {
            const int q = p * 256 + tid, i = a.by_row(q);
            if (i >= n) continue;
            // (the ratio of two scales may pass the largest float, and 0 times infinity is no code; a code that is not 0 meets none above
            // 448 / 2^-9 < 2^18, since its value counted for the destination)
            const float s = fminf(src_scale[i] * inv, 0x1p127f);
            if (s != 1.f) w[p] = uint4{rescale_codes(w[p].x, s), rescale_codes(w[p].y, s), rescale_codes(w[p].z, s), rescale_codes(w[p].w, s)};
            ((uint4*)(a.to.K + dst * size))[q] = w[p];
        }
        return;
    }
    const int lg = a.from.log_page - 4, groups = 1 << lg, pieces = d << lg;
#pragma unroll
    for (int p = 0; p < NI; ++p) {
        const int q = p * 256 + tid, g = (q & (groups - 1)) * 16;
        if (q >= pieces || g >= n) continue;
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            uint32_t& x = (&w[p].x)[e / 4];
            const float4 s = *(const float4*)(src_scale + g + e);
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
            x = codes_of(lo[0] * inv * s.x, lo[1] * inv * s.y, hi[0] * inv * s.z, hi[1] * inv * s.w);      // (in this order: 0 stays 0, see K's; codes times 2^-120 are floats)
        }
        uint8_t* const out = a.to.V + dst * size + q * 16;
        if (g + 16 <= n) *(uint4*)out = w[p];
        else {
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (g + e < n) out[e] = (uint8_t)((&w[p].x)[e / 4] >> (8 * (e & 3)));
        }
    }
}

}  // namespace csat
