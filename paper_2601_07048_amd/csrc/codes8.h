// Keys and values of 8 bits: e4m3 codes, and one power of two (e8m0) for each block of tokens and key head.
#pragma once
#include "attend.h"
#include "jx_device.h"

namespace jx {

// Where the scales of a paged cache, or of rows that a search returned, lie: block b, key head h at b * n_kv_heads + h; a page has
// per_page blocks
struct Scales {
    const uint8_t *k, *v;
    int shift, per_page;  // block: 2^shift tokens
};

// 2^(byte - 127) as the conversions take it: they look at the exponent's eight bits alone, 0 being 2^-127 and 255 not a number
__device__ __forceinline__ float scale_bits(uint32_t byte) { return __uint_as_float(byte << 23); }
// ... as a number
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 0 ? 0x00400000u : byte == 255 ? 0x7FC00000u : byte << 23);
}

typedef float f32x2 __attribute__((ext_vector_type(2)));

// Four codes as float32
__device__ __forceinline__ f32x4 codes_f32(uint32_t w) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w, true);
    return (f32x4){lo[0], lo[1], hi[0], hi[1]};
}

// Four values y / scale as codes: to nearest even, multiples of 2^-9 under 2^-6, what is infinite or over 464 as what is not a number
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float scale) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    s16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, w);
}

// Codes c * 2^(from - 127) as codes at the scale `to`
__device__ __forceinline__ uint32_t codes_moved(uint32_t w, float from, float to) {
    const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, from, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, from, true);
    return codes_of(lo[0], lo[1], hi[0], hi[1], to);
}

// Two codes of a word as elements of type T, times the scale: exact where T has the number
template <typename T, bool HIGH>
__device__ __forceinline__ uint32_t codes_pair(uint32_t w, float scale) {
    if constexpr (__is_same(T, __bf16)) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HIGH));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, scale, HIGH));
}

// ---- attention of one row by a wavefront, over rows of codes that lie anywhere ------------------------------------------
struct RowCodes {
    long long at;    // bytes from k and v to a row; < 0: masked, not read
    float k, v;      // its scales
};

template <int N>
struct SoftmaxCodes {
    float m, l, acc[N];
};

// As walk_keys, with N codes (8 or 16) for each of LPR lanes of a row; q times scale * log2 e; where(i): the row of key i
template <int LPR, int N, typename Where>
__device__ __forceinline__ SoftmaxCodes<N> walk_codes(const uint8_t* k, const uint8_t* v, const float (&q)[N], bool inside, long long i0, long long i1,
                                                      Where where) {
    constexpr int AT_ONCE = 64 / LPR, U = N == 8 ? 2 : AT_ONCE >= 8 ? 4 : 8, W = N / 4;
    typedef uint32_t Words __attribute__((ext_vector_type(W)));
    const int lane = lane_id(), c = lane % LPR * N, group = lane / LPR;
    SoftmaxCodes<N> s;
    s.m = -INFINITY;
    s.l = 0.0f;
    for (int e = 0; e < N; e++) s.acc[e] = 0.0f;
    for (; i0 < i1; i0 += 64) {
        const int n = (int)min(64ll, i1 - i0);
        RowCodes mine = {-1, 0.0f, 0.0f};
        if (lane < n) mine = where(i0 + lane);
        const uint32_t lo = (uint32_t)mine.at, hi = (uint32_t)(mine.at >> 32);
        for (int j = 0; j < n; j += U * AT_ONCE) {
            Words kx[U], vx[U];
            float ks[U], vs[U];
            bool seen[U];
            for (int u = 0; u < U; u++) {
                const int from = (j + u * AT_ONCE + group) & 63;
                const long long at = (long long)(uint64_t)((uint64_t)(uint32_t)__shfl((int)hi, from, 64) << 32 | (uint32_t)__shfl((int)lo, from, 64));
                seen[u] = at >= 0 && j + u * AT_ONCE < 64;
                ks[u] = __shfl(mine.k, from, 64);
                vs[u] = __shfl(mine.v, from, 64);  // by all lanes; 0 where the key is masked
                if (!seen[u]) vs[u] = 0.0f;
                const bool read = seen[u] && inside;
                kx[u] = read ? *(const Words*)(k + at + c) : (Words)0u;
                vx[u] = read ? *(const Words*)(v + at + c) : (Words)0u;
            }
            float sc[U], top = s.m;
            for (int u = 0; u < U; u++) {
                float d = 0.0f;
                for (int w = 0; w < W; w++) {
                    const f32x4 x = codes_f32(kx[u][w]);
                    for (int e = 0; e < 4; e++) d = fmaf(x[e], q[w * 4 + e], d);
                }
                d = group_sum<LPR>(d) * ks[u];
                sc[u] = seen[u] ? d : -INFINITY;
                top = fmaxf(top, sc[u]);
            }
            const float base = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(s.m - base);
            s.m = top;
            s.l *= keep;
            for (int e = 0; e < N; e++) s.acc[e] *= keep;
            for (int u = 0; u < U; u++) {
                const float p = __builtin_amdgcn_exp2f(sc[u] - base), y = p * vs[u];
                s.l += p;
                for (int w = 0; w < W; w++) {
                    const f32x4 x = codes_f32(vx[u][w]);
                    for (int e = 0; e < 4; e++) s.acc[w * 4 + e] = fmaf(y, x[e], s.acc[w * 4 + e]);
                }
            }
        }
    }
    return s;
}

// The groups' softmaxes as one, in every group
template <int LPR, int N>
__device__ __forceinline__ void gather_codes(SoftmaxCodes<N>& s) {
    float top = s.m;
    for (int d = LPR; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float w = __builtin_amdgcn_exp2f(s.m - (top == -INFINITY ? 0.0f : top));
    s.m = top;
    s.l *= w;
    for (int e = 0; e < N; e++) s.acc[e] *= w;
    for (int d = LPR; d < 64; d *= 2) {
        s.l += __shfl_xor(s.l, d, 64);
        for (int e = 0; e < N; e++) s.acc[e] += __shfl_xor(s.acc[e], d, 64);
    }
}

}  // namespace jx
