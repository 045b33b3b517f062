// Norm and rotation of one head's row: a group of LPR lanes holds it, eight elements a lane.
#pragma once
#include "attend.h"
#include "jx_device.h"

namespace jx {

// What a lane needs of the angles of a token's position: of four pairs, or of the eight elements beside those of the other half, which
// the lane `other` holds
struct Angles {
    f32x8 co, si;
    bool turns;
    int other;
};

__device__ __forceinline__ Angles angles_at(const jx_rope_args& a, int pos, bool placed, int c) {
    const int half = a.rot_dim / 2, step = half / 8, c8 = c * 8;
    const bool low = c < step;
    Angles g = {{1, 1, 1, 1, 1, 1, 1, 1}, {0, 0, 0, 0, 0, 0, 0, 0}, placed && c8 < a.rot_dim, 0};
    if (g.turns) {
        const float *cs = a.d_cos + (size_t)pos * half, *sn = a.d_sin + (size_t)pos * half;
        if (a.interleaved) {
            for (int j = 0; j < 4; j++) {
                g.co[j] = cs[c * 4 + j];
                g.si[j] = sn[c * 4 + j];
            }
        } else {
            g.co = *(const f32x8*)(cs + (low ? c : c - step) * 8);
            g.si = *(const f32x8*)(sn + (low ? c : c - step) * 8);
            if (low)
                for (int j = 0; j < 8; j++) g.si[j] = -g.si[j];
        }
    }
    g.other = lane_id() + (low ? step : c8 < a.rot_dim ? -step : 0);
    return g;
}

__device__ __forceinline__ float sum_of_squares(f32x8 x) {
    float s = 0.0f;
    for (int j = 0; j < 8; j++) s = fmaf(x[j], x[j], s);
    return s;
}

// 1 / sqrt(mean square + eps) from the row's sum of squares
__device__ __forceinline__ float row_norm(const jx_rope_args& a, float s) { return 1.0f / sqrtf(s / (float)a.head_dim + a.eps); }

// The same of N rows that the lanes hold: square root and divisions are as dear as all else of a row, so each lane of four works out one
template <int N>
__device__ __forceinline__ void row_norms(const jx_rope_args& a, float (&s)[N]) {
    if constexpr (N == 1) {
        s[0] = row_norm(a, s[0]);
    } else if constexpr (N == 2) {
        const int n = __float_as_int(row_norm(a, lane_id() & 1 ? s[1] : s[0]));
        s[0] = __int_as_float(__builtin_amdgcn_update_dpp(0, n, 0xA0, 0xF, 0xF, true));  // quad_perm [0,0,2,2]
        s[1] = __int_as_float(__builtin_amdgcn_update_dpp(0, n, 0xF5, 0xF, 0xF, true));  // quad_perm [1,1,3,3]
    } else {
        static_assert(N % 4 == 0, "rows in fours");
        for (int r = 0; r < N; r += 4) {
            const float lo = lane_id() & 1 ? s[r + 1] : s[r], hi = lane_id() & 1 ? s[r + 3] : s[r + 2];
            const int n = __float_as_int(row_norm(a, lane_id() & 2 ? hi : lo));
            s[r] = __int_as_float(__builtin_amdgcn_update_dpp(0, n, 0x00, 0xF, 0xF, true));
            s[r + 1] = __int_as_float(__builtin_amdgcn_update_dpp(0, n, 0x55, 0xF, 0xF, true));
            s[r + 2] = __int_as_float(__builtin_amdgcn_update_dpp(0, n, 0xAA, 0xF, 0xF, true));
            s[r + 3] = __int_as_float(__builtin_amdgcn_update_dpp(0, n, 0xFF, 0xF, 0xF, true));
        }
    }
}

// (a, b) -> (a cos - b sin, b cos + a sin)
__device__ __forceinline__ f32x8 turned(const jx_rope_args& a, f32x8 x, const Angles& g) {
    if (a.interleaved) {
        for (int j = 0; j < 4; j++) {
            const float p = x[2 * j], q = x[2 * j + 1];
            x[2 * j] = g.turns ? fmaf(p, g.co[j], -(q * g.si[j])) : p;  // not by an angle of 0: 0 times an infinity is NaN
            x[2 * j + 1] = g.turns ? fmaf(q, g.co[j], p * g.si[j]) : q;
        }
    } else {
        f32x8 y;
        for (int j = 0; j < 8; j++) y[j] = __shfl(x[j], g.other, 64);
        for (int j = 0; j < 8; j++) x[j] = g.turns ? fmaf(x[j], g.co[j], y[j] * g.si[j]) : x[j];
    }
    return x;
}

// y = x / sqrt(mean(x^2) + eps) * w (NULL: y = x), turned
template <typename T, int LPR>
__device__ __forceinline__ f32x8 norm_and_turn(const jx_rope_args& a, f32x8 x, const T* w, bool inside, int c8, const Angles& g) {
    if (w) {
        const float n = row_norm(a, group_sum<LPR>(sum_of_squares(x)));
        f32x8 y = {0, 0, 0, 0, 0, 0, 0, 0};
        if (inside) y = load8(w + c8);
        for (int j = 0; j < 8; j++) x[j] = x[j] * n * y[j];
    }
    return turned(a, x, g);
}

// The same of N rows, the weights read once
template <typename T, int LPR, int N>
__device__ __forceinline__ void norm_rows(const jx_rope_args& a, f32x8 (&x)[N], const T* w, bool inside, int c8) {
    if (!w) return;
    f32x8 y = {0, 0, 0, 0, 0, 0, 0, 0};
    if (inside) y = load8(w + c8);
    float n[N];
    for (int r = 0; r < N; r++) n[r] = group_sum<LPR>(sum_of_squares(x[r]));
    row_norms<N>(a, n);
    for (int r = 0; r < N; r++)
        for (int j = 0; j < 8; j++) x[r][j] = x[r][j] * n[r] * y[j];
}

}  // namespace jx
