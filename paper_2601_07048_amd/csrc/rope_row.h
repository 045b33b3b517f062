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

// y = x / sqrt(mean(x^2) + eps) * w (NULL: y = x), then (a, b) -> (a cos - b sin, b cos + a sin)
template <typename T, int LPR>
__device__ __forceinline__ f32x8 norm_and_turn(const jx_rope_args& a, f32x8 x, const T* w, bool inside, int c8, const Angles& g) {
    if (w) {
        float s = 0.0f;
        for (int j = 0; j < 8; j++) s = fmaf(x[j], x[j], s);
        s = group_sum<LPR>(s);
        const float n = 1.0f / sqrtf(s / (float)a.head_dim + a.eps);
        f32x8 y = {0, 0, 0, 0, 0, 0, 0, 0};
        if (inside) y = load8(w + c8);
        for (int j = 0; j < 8; j++) x[j] = x[j] * n * y[j];
    }
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

}  // namespace jx
