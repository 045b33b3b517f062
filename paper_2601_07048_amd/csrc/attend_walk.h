// Attention of one query row by a wavefront, over key and value rows that lie anywhere.
#pragma once
#include "attend.h"
#include "jx_device.h"

namespace jx {

// Where a softmax stands: the largest score so far (in units of log2), the sum of 2^(score - m) and of the values so weighted.
// m = -infinity: nothing yet.  Everything is in 32 bits.
struct Softmax {
    float m, l;
    f32x8 acc;
};

__device__ __forceinline__ long long shfl64(long long v, int lane) {
    const int lo = __shfl((int)(uint32_t)v, lane, 64), hi = __shfl((int)(v >> 32), lane, 64);
    return ((long long)hi << 32) | (uint32_t)lo;
}

// Keys i0 .. i1 - 1 for a query whose elements 8 c .. 8 c + 7 (times scale * log2 e) are in q, c = lane % LPR: 64 / LPR keys at a
// time, one per group of LPR lanes.  where(i) = elements from k and v to row i, or < 0 where the key is masked: such rows are not
// read, so whatever is in them has no part in the result.  Each group of lanes has a Softmax of its own; see `gather`.
template <typename T, int LPR, typename Where>
__device__ __forceinline__ Softmax walk_keys(const T* k, const T* v, f32x8 q, bool inside, long long i0, long long i1, Where where) {
    constexpr int AT_ONCE = 64 / LPR, U = 4;
    typedef typename Vec<T>::x8 X8;
    const int lane = lane_id(), c8 = lane % LPR * 8, group = lane / LPR;
    Softmax s = {-INFINITY, 0.0f, {0, 0, 0, 0, 0, 0, 0, 0}};
    for (; i0 < i1; i0 += 64) {
        const long long mine = i0 + lane < i1 ? where(i0 + lane) : -1;
        const int n = (int)min(64ll, i1 - i0);
        for (int j = 0; j < n; j += U * AT_ONCE) {
            X8 kx[U], vx[U];
            bool seen[U];
            for (int u = 0; u < U; u++) {
                const long long at = shfl64(mine, (j + u * AT_ONCE + group) & 63);
                seen[u] = at >= 0 && j + u * AT_ONCE < 64;
                const bool read = seen[u] && inside;
                kx[u] = read ? *(const X8*)(k + at + c8) : (X8)(T)0.0f;
                vx[u] = read ? *(const X8*)(v + at + c8) : (X8)(T)0.0f;
            }
            float sc[U], top = s.m;
            for (int u = 0; u < U; u++) {
                const f32x8 x = __builtin_convertvector(kx[u], f32x8);
                float d = 0.0f;
                for (int e = 0; e < 8; e++) d = fmaf(x[e], q[e], d);
                d = group_sum<LPR>(d);
                sc[u] = seen[u] ? d : -INFINITY;
                top = fmaxf(top, sc[u]);
            }
            const float base = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(s.m - base);
            s.m = top;
            s.l *= keep;
            for (int e = 0; e < 8; e++) s.acc[e] *= keep;
            for (int u = 0; u < U; u++) {
                const float p = __builtin_amdgcn_exp2f(sc[u] - base);
                const f32x8 x = __builtin_convertvector(vx[u], f32x8);
                s.l += p;
                for (int e = 0; e < 8; e++) s.acc[e] = fmaf(p, x[e], s.acc[e]);
            }
        }
    }
    return s;
}

// The groups' softmaxes as one, in every group
template <int LPR>
__device__ __forceinline__ Softmax gather(Softmax s) {
    float top = s.m;
    for (int d = LPR; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d, 64));
    const float w = __builtin_amdgcn_exp2f(s.m - (top == -INFINITY ? 0.0f : top));
    s.m = top;
    s.l *= w;
    for (int e = 0; e < 8; e++) s.acc[e] *= w;
    for (int d = LPR; d < 64; d *= 2) {
        s.l += __shfl_xor(s.l, d, 64);
        for (int e = 0; e < 8; e++) s.acc[e] += __shfl_xor(s.acc[e], d, 64);
    }
    return s;
}

}  // namespace jx
