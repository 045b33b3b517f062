// Attention over rows of 8 bits that a search returned, joined with attention over other keys.
#include "codes8.h"

namespace jx {

namespace {

// As found_attention_kernel, with half the bytes to gather: 16 codes a lane, so that 4, 8 or 16 lanes hold a row.  The scales stand
// beside the scores and the weights, in 32 bits.
// Bound: the gathers.  1,000 tokens, 32 heads, 100 rows of 128 codes from 2 GB: 188 us, 4.4 TB/s, where gathers of 128 bytes with nothing to
// do beside them reach 4.5 (rows of 256 bytes 5.4: half the bytes are two thirds of the time); 16 tokens and 10 rows 5.6 us.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void found_attention8_kernel(jx_found_args a, Scales sc) {
    constexpr int N = 16;
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long t = i / a.n_heads;
    if (t >= a.n_tokens) return;
    const int h = (int)(i - t * a.n_heads), lane = lane_id(), c = lane % LPR * N;
    const bool inside = c < a.head_dim;
    float q[N];
    for (int b = 0; b < N; b += 8) {
        f32x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (inside) x = load8((const T*)a.d_q + t * a.q_token_stride + h * a.q_head_stride + c + b);
        for (int e = 0; e < 8; e++) q[b + e] = x[e] * (a.scale * LOG2E);
    }
    const int head = h / (a.n_heads / a.n_kv_heads);
    const long long off = head * a.head_stride;
    const uint32_t* ids = a.d_ids + i * a.k;
    SoftmaxCodes<N> s = walk_codes<LPR, N>((const uint8_t*)a.d_keys + off, (const uint8_t*)a.d_values + off, q, inside, 0, a.k, [&](long long j) {
        const uint32_t id = ids[j];
        if ((long long)id >= a.n_rows) return RowCodes{-1, 0.0f, 0.0f};
        const long long x = (long long)(id >> sc.shift) * a.n_kv_heads + head;
        return RowCodes{(long long)id * a.row_stride, scale_value(sc.k[x]), scale_value(sc.v[x])};
    });
    gather_codes<LPR>(s);
    float top = s.m, before = -INFINITY;
    if (a.d_part_lse) {
        before = a.d_part_lse[i] * LOG2E;
        top = fmaxf(top, before);
    }
    const float base = top == -INFINITY ? 0.0f : top;
    const float w = __builtin_amdgcn_exp2f(s.m - base), wb = __builtin_amdgcn_exp2f(before - base);
    const float l = s.l * w + wb;
    const float r = l == 0.0f ? 0.0f : 1.0f / l;
    if (lane < LPR && inside)
        for (int b = 0; b < N; b += 8) {
            f32x8 o;
            for (int e = 0; e < 8; e++) o[e] = s.acc[b + e] * w;
            if (before != -INFINITY) {
                const f32x8 p = load8((const T*)a.d_part_out + i * a.head_dim + c + b);
                for (int e = 0; e < 8; e++) o[e] = fmaf(p[e], wb, o[e]);
            }
            for (int e = 0; e < 8; e++) o[e] *= r;
            store8((T*)a.d_out + i * a.head_dim + c + b, o);
        }
    if (lane == 0 && a.d_lse) a.d_lse[i] = l == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * LN2;
}

template <typename T>
hipError_t launch(const jx_found_args& a, const Scales& sc, hipStream_t st) {
    const unsigned blocks = (unsigned)(found_threads(a) / 256);
    if (a.head_dim <= 64) found_attention8_kernel<T, 4><<<blocks, 256, 0, st>>>(a, sc);
    else if (a.head_dim <= 128) found_attention8_kernel<T, 8><<<blocks, 256, 0, st>>>(a, sc);
    else found_attention8_kernel<T, 16><<<blocks, 256, 0, st>>>(a, sc);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_found_attention8(const jx_found_args& a, const jx_kv_scales& s, hipStream_t st) {
    const Scales sc = {s.d_k, s.d_v, log2_of(s.block), 0};
    return a.dtype == JX_BF16 ? launch<__bf16>(a, sc, st) : launch<_Float16>(a, sc, st);
}

}  // namespace jx
