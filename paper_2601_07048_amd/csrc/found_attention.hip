// Attention over the rows that a search returned, joined with attention over other keys.
#include "attend_walk.h"

namespace jx {

namespace {

// out = sum_j softmax(scale q.k_j) v_j over the list of one (token, head).
// Bound: the gathers, two rows of head_dim elements for every entry of every list (nothing is shared: each head has its own list).
// A wavefront takes a list; see walk_keys.  1,000 tokens, 32 heads, 100 rows of 128 elements: 287 us, 5.7 TB/s; 16 tokens and 10
// rows, where the chain from id to row to result is what takes the time: 4.8 us.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void found_attention_kernel(jx_found_args a) {
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long t = i / a.n_heads;
    if (t >= a.n_tokens) return;
    const int h = (int)(i - t * a.n_heads), lane = lane_id(), c8 = lane % LPR * 8;
    const bool inside = c8 < a.head_dim;
    f32x8 q = {0, 0, 0, 0, 0, 0, 0, 0};
    if (inside) q = load8((const T*)a.d_q + t * a.q_token_stride + h * a.q_head_stride + c8);
    const float scale = a.scale * LOG2E;
    for (int e = 0; e < 8; e++) q[e] *= scale;
    const long long off = h / (a.n_heads / a.n_kv_heads) * a.head_stride;
    const uint32_t* ids = a.d_ids + i * a.k;
    Softmax s = walk_keys<T, LPR>((const T*)a.d_keys + off, (const T*)a.d_values + off, q, inside, 0, a.k, [&](long long j) {
        const uint32_t id = ids[j];
        return (long long)id < a.n_rows ? (long long)id * a.row_stride : -1ll;
    });
    s = gather<LPR>(s);
    float top = s.m, before = -INFINITY;
    if (a.d_part_lse) {
        before = a.d_part_lse[i] * LOG2E;
        top = fmaxf(top, before);
    }
    const float base = top == -INFINITY ? 0.0f : top;
    const float w = __builtin_amdgcn_exp2f(s.m - base), wb = __builtin_amdgcn_exp2f(before - base);
    const float l = s.l * w + wb;
    const float r = l == 0.0f ? 0.0f : 1.0f / l;
    if (lane < LPR && inside) {
        f32x8 o;
        for (int e = 0; e < 8; e++) o[e] = s.acc[e] * w;
        if (before != -INFINITY) {
            const f32x8 b = load8((const T*)a.d_part_out + i * a.head_dim + c8);
            for (int e = 0; e < 8; e++) o[e] = fmaf(b[e], wb, o[e]);
        }
        for (int e = 0; e < 8; e++) o[e] *= r;
        store8((T*)a.d_out + i * a.head_dim + c8, o);
    }
    if (lane == 0 && a.d_lse) a.d_lse[i] = l == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * LN2;
}

template <typename T>
hipError_t launch(const jx_found_args& a, hipStream_t st) {
    const unsigned blocks = (unsigned)(found_threads(a) / 256);
    const int lpr = row_lanes(a.head_dim);
    if (lpr == 8) found_attention_kernel<T, 8><<<blocks, 256, 0, st>>>(a);
    else if (lpr == 16) found_attention_kernel<T, 16><<<blocks, 256, 0, st>>>(a);
    else found_attention_kernel<T, 32><<<blocks, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_found_attention(const jx_found_args& a, hipStream_t st) {
    return a.dtype == JX_BF16 ? launch<__bf16>(a, st) : launch<_Float16>(a, st);
}

}  // namespace jx
