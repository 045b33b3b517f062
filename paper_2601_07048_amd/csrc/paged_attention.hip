// Attention of a step's new tokens over a paged cache.
#include "attend_walk.h"

namespace jx {

namespace {

// The request of row t (of those that begin at or before it, the last), or -1 for a row that belongs to none
__device__ __forceinline__ int request_of(const int32_t* q_start, int n_req, long long t) {
    if (n_req == 0 || t < q_start[0] || t >= q_start[n_req]) return -1;
    int lo = 0, hi = n_req;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (q_start[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// One (token, head) a wavefront; see walk_keys
template <typename T, int LPR>
__global__ __launch_bounds__(256) void paged_rows_kernel(jx_attend_args a, int page_shift) {
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long t = i / a.n_heads;
    if (t >= a.n_tokens) return;
    const int h = (int)(i - t * a.n_heads), lane = lane_id(), c8 = lane % LPR * 8;
    const bool inside = c8 < a.head_dim;
    f32x8 q = {0, 0, 0, 0, 0, 0, 0, 0};
    if (inside) q = load8((const T*)a.d_q + t * a.q_token_stride + h * a.q_head_stride + c8);
    const float scale = a.scale * LOG2E;
    for (int e = 0; e < 8; e++) q[e] *= scale;
    long long i0 = 0, i1 = 0;
    const int r = request_of(a.d_q_start, a.n_req, t);
    const int32_t* table = a.d_table;
    if (r >= 0) {
        const long long pos = (long long)a.d_kv_len[r] - (a.d_q_start[r + 1] - t);
        i1 = min(pos + 1, (long long)a.table_pages << page_shift);
        i0 = a.window ? max(pos + 1 - a.window, 0ll) : 0;
        table += (size_t)r * a.table_pages;
    }
    const long long off = h / (a.n_heads / a.n_kv_heads) * a.cache.head_stride;
    Softmax s = walk_keys<T, LPR>((const T*)a.cache.d_k + off, (const T*)a.cache.d_v + off, q, inside, i0, i1, [&](long long p) {
        const int32_t id = table[p >> page_shift];
        return (uint32_t)id < (uint32_t)a.cache.n_pages
                   ? id * a.cache.page_stride + (p & (a.cache.page - 1)) * a.cache.token_stride : -1ll;
    });
    s = gather<LPR>(s);
    const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;
    if (lane < LPR && inside) {
        for (int e = 0; e < 8; e++) s.acc[e] *= inv;
        store8((T*)a.d_out + i * a.head_dim + c8, s.acc);
    }
    if (lane == 0 && a.d_lse) a.d_lse[i] = s.l == 0.0f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * LN2;
}

template <typename T>
hipError_t launch(const jx_attend_args& a, hipStream_t st) {
    const unsigned blocks = (unsigned)((a.n_tokens * a.n_heads + 3) / 4);
    const int lpr = row_lanes(a.head_dim), shift = log2_of(a.cache.page);
    if (lpr == 8) paged_rows_kernel<T, 8><<<blocks, 256, 0, st>>>(a, shift);
    else if (lpr == 16) paged_rows_kernel<T, 16><<<blocks, 256, 0, st>>>(a, shift);
    else paged_rows_kernel<T, 32><<<blocks, 256, 0, st>>>(a, shift);
    return hipGetLastError();
}

}  // namespace

int64_t paged_attention_bytes(const jx_attend_args&) { return 0; }

hipError_t launch_paged_attention(const jx_attend_args& a, uint8_t*, hipStream_t st) {
    return a.dtype == JX_BF16 ? launch<__bf16>(a, st) : launch<_Float16>(a, st);
}

}  // namespace jx
