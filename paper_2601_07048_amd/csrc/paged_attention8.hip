// Attention of a step's new tokens over a paged cache of 8 bits.
#include "codes8.h"

namespace jx {

namespace {

// A wavefront takes a row (token, head) and walks over the keys that it sees.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void paged_rows8_kernel(jx_attend_args a, Scales sc, int page_shift) {
    constexpr int N = 16;
    const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const long long t = i / a.n_heads;
    if (t >= a.n_tokens) return;
    const int h = (int)(i - t * a.n_heads), lane = lane_id(), c = lane % LPR * N, d = a.head_dim;
    const bool inside = c < d;
    int lo = 0, hi = a.n_req;  // the last request that begins at or before t
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.d_q_start[mid] <= t) lo = mid;
        else hi = mid;
    }
    long long k0 = 0, k1 = 0;
    if (a.n_req && a.d_q_start[lo] <= t && t < a.d_q_start[lo + 1]) {
        const long long p = (long long)a.d_kv_len[lo] - a.d_q_start[lo + 1] + t;
        k1 = min(p + 1, (long long)a.table_pages << page_shift);
        k0 = a.window ? max(p + 1 - a.window, 0ll) : 0;
    }
    float q[N];
    for (int b = 0; b < N; b += 8) {
        f32x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
        if (inside) x = load8((const T*)a.d_q + t * a.q_token_stride + h * a.q_head_stride + c + b);
        for (int e = 0; e < 8; e++) q[b + e] = x[e] * (a.scale * LOG2E);
    }
    const int head = h / (a.n_heads / a.n_kv_heads);
    const long long off = head * a.cache.head_stride;
    const int32_t* table = a.d_table + (size_t)lo * a.table_pages;
    SoftmaxCodes<N> s = walk_codes<LPR, N>((const uint8_t*)a.cache.d_k + off, (const uint8_t*)a.cache.d_v + off, q, inside, k0, k1, [&](long long j) {
        const int id = table[j >> page_shift], place = (int)j & (a.cache.page - 1);
        if ((uint32_t)id >= (uint32_t)a.cache.n_pages) return RowCodes{-1, 0.0f, 0.0f};
        const long long x = ((long long)id * sc.per_page + (place >> sc.shift)) * a.n_kv_heads + head;
        return RowCodes{id * a.cache.page_stride + place * a.cache.token_stride, scale_value(sc.k[x]), scale_value(sc.v[x])};
    });
    gather_codes<LPR>(s);
    const float r = s.l == 0.0f ? 0.0f : 1.0f / s.l;
    if (lane < LPR && inside)
        for (int b = 0; b < N; b += 8) {
            f32x8 o;
            for (int e = 0; e < 8; e++) o[e] = s.acc[b + e] * r;
            store8((T*)a.d_out + i * d + c + b, o);
        }
    if (lane == 0 && a.d_lse) a.d_lse[i] = s.l == 0.0f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * LN2;
}

template <typename T>
hipError_t launch(const jx_attend_args& a, const Scales& sc, hipStream_t st) {
    const unsigned blocks = (unsigned)((a.n_tokens * a.n_heads + 3) / 4);
    const int shift = log2_of(a.cache.page);
    if (a.head_dim <= 64) paged_rows8_kernel<T, 4><<<blocks, 256, 0, st>>>(a, sc, shift);
    else if (a.head_dim <= 128) paged_rows8_kernel<T, 8><<<blocks, 256, 0, st>>>(a, sc, shift);
    else paged_rows8_kernel<T, 16><<<blocks, 256, 0, st>>>(a, sc, shift);
    return hipGetLastError();
}

}  // namespace

int64_t paged_attention8_bytes(const jx_attend_args&, const jx_kv_scales&) { return 0; }

hipError_t launch_paged_attention8(const jx_attend_args& a, const jx_kv_scales& s, uint8_t*, hipStream_t st) {
    const Scales sc = {s.d_k, s.d_v, log2_of(s.block), a.cache.page / s.block};
    return a.dtype == JX_BF16 ? launch<__bf16>(a, sc, st) : launch<_Float16>(a, sc, st);
}

}  // namespace jx
