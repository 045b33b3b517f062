// Queries and keys of a step made ready for attention: RMS norm per head, rotation by position, keys and values stored in the
// paged cache, in one pass over the projection's output.
#include "attend.h"
#include "jx_device.h"

namespace jx {

namespace {

// y = x / sqrt(mean(x^2) + eps) * w, then (a, b) -> (a cos - b sin, b cos + a sin) over the first rot_dim elements.
// Bound: bytes.  A group of LPR lanes holds one head's row, eight elements (16 bytes) a lane, so a row is read and written
// once and the norm is a sum over the group; the other half of a rotated pair is in the lane rot_dim / 16 further on (or in
// the same lane where neighbours are paired).  Sums, norm and rotation are in 32 bits, rounded once when stored.
template <typename T, int LPR>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(jx_rope_args a, int page_shift) {
    const int c = threadIdx.x % LPR;
    const int rows = a.n_heads + 2 * a.n_kv_heads;
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / LPR;
    const long long t = i / rows;
    if (t >= a.n_tokens) return;  // whole groups of LPR lanes
    const int row = (int)(i - t * rows);
    const bool is_q = row < a.n_heads, is_v = row >= a.n_heads + a.n_kv_heads;
    const int head = is_q ? row : is_v ? row - a.n_heads - a.n_kv_heads : row - a.n_heads;
    const bool inside = c * 8 < a.head_dim;
    const int pos = a.d_pos[t];
    const bool placed = (uint32_t)pos < (uint32_t)a.n_pos;
    T* to;
    if (is_q) {
        to = (T*)a.d_q_out + (t * a.n_heads + head) * a.head_dim;
    } else {
        const int64_t slot = a.d_slot[t];
        if (!placed || slot < 0 || (slot >> page_shift) >= a.cache.n_pages) return;
        to = (T*)(is_v ? a.cache.d_v : a.cache.d_k) + (slot >> page_shift) * a.cache.page_stride +
             (slot & (a.cache.page - 1)) * a.cache.token_stride + head * a.cache.head_stride;
    }
    f32x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (inside && placed) {
        const T* from = is_q   ? (const T*)a.d_q + t * a.q_token_stride + head * a.q_head_stride
                        : is_v ? (const T*)a.d_v + t * a.v_token_stride + head * a.v_head_stride
                               : (const T*)a.d_k + t * a.k_token_stride + head * a.k_head_stride;
        x = load8(from + c * 8);
    }
    if (!is_v && placed) {
        const T* w = (const T*)(is_q ? a.d_q_weight : a.d_k_weight);
        if (w) {
            float s = 0.0f;
            for (int j = 0; j < 8; j++) s = fmaf(x[j], x[j], s);
            s = group_sum<LPR>(s);
            const float r = 1.0f / sqrtf(s / (float)a.head_dim + a.eps);
            if (inside) {
                const f32x8 g = load8(w + c * 8);
                for (int j = 0; j < 8; j++) x[j] = x[j] * r * g[j];
            }
        }
        const int half = a.rot_dim / 2;
        const float* cs = a.d_cos + (size_t)pos * half;
        const float* sn = a.d_sin + (size_t)pos * half;
        if (a.interleaved) {
            if (c * 8 < a.rot_dim) {
                const f32x4 co = *(const f32x4*)(cs + c * 4), si = *(const f32x4*)(sn + c * 4);
                for (int j = 0; j < 4; j++) {
                    const float u = x[2 * j], v = x[2 * j + 1];
                    x[2 * j] = fmaf(u, co[j], -(v * si[j]));
                    x[2 * j + 1] = fmaf(v, co[j], u * si[j]);
                }
            }
        } else {
            const int step = half / 8;
            const bool low = c < step, turns = c < 2 * step;
            const int from = lane_id() + (low ? step : turns ? -step : 0);
            f32x8 y;
            for (int j = 0; j < 8; j++) y[j] = __shfl(x[j], from, 64);
            if (turns) {
                const int f = (low ? c : c - step) * 8;
                const f32x8 co = *(const f32x8*)(cs + f), si = *(const f32x8*)(sn + f);
                for (int j = 0; j < 8; j++) x[j] = fmaf(x[j], co[j], low ? -(y[j] * si[j]) : y[j] * si[j]);
            }
        }
    }
    if (inside) store8(to + c * 8, x);
}

template <typename T>
hipError_t launch(const jx_rope_args& a, hipStream_t st) {
    const int lpr = row_lanes(a.head_dim);
    const long long threads = a.n_tokens * (a.n_heads + 2 * a.n_kv_heads) * lpr;
    const unsigned blocks = (unsigned)((threads + 255) / 256);
    const int shift = log2_of(a.cache.page);
    if (lpr == 8) qk_norm_rope_kernel<T, 8><<<blocks, 256, 0, st>>>(a, shift);
    else if (lpr == 16) qk_norm_rope_kernel<T, 16><<<blocks, 256, 0, st>>>(a, shift);
    else qk_norm_rope_kernel<T, 32><<<blocks, 256, 0, st>>>(a, shift);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(const jx_rope_args& a, hipStream_t st) {
    return a.dtype == JX_BF16 ? launch<__bf16>(a, st) : launch<_Float16>(a, st);
}

}  // namespace jx
