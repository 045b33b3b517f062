// Queries and keys of a step made ready for attention: RMS norm per head, rotation by position, keys and values stored in the
// paged cache, in one pass over the projection's output.
#include "rope_row.h"

namespace jx {

namespace {

// y = x / sqrt(mean(x^2) + eps) * w, then (a, b) -> (a cos - b sin, b cos + a sin) over the first rot_dim elements.
// Bound: bytes.  A group of LPR lanes holds one head's row, eight elements (16 bytes) a lane, so a row is read and written
// once and the norm is a sum over the group; the other half of a rotated pair is in the lane rot_dim / 16 further on (or in
// the same lane where neighbours are paired).  Sums, norm and rotation are in 32 bits, rounded once when stored.  With many
// tokens a group takes ROWS heads of one: as many reads on their way, and the angles once (8,191 tokens of 48 heads of 128
// elements, a call: 46.6 us, with one head a group 52).  The kernel then takes 45 us on inputs that no cache holds, 4.5 TB/s read
// and written; 64 tokens 3.8.
template <typename T, int LPR, int ROWS>
__global__ __launch_bounds__(256) void qk_norm_rope_kernel(jx_rope_args a, int page_shift) {
    typedef typename Vec<T>::x8 X8;
    const int c = threadIdx.x % LPR, c8 = c * 8;
    const int rows = a.n_heads + 2 * a.n_kv_heads, groups = (rows + ROWS - 1) / ROWS;
    const uint32_t i = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, t = i / groups;
    if (t >= a.n_tokens) return;  // whole groups of LPR lanes
    const int row0 = (int)(i - t * groups) * ROWS;
    const bool inside = c8 < a.head_dim;
    const int pos = a.d_pos[t];
    const int64_t slot = a.d_slot[t];
    const bool placed = (uint32_t)pos < (uint32_t)a.n_pos;
    const bool stored = placed && slot >= 0 && (slot >> page_shift) < a.cache.n_pages;
    const int64_t place = (slot >> page_shift) * a.cache.page_stride + (slot & (a.cache.page - 1)) * a.cache.token_stride;
    X8 raw[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        const int row = row0 + r, kv = row - a.n_heads, v = kv - a.n_kv_heads;
        const T* from = kv < 0  ? (const T*)a.d_q + t * a.q_token_stride + row * a.q_head_stride
                        : v < 0 ? (const T*)a.d_k + t * a.k_token_stride + kv * a.k_head_stride
                                : (const T*)a.d_v + t * a.v_token_stride + v * a.v_head_stride;
        raw[r] = inside && row < rows && (kv < 0 ? placed : stored) ? *(const X8*)(from + c8) : (X8)(T)0.0f;
    }
    const Angles angles = angles_at(a, pos, placed, c);
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        const int row = row0 + r, kv = row - a.n_heads, v = kv - a.n_kv_heads;
        if (v >= 0) {
            if (row < rows && stored && inside) *(X8*)((T*)a.cache.d_v + place + v * a.cache.head_stride + c8) = raw[r];
            continue;
        }
        const f32x8 x = norm_and_turn<T, LPR>(a, __builtin_convertvector(raw[r], f32x8), (const T*)(kv < 0 ? a.d_q_weight : a.d_k_weight), inside, c8, angles);
        T* to = kv < 0 ? (T*)a.d_q_out + ((int64_t)t * a.n_heads + row) * a.head_dim : (T*)a.cache.d_k + place + kv * a.cache.head_stride;
        if (inside && (kv < 0 || stored)) store8(to + c8, placed ? x : (f32x8)0.0f);
    }
}

template <typename T, int LPR>
hipError_t launch(const jx_rope_args& a, hipStream_t st) {
    const unsigned blocks = (unsigned)(rope_threads(a) / 256);
    const int shift = log2_of(a.cache.page);
    if (rope_many(a)) qk_norm_rope_kernel<T, LPR, 4><<<blocks, 256, 0, st>>>(a, shift);
    else qk_norm_rope_kernel<T, LPR, 1><<<blocks, 256, 0, st>>>(a, shift);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_dim(const jx_rope_args& a, hipStream_t st) {
    const int lpr = row_lanes(a.head_dim);
    return lpr == 8 ? launch<T, 8>(a, st) : lpr == 16 ? launch<T, 16>(a, st) : launch<T, 32>(a, st);
}

}  // namespace

hipError_t launch_qk_norm_rope(const jx_rope_args& a, hipStream_t st) {
    return a.dtype == JX_BF16 ? launch_dim<__bf16>(a, st) : launch_dim<_Float16>(a, st);
}

}  // namespace jx
