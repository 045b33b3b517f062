// Queries and keys of a step made ready for attention over a cache of 8 bits: RMS norm per head, rotation by position, keys and
// values put into their blocks as e4m3 beside one power of two for each block and key head.
#include "codes8.h"
#include "rope_row.h"

namespace jx {

namespace {

// Queries are those of qk_norm_rope_kernel.  Keys (y as there) and values (y = x) of the rows that lie in one block, one head: with
// E = the largest exponent among the new |y|, the scale is 2^(E - 7), or what the block has if that is more and the block has tokens
// in front of the new ones; codes are y / scale, rounded once.  So the largest code is 128 up to 256: e4m3 has as many digits at any power of two, and
// what a block holds moves to a larger scale by its exponents alone, but for numbers under 2^-6 of the scale.
// Bound: bytes for many tokens, the chain slot - row - largest - store for few.  A workgroup takes a run of rows of one block, one
// head, keys or values: LPR lanes a row as for the queries, rows held in registers from their one read to their store, the largest
// through LDS.
struct Args {
    jx_rope_args a;
    uint8_t *k_scale, *v_scale;
    int page_shift, block_shift;
    unsigned q_blocks;  // workgroups for the queries
    int rows;           // rows of a workgroup for keys and values: it takes the runs that begin there
};

template <typename T>
constexpr float LARGEST = __is_same(T, _Float16) ? 0x1.ep15f : 0x1.ep127f;  // the largest code times the largest scale that the type holds

template <typename T, int LPR, int ROWS>
__device__ __forceinline__ void queries(const Args& g) {
    typedef typename Vec<T>::x8 X8;
    const jx_rope_args& a = g.a;
    const int c = threadIdx.x % LPR, c8 = c * 8;
    const int groups = (a.n_heads + ROWS - 1) / ROWS;
    const uint32_t i = blockIdx.x * (256 / LPR) + threadIdx.x / LPR, t = i / groups;
    if (t >= a.n_tokens) return;  // whole groups of LPR lanes
    const int row0 = (int)(i - t * groups) * ROWS;
    const bool inside = c8 < a.head_dim;
    const int pos = a.d_pos[t];
    const bool placed = (uint32_t)pos < (uint32_t)a.n_pos;
    X8 raw[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; r++)
        raw[r] = inside && row0 + r < a.n_heads && placed ? *(const X8*)((const T*)a.d_q + t * a.q_token_stride + (row0 + r) * a.q_head_stride + c8) : (X8)(T)0.0f;
    const Angles angles = angles_at(a, pos, placed, c);
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        const f32x8 x = norm_and_turn<T, LPR>(a, __builtin_convertvector(raw[r], f32x8), (const T*)a.d_q_weight, inside, c8, angles);
        if (inside && row0 + r < a.n_heads) store8((T*)a.d_q_out + ((int64_t)t * a.n_heads + row0 + r) * a.head_dim + c8, placed ? x : (f32x8)0.0f);
    }
}

// ITER: rows of a block / rows that the workgroup holds at a time
template <typename T, int LPR, int ITER>
__device__ __forceinline__ void keys_values(const Args& g, float* red) {
    typedef typename Vec<T>::x8 X8;
    constexpr int AT_ONCE = 256 / LPR;
    const jx_rope_args& a = g.a;
    const int tid = threadIdx.x, lane = lane_id(), c = tid % LPR, c8 = c * 8, mine = tid / LPR;
    const uint32_t i = blockIdx.x - g.q_blocks, roles = 2 * a.n_kv_heads;
    const int64_t t0 = (int64_t)(i / roles) * g.rows;
    const int role = (int)(i % roles), head = role >> 1, block = 1 << g.block_shift;
    const bool key = (role & 1) == 0, inside = c8 < a.head_dim;
    const int64_t token_stride = key ? a.k_token_stride : a.v_token_stride;
    const T* from = (const T*)(key ? a.d_k : a.d_v) + head * (key ? a.k_head_stride : a.v_head_stride) + c8;
    uint8_t* cache = (uint8_t*)(key ? a.cache.d_k : a.cache.d_v) + head * a.cache.head_stride;
    // the block of a row, -1 where it is not stored; the slots of a cache are below 2^43
    auto block_of = [&](int64_t t) -> int64_t {
        if (t < 0 || t >= a.n_tokens) return -1;
        const int64_t slot = a.d_slot[t];
        const bool stored = (uint32_t)a.d_pos[t] < (uint32_t)a.n_pos && slot >= 0 && (slot >> g.page_shift) < a.cache.n_pages;
        return stored ? slot >> g.block_shift : -1;
    };
    const int64_t own = lane < g.rows ? block_of(t0 + lane) : -1, before = lane < g.rows ? block_of(t0 + lane - 1) : -1;
    for (uint64_t begins = ballot(own >= 0 && own != before); begins; begins &= begins - 1) {
        const int64_t t = t0 + __builtin_ctzll(begins);
        const int64_t slot = a.d_slot[t], b = slot >> g.block_shift;
        const uint64_t others = ~ballot(lane < block && block_of(t + lane) == b);
        const int count = others ? __builtin_ctzll(others) : 64;  // rows of the run, at most those of a block
        const int first = (int)(slot & (block - 1));
        uint8_t* scale = (key ? g.k_scale : g.v_scale) + b * a.n_kv_heads + head;
        const uint32_t old = first ? *scale : 0;
        auto place = [&](int64_t s) { return (s >> g.page_shift) * a.cache.page_stride + (s & (a.cache.page - 1)) * a.cache.token_stride + c8; };
        f32x8 x[ITER];
        float most = 0.0f;
#pragma unroll
        for (int r = 0; r < ITER; r++) {
            const int row = r * AT_ONCE + mine;
            const bool there = row < count;
            X8 raw = there && inside ? *(const X8*)(from + (t + row) * token_stride) : (X8)(T)0.0f;
            x[r] = __builtin_convertvector(raw, f32x8);
            if (key) x[r] = norm_and_turn<T, LPR>(a, x[r], (const T*)a.d_k_weight, inside, c8, angles_at(a, there ? a.d_pos[t + row] : 0, there, c));
            for (int j = 0; j < 8; j++) {
                const float y = fabsf(x[r][j]);
                if (y < INFINITY) {  // not what is not a number
                    x[r][j] = fminf(fmaxf(x[r][j], -LARGEST<T>), LARGEST<T>);
                    most = fmaxf(most, fminf(y, LARGEST<T>));
                }
            }
        }
        for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d, 64));
        if (lane == 0) red[tid >> 6] = most;
        __syncthreads();
        most = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
        const uint32_t byte = max(max((int)(__float_as_uint(most) >> 23) - 7, 1), (int)old);
        const float to = scale_bits(byte);
#pragma unroll
        for (int r = 0; r < ITER; r++) {
            const int row = r * AT_ONCE + mine;
            if (row < count && inside) {
                const int64_t s = a.d_slot[t + row];
                const uint2 w = make_uint2(codes_of(x[r][0], x[r][1], x[r][2], x[r][3], to), codes_of(x[r][4], x[r][5], x[r][6], x[r][7], to));
                *(uint2*)(cache + place(s)) = w;
            }
        }
        if (first && byte != old) {
            const int64_t s0 = slot - first;
            for (int row = mine; row < first; row += AT_ONCE)
                if (inside) {
                    uint2* p = (uint2*)(cache + place(s0 + row));
                    const uint2 w = *p;
                    *p = make_uint2(codes_moved(w.x, scale_bits(old), to), codes_moved(w.y, scale_bits(old), to));
                }
        }
        __syncthreads();  // every wavefront has read the old scale and red
        if (tid == 0) *scale = (uint8_t)byte;
    }
}

template <typename T, int LPR, int ROWS, int ITER>
__global__ __launch_bounds__(256) void qk_norm_rope8_kernel(Args g) {
    __shared__ float red[4];
    if (blockIdx.x < g.q_blocks) queries<T, LPR, ROWS>(g);
    else keys_values<T, LPR, ITER>(g, red);
}

template <typename T, int LPR, int ITER>
hipError_t launch(const Args& g, bool many, unsigned blocks, hipStream_t st) {
    if (many) qk_norm_rope8_kernel<T, LPR, 4, ITER><<<blocks, 256, 0, st>>>(g);
    else qk_norm_rope8_kernel<T, LPR, 1, ITER><<<blocks, 256, 0, st>>>(g);
    return hipGetLastError();
}

template <typename T, int LPR>
hipError_t launch_block(const Args& g, bool many, unsigned blocks, hipStream_t st) {
    const int iter = ((1 << g.block_shift) * LPR + 255) / 256;
    if (iter <= 1) return launch<T, LPR, 1>(g, many, blocks, st);
    if (iter == 2) return launch<T, LPR, 2>(g, many, blocks, st);
    if constexpr (LPR >= 16)
        if (iter == 4) return launch<T, LPR, 4>(g, many, blocks, st);
    if constexpr (LPR == 32) return launch<T, LPR, 8>(g, many, blocks, st);
    return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_dim(const Args& g, bool many, unsigned blocks, hipStream_t st) {
    const int lpr = row_lanes(g.a.head_dim);
    return lpr == 8    ? launch_block<T, 8>(g, many, blocks, st)
           : lpr == 16 ? launch_block<T, 16>(g, many, blocks, st)
                       : launch_block<T, 32>(g, many, blocks, st);
}

}  // namespace

hipError_t launch_qk_norm_rope8(const jx_rope_args& a, const jx_kv_scales& s, hipStream_t st) {
    const Rope8Grid n = rope8_grid(a, s.block);
    const Args g = {a, s.d_k, s.d_v, log2_of(a.cache.page), log2_of(s.block), (unsigned)n.q_blocks, n.rows};
    const unsigned blocks = (unsigned)(n.q_blocks + n.kv_blocks);
    return a.dtype == JX_BF16 ? launch_dim<__bf16>(g, n.q_rows == 4, blocks, st) : launch_dim<_Float16>(g, n.q_rows == 4, blocks, st);
}

}  // namespace jx
