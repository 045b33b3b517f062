// Queries and keys of a step made ready for attention over a cache of 8 bits: RMS norm per head, rotation by position, keys and
// values put into their blocks as e4m3 beside one power of two for each block and key head.
#include <type_traits>
#include "attend_walk.h"
#include "codes8.h"
#include "rope_row.h"

namespace jx {

namespace {

// Queries are those of qk_norm_rope_kernel.  Keys (y as there) and values (y = x) of the rows that lie in one block, one head: with
// E = the largest exponent among the new |y|, the scale is 2^(E - 7), or what the block has if that is more and the block has tokens
// in front of the new ones; codes are y / scale, rounded once.  So the largest code is 128 up to 256: e4m3 has as many digits at any power of two, and
// what a block holds moves to a larger scale by its exponents alone, but for numbers under 2^-6 of the scale.
// Bound: bytes for many tokens, the chain slot - row - largest - store for few.  A team takes the rows of one block, one head, keys or
// values: LPR lanes a row as for the queries, rows held in registers from their one read to their store.  A team is as many lanes as
// the block has rows for, up to a wavefront (with four rows a lane), and a workgroup for larger blocks, whose largest value goes through LDS.
// With very many tokens the queries are a launch of their own, which has more wavefronts resident than these have registers for: 8,191
// tokens, 32 + 16 heads of 128 elements, blocks of 32: 29.4 us for the queries, 4.5 TB/s read and written, 17.6 for keys and values, where the vector
// instructions (590 a wavefront) and the chain share the time (20.3 where maxima and conversions of values take one element at a time); 56 to 63
// in one launch.  64 tokens 5.6 us, 1,111 with a scale each 9.
struct Args {
    jx_rope_args a;
    uint8_t *k_scale, *v_scale;
    int page_shift, block_shift;
    Rope8Grid n;
};

template <typename T>
constexpr float LARGEST = __is_same(T, _Float16) ? 0x1.ep15f : 0x1.ep127f;  // the largest code times the largest scale that the type holds

template <typename T, int LPR, int ROWS>
__device__ __forceinline__ void queries(const Args& g, uint32_t block) {
    typedef typename Vec<T>::x8 X8;
    const jx_rope_args& a = g.a;
    const int c = threadIdx.x % LPR, c8 = c * 8;
    const int groups = (a.n_heads + ROWS - 1) / ROWS;
    const uint32_t i = block * (256 / LPR) + threadIdx.x / LPR, t = i / groups;
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
    f32x8 x[ROWS];
    for (int r = 0; r < ROWS; r++) x[r] = __builtin_convertvector(raw[r], f32x8);
    norm_rows<T, LPR, ROWS>(a, x, (const T*)a.d_q_weight, inside, c8);
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        x[r] = turned(a, x[r], angles);
        if (inside && row0 + r < a.n_heads) store8((T*)a.d_q_out + ((int64_t)t * a.n_heads + row0 + r) * a.head_dim + c8, placed ? x[r] : (f32x8)0.0f);
    }
}

constexpr uint32_t INFINITE = 0x7F800000u;
template <typename T>
constexpr uint32_t MOST_BYTE = __is_same(T, _Float16) ? 127 + 15 - 7 : 127 + 127 - 7;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t largest_number(f32x8 x) {
    uint32_t m = 0;
    for (int j = 0; j < 8; j++) {
        const uint32_t y = __float_as_uint(x[j]) & 0x7FFFFFFFu;
        m = y < INFINITE ? max(m, y) : m;
    }
    return m;
}

// The largest |x| of eight elements that is a number, as the bits of a float32: those are in order.  Maxima pass over what is not a number; an
// infinity has the eight looked at again.
__device__ __forceinline__ uint32_t largest(f32x8 x) {
    float m = 0.0f;
    for (int j = 0; j < 8; j += 2) m = fmaxf(fmaxf(m, fabsf(x[j])), fabsf(x[j + 1]));
    uint32_t bits = __float_as_uint(m);
    if (ballot(bits >= INFINITE)) bits = largest_number(x);
    return bits;
}
// ... of elements of type T, two at a time
template <typename T>
__device__ __forceinline__ uint32_t largest(typename Vec<T>::x8 x) {
    const u32x4 w = __builtin_bit_cast(u32x4, x) & 0x7FFF7FFFu;
    auto pair = [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    };
    const uint32_t p = pair(pair(w[0], w[1]), pair(w[2], w[3])), m = max(p & 0xFFFFu, p >> 16);
    if (ballot(m >= (__is_same(T, __bf16) ? 0x7F80u : 0x7C00u))) return largest_number(__builtin_convertvector(x, f32x8));
    if constexpr (__is_same(T, __bf16)) return m << 16;
    else return __float_as_uint((float)__builtin_bit_cast(_Float16, (uint16_t)m));
}

// The largest over a team of 8 to 64 lanes
__device__ __forceinline__ uint32_t team_max(uint32_t v, int team) {
    v = max(v, dpp_u32<0xB1>(v));
    v = max(v, dpp_u32<0x4E>(v));
    v = max(v, dpp_u32<0x141>(v));
    if (team >= 16) v = max(v, dpp_u32<0x140>(v));
    if (team >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
    if (team >= 64) v = max(v, (uint32_t)__shfl_xor((int)v, 32, 64));
    return v;
}

// The scale's byte, from the largest of a block's new rows and what the block has
template <typename T>
__device__ __forceinline__ uint32_t scale_byte(uint32_t most, uint32_t old) {
    return max(min(max((int)(most >> 23) - 7, 1), (int)MOST_BYTE<T>), (int)old);
}

// held: whether values over LARGEST are possible, which would be rounded up to what the type does not have
template <typename T>
__device__ __forceinline__ uint2 encode(f32x8 x, float scale, bool held) {
    if (held)
        for (int j = 0; j < 8; j++) x[j] = fabsf(x[j]) < INFINITY ? fminf(fmaxf(x[j], -LARGEST<T>), LARGEST<T>) : x[j];
    return make_uint2(codes_of(x[0], x[1], x[2], x[3], scale), codes_of(x[4], x[5], x[6], x[7], scale));
}
// ... elements of type T, two at a time
template <typename T>
__device__ __forceinline__ uint2 encode(typename Vec<T>::x8 x, float scale, bool held) {
    if (held) return encode<T>(__builtin_convertvector(x, f32x8), scale, true);
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    auto two = [&](s16x2 w, T a, T b, auto high) {
        const typename Vec<T>::x2 y = {a, b};
        if constexpr (__is_same(T, __bf16)) return __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, y, scale, high());
        else return __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, y, scale, high());
    };
    auto four = [&](int j) {
        const s16x2 w = two(s16x2{0, 0}, x[j], x[j + 1], std::false_type());
        return __builtin_bit_cast(uint32_t, two(w, x[j + 2], x[j + 3], std::true_type()));
    };
    return make_uint2(four(0), four(4));
}

// ITER: rows of a block / rows that the team holds at a time
template <typename T, int LPR, int ITER, bool WIDE>
__device__ __forceinline__ void keys_values(const Args& g, uint32_t (&red)[2][4]) {
    typedef typename Vec<T>::x8 X8;
    const jx_rope_args& a = g.a;
    const int tid = threadIdx.x, lane = lane_id(), team = WIDE ? 256 : g.n.team, at_once = team / LPR;
    const int in_team = tid & (team - 1), c = in_team % LPR, c8 = c * 8, mine = in_team / LPR;
    const uint32_t i = (blockIdx.x * 256 + tid) / team, window = i / a.n_kv_heads;
    const int64_t t0 = (int64_t)window * g.n.rows;
    if (t0 >= a.n_tokens) return;  // whole teams
    const int head = (int)(i - window * a.n_kv_heads), block = 1 << g.block_shift;
    const bool inside = c8 < a.head_dim;
    // the slot of a row, -1 where it is not stored, and its position; no branch, so that reads of several rows are on their way together
    struct At {
        int64_t slot;
        int pos;
    };
    auto row_at = [&](int64_t t) {
        const int64_t i = min(max(t, (int64_t)0), a.n_tokens - 1), slot = a.d_slot[i];
        const int pos = a.d_pos[i];
        const bool stored = t == i && (uint32_t)pos < (uint32_t)a.n_pos && slot >= 0 && (slot >> g.page_shift) < a.cache.n_pages;
        return At{stored ? slot : -1, stored ? pos : 0};
    };
    auto block_of = [&](int64_t slot) { return slot >> g.block_shift; };  // of -1: -1

    // The run that begins with row t in slot `slot`; rows: the team's, from t on
    auto store = [&](int64_t t, int64_t slot, const At (&rows)[ITER]) {
        const int64_t b = block_of(slot), at = b * a.n_kv_heads + head;
        const int first = (int)(slot & (block - 1)), begin = (int)(slot & (a.cache.page - 1)) - first;  // of the block in its page
        const int64_t to = (slot >> g.page_shift) * a.cache.page_stride + begin * a.cache.token_stride + head * a.cache.head_stride;  // the block's first
        const uint32_t old_k = first ? g.k_scale[at] : 0, old_v = first ? g.v_scale[at] : 0;
        const T* from_k = (const T*)a.d_k + t * a.k_token_stride + head * a.k_head_stride;
        const T* from_v = (const T*)a.d_v + t * a.v_token_stride + head * a.v_head_stride;
        uint8_t *to_k = (uint8_t*)a.cache.d_k + to, *to_v = (uint8_t*)a.cache.d_v + to;
        X8 k[ITER], v[ITER];
        int places[ITER];  // in the block; -1: not a row of this run, or not a part of one
#pragma unroll
        for (int r = 0; r < ITER; r++) {
            const int row = r * at_once + mine;
            const bool there = row < block && block_of(rows[r].slot) == b;
            places[r] = there && inside ? (int)rows[r].slot & (block - 1) : -1;
            k[r] = v[r] = (X8)(T)0.0f;
            if (places[r] >= 0) {
                k[r] = *(const X8*)(from_k + row * a.k_token_stride + c8);
                v[r] = *(const X8*)(from_v + row * a.v_token_stride + c8);
            }
        }
        // the angles of two rows are asked for with them: those of more have no registers
        constexpr int EARLY = ITER <= 2 ? ITER : 0;
        Angles angles[EARLY ? EARLY : 1];
#pragma unroll
        for (int r = 0; r < EARLY; r++) angles[r] = angles_at(a, rows[r].pos, places[r] >= 0, c);
        f32x8 x[ITER];
        uint32_t most_k = 0, most_v = 0;
        for (int r = 0; r < ITER; r++) x[r] = __builtin_convertvector(k[r], f32x8);
        norm_rows<T, LPR, ITER>(a, x, (const T*)a.d_k_weight, inside, c8);
#pragma unroll
        for (int r = 0; r < ITER; r++) {
            if (!ballot(places[r] >= 0)) continue;
            x[r] = turned(a, x[r], EARLY ? angles[EARLY ? r : 0] : angles_at(a, rows[r].pos, places[r] >= 0, c));
            most_k = max(most_k, largest(x[r]));
            most_v = max(most_v, largest<T>(v[r]));
        }
        most_k = team_max(most_k, team);
        most_v = team_max(most_v, team);
        if (WIDE) {
            if (lane == 0) {
                red[0][tid >> 6] = most_k;
                red[1][tid >> 6] = most_v;
            }
            __syncthreads();
            most_k = max(max(red[0][0], red[0][1]), max(red[0][2], red[0][3]));
            most_v = max(max(red[1][0], red[1][1]), max(red[1][2], red[1][3]));
        }
        const uint32_t byte_k = scale_byte<T>(most_k, old_k), byte_v = scale_byte<T>(most_v, old_v);
        const bool held = ballot(max(byte_k, byte_v) >= MOST_BYTE<T>) != 0;
#pragma unroll
        for (int r = 0; r < ITER; r++)
            if (places[r] >= 0) {
                const int64_t row = places[r] * a.cache.token_stride + c8;
                *(uint2*)(to_k + row) = encode<T>(x[r], scale_bits(byte_k), held);
                *(uint2*)(to_v + row) = encode<T>(v[r], scale_bits(byte_v), held);
            }
        auto move = [&](uint8_t* cache, uint32_t from, uint32_t to) {
            if (first && from != to && inside)
                for (int row = mine; row < first; row += at_once) {
                    uint2* p = (uint2*)(cache + row * a.cache.token_stride + c8);
                    const uint2 w = *p;
                    *p = make_uint2(codes_moved(w.x, scale_bits(from), scale_bits(to)), codes_moved(w.y, scale_bits(from), scale_bits(to)));
                }
        };
        move(to_k, old_k, byte_k);
        move(to_v, old_v, byte_v);
        if (WIDE) __syncthreads();  // every wavefront has read the old scales and red
        if (in_team == 0) {
            g.k_scale[at] = (uint8_t)byte_k;
            g.v_scale[at] = (uint8_t)byte_v;
        }
    };
    At rows[ITER];
    if (g.n.rows == 1) {
        const int64_t slot = row_at(t0).slot, before = row_at(t0 - 1).slot;
#pragma unroll
        for (int r = 0; r < ITER; r++) rows[r] = row_at(t0 + r * at_once + mine);
        if (slot >= 0 && block_of(before) != block_of(slot)) store(t0, slot, rows);
        return;
    }
    // a team of 64 lanes or more: the runs that begin among `rows` rows, of up to 32 rows each
    const At at = row_at(t0 + lane);
    const int64_t before = row_at(t0 + lane - 1).slot;
    for (uint64_t begins = ballot(lane < g.n.rows && at.slot >= 0 && block_of(before) != block_of(at.slot)); begins; begins &= begins - 1) {
        const int j = __builtin_ctzll(begins);
#pragma unroll
        for (int r = 0; r < ITER; r++) {
            const int from = j + r * at_once + mine;
            rows[r] = block <= 32 ? At{shfl64(at.slot, from), __shfl(at.pos, from, 64)} : row_at(t0 + from);
        }
        store(t0 + j, (int64_t)readlane64((uint64_t)at.slot, j), rows);
    }
}

template <typename T, int LPR, int ITER, bool WIDE>
__global__ __launch_bounds__(256) void qk_norm_rope8_kernel(Args g) {
    __shared__ uint32_t red[2][4];
    if (blockIdx.x < g.n.kv_blocks) keys_values<T, LPR, ITER, WIDE>(g, red);
    else if (g.n.q_rows == 4) queries<T, LPR, 4>(g, blockIdx.x - (uint32_t)g.n.kv_blocks);
    else queries<T, LPR, 1>(g, blockIdx.x - (uint32_t)g.n.kv_blocks);
}

template <typename T, int LPR>
__global__ __launch_bounds__(256) void qk_norm_rope8_queries_kernel(Args g) {
    queries<T, LPR, 4>(g, blockIdx.x);
}

template <typename T, int LPR, int ITER, bool WIDE>
hipError_t launch(const Args& g, hipStream_t st) {
    if (g.n.apart) qk_norm_rope8_queries_kernel<T, LPR><<<(unsigned)g.n.q_blocks, 256, 0, st>>>(g);
    qk_norm_rope8_kernel<T, LPR, ITER, WIDE><<<(unsigned)(g.n.kv_blocks + (g.n.apart ? 0 : g.n.q_blocks)), 256, 0, st>>>(g);
    return hipGetLastError();
}

template <typename T, int LPR>
hipError_t launch_block(const Args& g, hipStream_t st) {
    const int lanes = LPR << g.block_shift;
    if (lanes <= 64) return launch<T, LPR, 1, false>(g, st);
    if (lanes == 128) return launch<T, LPR, 2, false>(g, st);
    if (lanes == 256) return launch<T, LPR, 4, false>(g, st);
    if (lanes == 512) return launch<T, LPR, 2, true>(g, st);
    if constexpr (LPR >= 16)
        if (lanes == 1024) return launch<T, LPR, 4, true>(g, st);
    if constexpr (LPR == 32) return launch<T, LPR, 8, true>(g, st);
    return hipErrorInvalidValue;
}

template <typename T>
hipError_t launch_dim(const Args& g, hipStream_t st) {
    const int lpr = row_lanes(g.a.head_dim);
    return lpr == 8 ? launch_block<T, 8>(g, st) : lpr == 16 ? launch_block<T, 16>(g, st) : launch_block<T, 32>(g, st);
}

}  // namespace

hipError_t launch_qk_norm_rope8(const jx_rope_args& a, const jx_kv_scales& s, hipStream_t st) {
    const Args g = {a, s.d_k, s.d_v, log2_of(a.cache.page), log2_of(s.block), rope8_grid(a, s.block)};
    return a.dtype == JX_BF16 ? launch_dim<__bf16>(g, st) : launch_dim<_Float16>(g, st);
}

}  // namespace jx
