// Attention of a step's new tokens over a paged cache.
#include "attend_walk.h"

namespace jx {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

constexpr int CLEARERS = 8;      // workgroups that look for rows of no request
constexpr int MAX_SLOTS = 1024;  // tiles that are shared out by keys; of more there are enough without

// A tile that several workgroups share: parts 2 work + 1 of the first of them, 2 work of the pieces - 1 that follow.  0 pieces: none
struct __attribute__((aligned(16))) Join {
    int pieces, head, first, count;  // of the tile: key head, first row and number of rows
    int start, unused[3];            // of the request: its first row of q
};

struct PagedArgs {
    jx_attend_args a;
    int page_shift, group;  // group: query heads of a key head
    uint32_t group_mul, group_shift;  // see by_group
    int near;               // whether the rows that one load of a wavefront takes lie in one page, less than 2^31 bytes apart
    int slots, n_work;      // tiles at most; workgroups that share them, 0 = a workgroup a tile
    float* part;            // [2 n_work][4]: of 32 rows, over a part of a tile's keys, sums [NB][4][64][4], largest scores and
                            // weights' sums [2][32]; the sums as a wavefront holds them, see part_at
    Join* joins;            // [n_work]
};

__device__ __attribute__((aligned(16))) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

// n / group for 0 <= n < 2^31, by a product with the reciprocal rounded up to 32 bits: group_mul = ceil(2^(31 + b) / group),
// 2^(b - 1) < group <= 2^b, is too large by less than 1 / 2^31 of itself.
__device__ __forceinline__ int by_group(const PagedArgs& g, int n) {
    return g.group == 1 ? n : (int)(__umulhi((uint32_t)n, g.group_mul) >> g.group_shift);
}

// ---- a tile: ROWS consecutive rows (token, head of the group) of one request -------------------------------------------
// Request r has rows (q_start[r + 1] - q_start[r]) * group for each key head.  Its tiles are the slots from
// q_start[r] * group / ROWS + r on: that leaves room for each request's last, partly filled one without a sum over the requests,
// at the price of slots that stay empty.
struct Tile {
    int r;               // request, -1: an empty slot
    int start;           // the request's first row of q
    int first, count;    // first row and number of rows
    int p0, p1;          // positions of the first and the last row's token
    int lo, hi;          // the keys that any of its rows sees: [lo, hi), lo rounded down to a multiple of 64
};

__device__ __forceinline__ int clamp_rows(int start, const jx_attend_args& a) { return min(max(start, 0), (int)a.n_tokens); }

template <int ROWS>
__device__ __forceinline__ int first_slot(int start, int r, const PagedArgs& g) {
    return (int)((long long)clamp_rows(start, g.a) * g.group / ROWS) + r;
}

template <int ROWS>
__device__ __forceinline__ Tile make_tile(const PagedArgs& g, int r, int slot, int start, int end, int len) {
    Tile t;
    const int b = clamp_rows(start, g.a), e = clamp_rows(end, g.a);
    t.start = b;
    t.first = (slot - first_slot<ROWS>(start, r, g)) * ROWS;
    t.count = min((e - b) * g.group - t.first, ROWS);
    t.r = t.count > 0 && t.first >= 0 ? r : -1;
    if (t.r < 0) t.count = t.first = 1;
    const int p = max(len, 0) - (e - b);  // n_tokens is below 2^29
    t.p0 = p + by_group(g, t.first);
    t.p1 = p + by_group(g, t.first + t.count - 1);
    const int hi = min(t.p1 + 1, g.a.table_pages << g.page_shift);
    const int lo = g.a.window && t.p0 >= g.a.window ? t.p0 + 1 - g.a.window : 0;
    t.lo = hi > lo ? lo & ~63 : 0;
    t.hi = hi > lo ? hi : 0;
    return t;
}

// The last of 0 .. n - 1 for which before() holds (it holds for all up to that one; 0 if for none), by all lanes of a wavefront
template <typename Before>
__device__ __forceinline__ int last_before(int n, Before before) {
    int lo = 0;
    while (n > 1) {
        const int step = (n + 63) >> 6, at = lane_id() * step;
        const int k = max(__popcll(ballot(at < n && before(lo + min(at, n - 1)))) - 1, 0);
        lo += k * step;
        n = min(step, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// ---- rows of keys and values in LDS ------------------------------------------------------------------------------------
// A row is CH chunks of 16 bytes; chunk c of row r lies at place c ^ mix(r).  The matrix instructions' operands are read as the
// same chunk of 32 consecutive keys (K) and as four consecutive rows of 16 or 32 elements (V, transposed on the way); mix
// spreads both over the banks: any 8 and any 16 consecutive rows (8 chunks: half as many places) get different places, and so
// do rows r .. r + 3 beside pairs and quadruples of neighbouring chunks.
template <int CH>
__device__ __forceinline__ constexpr int mix(int r) {
    return CH == 8 ? (r & 1) * 2 ^ (r >> 1 & 1) * 4 ^ (r >> 2 & 1) ^ (r >> 3 & 1) * 2
                   : (r & 1) * 6 ^ (r >> 1 & 1) * 12 ^ (r >> 2 & 1) ^ (r >> 3 & 1) * 2;
}

typedef __attribute__((address_space(3))) char* lds_ptr;

__device__ __forceinline__ void load_lds16(const void* from, lds_ptr to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Element e of row r (of 32) among the sums that a wavefront leaves for join_kernel; elements 4 i .. 4 i + 3 are together
__device__ __forceinline__ int part_at(int r, int e) { return ((e >> 3) * 64 + r + (e >> 2 & 1) * 32) * 4 + (e & 3); }
constexpr int part_floats(int nb) { return nb * 1024 + 64; }

template <typename T>
struct Mfma;
template <>
struct Mfma<__bf16> {
    static __device__ __forceinline__ f32x16 mul(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Vec<__bf16>::x8, a), __builtin_bit_cast(Vec<__bf16>::x8, b), c, 0, 0, 0);
    }
};
template <>
struct Mfma<_Float16> {
    static __device__ __forceinline__ f32x16 mul(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Vec<_Float16>::x8, a), __builtin_bit_cast(Vec<_Float16>::x8, b), c, 0, 0, 0);
    }
};

__device__ __forceinline__ float both_halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float both_halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// ---- many rows: four wavefronts of 32 rows each over the same keys ------------------------------------------------------
// S^T = K Q^T, 64 keys by 32 rows at a time, so that a lane holds 32 scores of one row (the other lane with that row, 32 further on,
// the rest); then O^T += V^T P^T, where the scores' registers are already the second operand of the matrix instruction if the keys
// of the first are taken in the same order.  The running maximum moves only when a row's scores rise by more than 2^8 over it:
// weights of up to 2^8 round no worse, and most tiles leave the sums alone.
template <typename T, int NB>
struct Rows32 {
    static constexpr int CH = NB <= 2 ? 8 : NB <= 4 ? 16 : 32, PITCH = CH * 16;
    s16x8 q[2 * NB];
    f32x16 o[NB];        // sums
    float m, l, top;     // running maximum and sum of weights, the scores' largest
    int k_at, v_at;  // a lane's first place in a row of keys, of values

    __device__ __forceinline__ void begin() {
        const int lane = lane_id(), row = lane & 31, h = lane >> 5, i = lane & 15;
        k_at = row * PITCH + (h ^ mix<CH>(row)) * 16;
        const int vr = 4 * h + (i >> 2), vc = (lane >> 4 & 1) * 2 + (i >> 1 & 1);
        v_at = vr * PITCH + (vc ^ mix<CH>(vr)) * 16 + (i & 1) * 8;
        m = -INFINITY;
        l = 0.0f;
        for (int b = 0; b < NB; b++) o[b] = (f32x16)0.0f;
    }

    __device__ __forceinline__ s16x8 keys_at(lds_ptr k, int i) const {  // operand i of 4 NB: 32 keys by 16 elements
        return *(const __attribute__((address_space(3))) s16x8*)(k + (k_at ^ (i / 2 * 32)) + i % 2 * 32 * PITCH);
    }
    __device__ __forceinline__ s16x8 values_at(lds_ptr v, int i) const {  // operand i of 4 NB: 32 elements by 16 keys
        const int x = i / NB, b = i % NB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + (v_at ^ (b * 64)) + x * 16 * PITCH));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + (v_at ^ (b * 64) ^ 32) + (x * 16 + 8) * PITCH));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }

    // The first tile's scores
    __device__ __forceinline__ void scores(lds_ptr k, f32x16 (&s)[2]) {
        for (int kb = 0; kb < 2; kb++) s[kb] = (f32x16)0.0f;
        for (int i = 0; i < 4 * NB; i++) s[i & 1] = Mfma<T>::mul(keys_at(k, i), q[i / 2], s[i & 1]);
        largest(s);
    }

    __device__ __forceinline__ void largest(const f32x16 (&s)[2]) {
        top = -INFINITY;
        for (int i = 0; i < 32; i += 2) top = fmaxf(fmaxf(top, s[i >> 4][i & 15]), s[i >> 4][(i & 15) + 1]);
    }

    // Moves the running maximum if these scores rise far over it; c = scale * log2 e
    __device__ __forceinline__ void raise(float c) {
        const float t = both_halves_max(top) * c;
        if (ballot(t > m + 8.0f)) {
            const float to = fmaxf(t, m), keep = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.0f : to));
            m = to;
            l *= keep;
            for (int b = 0; b < NB; b++)
                for (int i = 0; i < 16; i++) o[b][i] *= keep;
        }
    }

    // One tile's scores to weights while the next one's scores are formed, then the weighted values, while the next scores' largest
    // is looked for: matrix and vector instructions alternate, reads of LDS run AHEAD matrix instructions before their use.
    // What stands between two fences is not moved over them.
    __device__ __forceinline__ void advance(const f32x16 (&s)[2], f32x16 (&next)[2], lds_ptr k, lds_ptr v, float c) {
        constexpr int N = 4 * NB, AHEAD = 3, EACH = 32 / N;  // matrix instructions of each half; scores for each of them
        const float base = m == -INFINITY ? 0.0f : m;
        next[0] = next[1] = (f32x16)0.0f;
        s16x8 kf[AHEAD], vf[AHEAD], p[4];
        float w[8], sum = 0.0f;
        for (int i = 0; i < AHEAD; i++) kf[i] = keys_at(k, i);
#pragma unroll
        for (int i = 0; i < N; i++) {
            next[i & 1] = Mfma<T>::mul(kf[i % AHEAD], q[i / 2], next[i & 1]);
            if (i + AHEAD < N) kf[i % AHEAD] = keys_at(k, i + AHEAD);
            else vf[i + AHEAD - N] = values_at(v, i + AHEAD - N);
#pragma unroll
            for (int e = i * EACH; e < (i + 1) * EACH; e++) {
                w[e & 7] = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], c, -base));
                sum += w[e & 7];
                if ((e & 7) == 7) {
                    f32x8 y;
                    for (int j = 0; j < 8; j++) y[j] = w[j];
                    p[e >> 3] = __builtin_bit_cast(s16x8, __builtin_convertvector(y, typename Vec<T>::x8));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        l += sum;
        top = -INFINITY;
#pragma unroll
        for (int i = 0; i < N; i++) {
            o[i % NB] = Mfma<T>::mul(vf[i % AHEAD], p[i / NB], o[i % NB]);
            if (i + AHEAD < N) vf[i % AHEAD] = values_at(v, i + AHEAD);
#pragma unroll
            for (int e = i * EACH; e < (i + 1) * EACH; e++)
                if (e & 1) top = fmaxf(fmaxf(top, next[e >> 4][(e & 15) - 1]), next[e >> 4][e & 15]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// Whether any element of a tile is infinite or not a number
template <typename T>
__device__ __forceinline__ bool odd_values_in(lds_ptr v, int bytes) {
    uint32_t worst = 0;
    for (int at = lane_id() * 16; at < bytes; at += 64 * 16) {
        const s16x8 y = *(const __attribute__((address_space(3))) s16x8*)(v + at);
        for (int j = 0; j < 8; j++) worst = max(worst, (uint32_t)(y[j] & 0x7FFF));
    }
    return ballot(worst >= (__is_same(T, __bf16) ? 0x7F80u : 0x7C00u)) != 0;
}

// A lane's row: whether there is one, its query head, its token's row of q, its position
struct RowAt {
    bool mine;
    int head, token, pos;
};

// Rows that belong to no request: zeros and -infinity, by workgroups `block` of `blocks`
template <typename T>
__device__ void clear_rows(const jx_attend_args& a, int block, int blocks) {
    const int n = (int)a.n_tokens, b = a.n_req ? clamp_rows(a.d_q_start[0], a) : n, e = a.n_req ? clamp_rows(a.d_q_start[a.n_req], a) : n;
    const int chunks = a.n_heads * (a.head_dim / 8), outside = b + max(n - max(b, e), 0);
    for (int i = block; i < outside; i += blocks) {
        const long long t = i < b ? i : i - b + max(b, e);
        for (int c = threadIdx.x; c < chunks; c += 256) ((uint4*)a.d_out)[t * chunks + c] = make_uint4(0, 0, 0, 0);
        if (a.d_lse)
            for (int h = threadIdx.x; h < a.n_heads; h += 256) a.d_lse[t * a.n_heads + h] = -INFINITY;
    }
}

template <typename T, int NB>
__global__ __launch_bounds__(256, NB <= 4 ? 2 : 1) void paged_tile_kernel(PagedArgs g) {
    typedef Rows32<T, NB> R;
    constexpr int ROWS = 128, KEYS = 64, TILE = KEYS * R::PITCH;
    constexpr int LOADS = KEYS * R::CH / 256;
    extern __shared__ __attribute__((aligned(1024))) char lds[];  // [2] keys, [2] values; slots' sums of units, their requests
    const jx_attend_args& a = g.a;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int sharers = (int)gridDim.x - CLEARERS;
    if ((int)blockIdx.x >= sharers) {
        clear_rows<T>(a, (int)blockIdx.x - sharers, CLEARERS);
        return;
    }
    const lds_ptr ring = (lds_ptr)lds;
    int* starts = (int*)(lds + 4 * TILE);               // [n_req + 1]
    int* lens = starts + a.n_req + 1;                   // [n_req + 1]
    int* cum = lens + a.n_req + 1;                      // [slots + 1]
    uint16_t* req = (uint16_t*)(cum + g.slots + 1);     // [slots]

    // This workgroup's share: units (64 keys of a tile) x0 .. x1 - 1 of all tiles of all key heads.  The first `rem` shares are
    // `each` + 1 units, the others `each`; the launch has seen to it that all units are less than 2^31.
    uint32_t x0 = 0, x1 = 1, per_head = 1, each = 1, rem = 0;
    int head = 0, slot = 0, work = 0;
    if (g.n_work) {
        for (int i = tid; i <= a.n_req; i += 256) {
            starts[i] = a.d_q_start[i];
            lens[i] = i < a.n_req ? a.d_kv_len[i] : 0;
        }
        __syncthreads();
        for (int s = tid; s < g.slots; s += 256) {
            int lo = 0, hi = a.n_req;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_slot<ROWS>(starts[mid], mid, g) <= s) lo = mid;
                else hi = mid;
            }
            const Tile t = make_tile<ROWS>(g, lo, s, starts[lo], starts[lo + 1], lens[lo]);
            cum[s + 1] = t.r < 0 ? 0 : max((t.hi - t.lo + KEYS - 1) / KEYS, 1);
            req[s] = (uint16_t)lo;
        }
        if (tid == 0) cum[0] = 0;
        __syncthreads();
        if (wave == 0) {
            int carry = 0;
            for (int s0 = 0; s0 < g.slots; s0 += 64) {
                int v = s0 + lane < g.slots ? cum[s0 + lane + 1] : 0;
                for (int d = 1; d < 64; d *= 2) {
                    const int o = __shfl_up(v, d, 64);
                    if (lane >= d) v += o;
                }
                if (s0 + lane < g.slots) cum[s0 + lane + 1] = carry + v;
                carry += __shfl(v, 63, 64);
            }
        }
        __syncthreads();
        per_head = __builtin_amdgcn_readfirstlane(cum[g.slots]);
        const uint32_t all = per_head * a.n_kv_heads, shares = min((uint32_t)g.n_work, all);  // none is empty
        // consecutive shares stay on one XCD's cache; few are spread over all
        work = all < (uint32_t)g.n_work ? (int)blockIdx.x : (int)(blockIdx.x % 8) * (g.n_work / 8) + (int)(blockIdx.x / 8);
        if (tid == 0) g.joins[work].pieces = 0;
        if ((uint32_t)work >= shares) return;
        each = all / shares;
        rem = all - each * shares;
        x0 = work * each + min((uint32_t)work, rem);
        x1 = x0 + each + ((uint32_t)work < rem);
        head = (int)(x0 / per_head);
    } else {
        head = (int)(blockIdx.x % a.n_kv_heads);
        slot = g.slots - 1 - (int)(blockIdx.x / a.n_kv_heads);
    }

    const int d = a.head_dim, page_mask = a.cache.page - 1;
    const uint32_t page_chunks = (uint32_t)(a.cache.page_stride / 8), token_chunks = (uint32_t)(a.cache.token_stride / 8);
    const float c = fmaxf(fabsf(a.scale) * LOG2E, 1e-30f);  // a scale of 0 has to leave -infinity what it is
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
    while (x0 < x1) {
        int u0 = 0, units = 1, u1 = 1;
        Tile t;
        if (g.n_work) {
            if (x0 >= (head + 1) * per_head) head++;
            const int at = (int)(x0 - head * per_head);
            slot = last_before(g.slots, [&](int i) { return cum[i] <= at; });
            u0 = at - cum[slot];
            units = cum[slot + 1] - cum[slot];
            u1 = (int)min((uint32_t)units, u0 + (x1 - x0));
            const int r = req[slot];
            t = make_tile<ROWS>(g, r, slot, starts[r], starts[r + 1], lens[r]);
        } else {
            const int r = last_before(a.n_req, [&](int i) { return first_slot<ROWS>(a.d_q_start[i], i, g) <= slot; });
            t = make_tile<ROWS>(g, r, slot, a.d_q_start[r], a.d_q_start[r + 1], a.d_kv_len[r]);
            if (t.r < 0) return;
            u1 = units = max((t.hi - t.lo + KEYS - 1) / KEYS, 1);
        }
        const bool whole = u0 == 0 && u1 == units;
        const int key0 = t.lo + u0 * KEYS, key1 = min(t.lo + u1 * KEYS, t.hi);

        // rows of this wavefront
        R x;
        x.begin();
        const int rows0 = ((wave + work) & 3) * 32;  // tiles of few rows: the workgroups of a CU keep different SIMDs busy
        const bool busy = rows0 < t.count;
        auto row_of = [&](int of_lane) {
            const int row = rows0 + (of_lane & 31), rr = t.first + min(row, t.count - 1), token = by_group(g, rr);
            return RowAt{row < t.count, head * g.group + (rr - token * g.group), t.start + token, t.p0 + token - by_group(g, t.first)};
        };
        const RowAt at_row = row_of(lane);
        const int pos = at_row.pos;
        if (busy) {
            const T* q = (const T*)a.d_q + at_row.token * a.q_token_stride + at_row.head * a.q_head_stride + (lane >> 5) * 8;
            for (int i = 0; i < 2 * NB; i++) {
                uint4 w = i * 16 + (lane >> 5) * 8 < d && at_row.mine ? *(const uint4*)(q + i * 16) : make_uint4(0, 0, 0, 0);
                w = make_uint4(w.x ^ flip, w.y ^ flip, w.z ^ flip, w.w ^ flip);
                x.q[i] = __builtin_bit_cast(s16x8, w);
            }
        }
        const int rows_end = min(t.count, rows0 + 32) - 1;
        const int w0 = t.p0 + by_group(g, t.first + rows0) - by_group(g, t.first);            // positions of the wavefront's
        const int w1 = t.p0 + by_group(g, t.first + max(rows_end, 0)) - by_group(g, t.first);    // first and last row

        const char* kb = (const char*)a.cache.d_k + head * a.cache.head_stride * 2;
        const char* vb = (const char*)a.cache.d_v + head * a.cache.head_stride * 2;
        const int32_t* table = a.d_table + (size_t)t.r * a.table_pages;
        auto page_of = [&](int key) {  // the page of key `key`, -1 where there is none to see
            int id = key < key1 ? table[key >> g.page_shift] : -1;
            return (uint32_t)id < (uint32_t)a.cache.n_pages ? id : -1;
        };
        // Where key `key` lies, in chunks from the head's first; the page has been looked up
        auto row_at = [&](int id, int key) {
            return (uint64_t)(uint32_t)id * page_chunks + (uint64_t)(uint32_t)(key & page_mask) * token_chunks;
        };
        bool odd_values = false;  // values that are not finite where not every row looks: see below
        // 64 rows of keys or values, from key `key` on, on their way into LDS; lane i has the page of the i-th.  The rows of one load of a
        // wavefront are neighbours in a page, if that has as many: their place is then a matter of scalar instructions.
        const uint32_t lane_off = (lane / R::CH * token_chunks + (lane % R::CH ^ mix<R::CH>(tid / R::CH))) * 16;
        auto stage = [&](const char* from, int key, int ids, lds_ptr to) {
            if (g.near && d == NB * 32 && !ballot(ids < 0)) {
                for (int i = 0; i < LOADS; i++) {
                    const int at = i * (256 / R::CH) + wave * (64 / R::CH);
                    const uint64_t row = row_at(__builtin_amdgcn_readlane(ids, at), key + at);
                    load_lds16(from + row * 16 + (lane_off ^ (i & 1) * mix<R::CH>(256 / R::CH) * 16), to + (i * 256 + wave * 64) * 16);
                }
                return;
            }
            const uint64_t rows = row_at(max(ids, 0), key + lane);
#pragma unroll 1
            for (int i = 0; i < LOADS; i++) {
                const int at = i * (256 / R::CH) + tid / R::CH, chunk = tid % R::CH ^ mix<R::CH>(at);
                const char* p = from + ((uint64_t)shfl64((long long)rows, at) + chunk) * 16;
                load_lds16(__shfl(ids, at, 64) >= 0 && chunk * 8 < d ? p : (const char*)zero_chunk, to + (i * 256 + wave * 64) * 16);
            }
        };
        // One tile's weights and values, the next one's scores; the keys after that and the next values on their way into the places that
        // the last step has read.  The compiler has to know that those are apart: it would wait for what is on its way before it reads.
        auto step = [&](int key, uint64_t there, int ids_v, int ids_k, f32x16 (&s)[2], f32x16 (&next)[2], const lds_ptr __restrict k,
                        const lds_ptr __restrict v, const lds_ptr __restrict next_k, const lds_ptr __restrict next_v) __attribute__((always_inline)) {
            if (key + 2 * KEYS < key1) stage(kb, key + 2 * KEYS, ids_k, next_k);
            if (key + KEYS < key1) stage(vb, key + KEYS, ids_v, next_v);
            if (!busy) return;
            const bool all = there == ~0ull && key + KEYS - 1 <= w0 && (!a.window || key > w1 - a.window);
            if (!all) {
                const int after = pos - key;  // the last key that the row sees, from here
                uint64_t seen = after < 0 ? 0 : after >= 63 ? ~0ull : (2ull << after) - 1;
                if (a.window) {
                    const int gone = after - a.window + 1;  // keys that have left the window
                    seen &= gone <= 0 ? ~0ull : gone > 63 ? 0 : ~0ull << gone;
                }
                seen &= there;
                seen >>= (lane >> 5) * 4;
                for (int b = 0; b < 2; b++)
                    for (int i = 0; i < 16; i++)
                        if (!((uint32_t)(seen >> (b * 32)) >> ((i & 3) + 8 * (i >> 2)) & 1)) s[b][i] = -INFINITY;
                x.largest(s);
                odd_values |= odd_values_in<T>(v, TILE);
            }
            x.raise(c);
            x.advance(s, next, k, v, c);  // the scores after the last tile are of no use: what lies there is read all the same
        };
        // Keys of tile i lie in half i & 1 of the ring's first part, values in the same half of its second
        f32x16 s0[2], s1[2];
        __syncthreads();  // the ring is free
        int ids = page_of(key0 + lane), ids_1 = page_of(key0 + KEYS + lane);
        if (key0 < key1) {
            stage(kb, key0, ids, ring);
            stage(vb, key0, ids, ring + 2 * TILE);
            if (key0 + KEYS < key1) stage(kb, key0 + KEYS, ids_1, ring + TILE);
            __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
            __syncthreads();
            if (busy) x.scores(ring, s0);
        }
        for (int key = key0; key < key1; key += 2 * KEYS) {
#pragma unroll
            for (int odd = 0; odd < 2; odd++) {
                const int at = key + odd * KEYS;
                if (at >= key1) break;
                const uint64_t there = ballot(ids >= 0);
                const int ids_2 = page_of(at + 2 * KEYS + lane);
                __builtin_amdgcn_s_waitcnt(0x0F70);  // this tile's values and the next one's keys have arrived
                __syncthreads();
                if (odd) step(at, there, ids_1, ids_2, s1, s0, ring, ring + 3 * TILE, ring + TILE, ring + 2 * TILE);
                else step(at, there, ids_1, ids_2, s0, s1, ring + TILE, ring + 2 * TILE, ring, ring + 3 * TILE);
                ids = ids_1;
                ids_1 = ids_2;
            }
        }

        // results; the rows' places are worked out again rather than held over the loop
        int again = lane;
        asm("" : "+v"(again));
        const RowAt y = row_of(again);
        const float l = both_halves_sum(x.l);
        float* part = NULL;
        if (!whole) {
            part = g.part + ((size_t)(2 * work + (u0 == 0)) * 4 + rows0 / 32) * part_floats(NB);
            if (u0 == 0 && tid == 0) {  // the first of the workgroups that share this tile names it
                const uint32_t end = x0 + units - 1, large = rem * (each + 1);  // the tile's last unit, and whose it is
                const int last = (int)(end < large ? end / (each + 1) : rem + (end - large) / each);
                g.joins[work] = {last - work + 1, head, t.first, t.count, t.start, {0, 0, 0}};
            }
        }
        const long long oi = (long long)y.token * a.n_heads + y.head;
        if (busy && !odd_values) {
            if (y.mine && whole) {
                const float inv = l == 0.0f ? 0.0f : 1.0f / l;
                T* out = (T*)a.d_out + oi * d + (lane >> 5) * 4;
                for (int b = 0; b < NB; b++)
                    for (int i = 0; i < 4; i++)
                        if (b * 32 + i * 8 + (lane >> 5) * 4 < d) {
                            f32x4 w;
                            for (int j = 0; j < 4; j++) w[j] = x.o[b][i * 4 + j] * inv;
                            *(typename Vec<T>::x4*)(out + b * 32 + i * 8) = __builtin_convertvector(w, typename Vec<T>::x4);
                        }
                if (lane < 32 && a.d_lse) a.d_lse[oi] = l == 0.0f ? -INFINITY : (x.m + __builtin_amdgcn_logf(l)) * LN2;
            } else if (y.mine) {
                for (int b = 0; b < NB; b++)
                    for (int i = 0; i < 4; i++) {
                        f32x4 w;
                        for (int j = 0; j < 4; j++) w[j] = x.o[b][i * 4 + j];
                        *(f32x4*)(part + ((b * 4 + i) * 64 + lane) * 4) = w;
                    }
                part[NB * 1024 + lane] = lane < 32 ? x.m : l;
            }
        } else if (busy) {
            // A weight of 0 times such a value is not 0: these 32 rows are done again, key by key
            constexpr int LPR = R::CH;
            const int c8 = lane % LPR * 8;
            for (int i = rows0; i < min(t.count, rows0 + 32); i++) {
                const int ri = t.first + i, tok = by_group(g, ri), hq = head * g.group + ri - tok * g.group;
                const long long tt = t.start + tok;
                const int p = t.p0 + tok - by_group(g, t.first);
                f32x8 q = {0, 0, 0, 0, 0, 0, 0, 0};
                if (c8 < d) q = load8((const T*)a.d_q + tt * a.q_token_stride + hq * a.q_head_stride + c8);
                for (int e = 0; e < 8; e++) q[e] *= a.scale * LOG2E;
                const int k0 = a.window ? max(key0, p + 1 - a.window) : key0, k1 = min(key1, p + 1);
                Softmax s = walk_keys<T, LPR>((const T*)kb, (const T*)vb, q, c8 < d, k0, k1, [&](long long key) {
                    const int id = page_of((int)key);
                    return id < 0 ? -1ll : (long long)row_at(id, (int)key) * 8;
                });
                s = gather<LPR>(s);
                const long long o = tt * a.n_heads + hq;
                if (whole) {
                    const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;
                    for (int e = 0; e < 8; e++) s.acc[e] *= inv;
                    if (lane < LPR && c8 < d) store8((T*)a.d_out + o * d + c8, s.acc);
                    if (lane == 0 && a.d_lse) a.d_lse[o] = s.l == 0.0f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * LN2;
                } else {
                    if (lane < LPR && c8 < d)
                        for (int e = 0; e < 8; e++) part[part_at(i & 31, c8 + e)] = s.acc[e];
                    if (lane == 0) {
                        part[NB * 1024 + (i & 31)] = s.m;
                        part[NB * 1024 + 32 + (i & 31)] = s.l;
                    }
                }
            }
        }
        x0 += u1 - u0;
    }
}

// The parts of a tile that several workgroups shared, as one: the tile that workgroup blockIdx.x began and did not end.
// blockIdx.y: which 32 elements.  A wavefront takes 32 rows, as their lanes held them when the parts were written; of a tile of few
// rows the wavefronts share out the pieces.  Bound: the time that a chain of reads takes, hence PIECES at once.
template <typename T, int NB>
__global__ __launch_bounds__(256) void join_kernel(PagedArgs g) {
    constexpr int PIECES = 4;
    __shared__ float others[4][18][64];
    const jx_attend_args& a = g.a;
    const Join j = g.joins[blockIdx.x];
    if (!j.pieces) return;
    const int work = (int)blockIdx.x, d = a.head_dim, lane = lane_id(), wave = (int)(threadIdx.x >> 6), b = (int)blockIdx.y;
    const int groups = j.count <= 32 ? 1 : j.count <= 64 ? 2 : 4;  // of rows
    const int row = wave % groups * 32 + (lane & 31);
    float m = -INFINITY, l = 0.0f;
    f32x4 s[4];
    for (int i = 0; i < 4; i++) s[i] = (f32x4)0.0f;
    if (row < j.count) {
        const float* parts = g.part + (wave % groups) * part_floats(NB) + lane * 4 + b * 1024;
        const int to_m = NB * 1024 - b * 1024 - lane * 4 + (lane & 31);
        for (int i0 = wave / groups; i0 < j.pieces; i0 += PIECES * (4 / groups)) {
            float pm[PIECES], pl[PIECES], top = m;
            f32x4 y[PIECES][4];
            for (int u = 0; u < PIECES; u++) {
                const int i = min(i0 + u * (4 / groups), j.pieces - 1);
                const float* p = parts + (size_t)(2 * (work + i) + (i == 0)) * 4 * part_floats(NB);
                pm[u] = p[to_m];
                pl[u] = p[to_m + 32];
                for (int k = 0; k < 4; k++) y[u][k] = *(const f32x4*)(p + k * 256);
            }
            for (int u = 0; u < PIECES; u++) {
                if (i0 + u * (4 / groups) >= j.pieces) pm[u] = -INFINITY;
                top = fmaxf(top, pm[u]);
            }
            const float base = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m - base);
            m = top;
            l *= keep;
            for (int k = 0; k < 4; k++)
                for (int e = 0; e < 4; e++) s[k][e] *= keep;
            for (int u = 0; u < PIECES; u++) {
                if (pm[u] == -INFINITY) continue;  // nothing, or not a piece
                const float w = __builtin_amdgcn_exp2f(pm[u] - base);
                l = fmaf(pl[u], w, l);
                for (int k = 0; k < 4; k++)
                    for (int e = 0; e < 4; e++) s[k][e] = fmaf(y[u][k][e], w, s[k][e]);
            }
        }
    }
    if (groups < 4) {
        others[wave][16][lane] = m;
        others[wave][17][lane] = l;
        for (int i = 0; i < 16; i++) others[wave][i][lane] = s[i >> 2][i & 3];
        __syncthreads();
        if (wave >= groups) return;
        float top = m;
        for (int w = wave + groups; w < 4; w += groups) top = fmaxf(top, others[w][16][lane]);
        const float base = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= keep;
        for (int i = 0; i < 16; i++) s[i >> 2][i & 3] *= keep;
        for (int w = wave + groups; w < 4; w += groups) {
            const float f = __builtin_amdgcn_exp2f(others[w][16][lane] - base);
            l = fmaf(others[w][17][lane], f, l);
            for (int i = 0; i < 16; i++) s[i >> 2][i & 3] = fmaf(others[w][i][lane], f, s[i >> 2][i & 3]);
        }
    }
    if (row >= j.count) return;
    const int rr = j.first + row, token = by_group(g, rr);
    const long long o = (j.start + (long long)token) * a.n_heads + j.head * g.group + rr - token * g.group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    for (int k = 0; k < 4; k++) {
        const int e = b * 32 + k * 8 + (lane >> 5) * 4;
        for (int i = 0; i < 4; i++) s[k][i] *= inv;
        if (e < d) *(typename Vec<T>::x4*)((T*)a.d_out + o * d + e) = __builtin_convertvector(s[k], typename Vec<T>::x4);
    }
    if (b == 0 && lane < 32 && a.d_lse) a.d_lse[o] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

struct Plan {
    int slots, n_work;
    int64_t part, joins, total;
};

int blocks_of(int head_dim) { return head_dim <= 64 ? 2 : head_dim <= 128 ? 4 : 8; }

Plan make_plan(const jx_attend_args& a) {
    constexpr int ROWS = 128;
    const int nb = blocks_of(a.head_dim);
    Plan p = {};
    const long long rows = a.n_tokens * (a.n_heads / a.n_kv_heads);
    p.slots = a.n_req ? (int)(rows / ROWS + a.n_req) : 0;
    const double units = ((double)a.table_pages * a.cache.page / 64 + 1) * p.slots * a.n_kv_heads;  // at most
    if (p.slots && p.slots <= MAX_SLOTS && units < 2e9) p.n_work = a.head_dim <= 128 ? 512 : 256;
    auto up = [](int64_t x) { return (x + 255) & ~(int64_t)255; };
    p.part = 0;
    p.joins = up((int64_t)2 * p.n_work * 4 * part_floats(nb) * 4);
    p.total = p.joins + up((int64_t)p.n_work * sizeof(Join));
    return p;
}

template <typename T, int NB>
hipError_t launch_tiles(const PagedArgs& g, hipStream_t st) {
    constexpr int TILE = 64 * Rows32<T, NB>::PITCH;
    const size_t lds = 4 * TILE + (g.n_work ? (size_t)(g.a.n_req + 1) * 8 + (size_t)(g.slots + 1) * 4 + (size_t)g.slots * 2 : 0);
    hipError_t e = hipFuncSetAttribute((const void*)paged_tile_kernel<T, NB>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess) return e;
    const unsigned blocks = (g.n_work ? g.n_work : (unsigned)(g.slots * g.a.n_kv_heads)) + CLEARERS;
    paged_tile_kernel<T, NB><<<blocks, 256, lds, st>>>(g);
    e = hipGetLastError();
    if (e != hipSuccess || !g.n_work) return e;
    join_kernel<T, NB><<<dim3(g.n_work, (g.a.head_dim + 31) / 32), 256, 0, st>>>(g);
    return hipGetLastError();
}

template <typename T>
hipError_t launch(const jx_attend_args& a, uint8_t* work, hipStream_t st) {
    const Plan p = make_plan(a);
    const int rows = 64 / (blocks_of(a.head_dim) * 4);
    const int near = a.cache.page >= rows && a.cache.token_stride * rows < (1 << 29);
    const int group = a.n_heads / a.n_kv_heads, bits = group == 1 ? 1 : log2_of(group - 1) + 1;
    const uint32_t mul = (uint32_t)(((1ull << (31 + bits)) + group - 1) / group);
    PagedArgs g = {a, log2_of(a.cache.page), group, mul, (uint32_t)bits - 1, near, p.slots, p.n_work, (float*)(work + p.part), (Join*)(work + p.joins)};
    const int nb = blocks_of(a.head_dim);
    return nb == 2 ? launch_tiles<T, 2>(g, st) : nb == 4 ? launch_tiles<T, 4>(g, st) : launch_tiles<T, 8>(g, st);
}

}  // namespace

int64_t paged_attention_bytes(const jx_attend_args& a) { return make_plan(a).total; }

hipError_t launch_paged_attention(const jx_attend_args& a, uint8_t* work, hipStream_t st) {
    return a.dtype == JX_BF16 ? launch<__bf16>(a, work, st) : launch<_Float16>(a, work, st);
}

}  // namespace jx
