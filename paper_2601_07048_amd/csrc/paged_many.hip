// Paged attention of chunks: tiles of 128 or 256 rows.
#include "paged_tiles.h"

namespace jx {

namespace {

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

// ---- many rows: four or eight wavefronts of 32 rows each over the same keys ---------------------------------------------
// S^T = K Q^T, 64 keys by 32 rows at a time, so that a lane holds 32 scores of one row (the other lane with that row, 32 further on,
// the rest); then O^T += V^T P^T, where the scores' registers are already the second operand of the matrix instruction if the keys
// of the first are taken in the same order.  The running maximum moves only when a row's scores rise by more than 2^8 over it:
// weights of up to 2^8 round no worse, and most tiles leave the sums alone.
// Bound: the matrix instructions, and with them the card's power: a chunk of 4,096 tokens over 16,384 keys, 32 heads of 128 elements,
// 952 us a call with the join's 15, or 1.0 PFLOP/s of the products, at a clock that falls to 1.7 GHz.  32 rows a wavefront, since 64 need more registers than there are
// (slower by the spills); 8 wavefronts over the same keys halve what is read again.  256 elements have one wavefront on a SIMD:
// 0.5 to 0.6 PFLOP/s; two there, with 32 of the 64 keys each, were not faster (their registers spill).
template <typename T, int NB>
struct Rows32 {
    static constexpr int CH = NB <= 2 ? 8 : NB <= 4 ? 16 : 32, PITCH = CH * 16;
    s16x8 q[2 * NB];
    f32x16 o[NB];        // sums
    float m, l, top;     // running maximum less BELOW and sum of weights, the scores' largest
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
        return *(const __attribute__((address_space(3))) s16x8*)(k + (k_at ^ (i % (2 * NB) * 32)) + i / (2 * NB) * 32 * PITCH);
    }
    __device__ __forceinline__ s16x8 values_at(lds_ptr v, int i) const {  // operand i of 4 NB: 32 elements by 16 keys
        const int x = i / NB, b = i % NB;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + (v_at ^ (b * 64)) + x * 16 * PITCH));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + (v_at ^ (b * 64) ^ 32) + (x * 16 + 8) * PITCH));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }

    // The first tile's scores
    __device__ __forceinline__ void scores(lds_ptr k, f32x16 (&s)[2]) {
        constexpr int N = 4 * NB, AHEAD = 6;
        s16x8 kf[AHEAD];
        for (int kb = 0; kb < 2; kb++) s[kb] = (f32x16)0.0f;
        for (int i = 0; i < AHEAD; i++) kf[i] = keys_at(k, i);
#pragma unroll
        for (int i = 0; i < N; i++) {
            s[i / (2 * NB)] = Mfma<T>::mul(kf[i % AHEAD], q[i % (2 * NB)], s[i / (2 * NB)]);
            if (i + AHEAD < N) kf[i % AHEAD] = keys_at(k, i + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        }
        largest(s);
    }

    __device__ __forceinline__ void largest(const f32x16 (&s)[2]) {
        top = -INFINITY;
        for (int i = 0; i < 32; i += 2) top = fmaxf(fmaxf(top, s[i >> 4][i & 15]), s[i >> 4][(i & 15) + 1]);
    }

    // Moves the running maximum if these scores rise far over it; c = scale * log2 e
    __device__ __forceinline__ void raise(float c) {
        const float t = both_halves_max(top) * c;
        if (ballot(t > m + BELOW<T> + 8.0f)) {
            const float to = fmaxf(t - BELOW<T>, m), keep = __builtin_amdgcn_exp2f(m - (to == -INFINITY ? 0.0f : to));
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
        constexpr int N = 4 * NB, AHEAD = 3;  // matrix instructions of each half, with 32 / N scores each
        const float base = m == -INFINITY ? 0.0f : m;
        s16x8 kf[AHEAD], vf[AHEAD], p[4];
        float w[8], sum = 0.0f;
        for (int i = 0; i < AHEAD; i++) kf[i] = keys_at(k, i);
#pragma unroll
        for (int i = 0; i < N; i++) {
            f32x16& to = next[i / (2 * NB)];  // the second half takes the registers that the first half's weights have left
            to = Mfma<T>::mul(kf[i % AHEAD], q[i % (2 * NB)], i % (2 * NB) ? to : (f32x16)0.0f);
            if (i + AHEAD < N) kf[i % AHEAD] = keys_at(k, i + AHEAD);
            else vf[i + AHEAD - N] = values_at(v, i + AHEAD - N);
#pragma unroll
            for (int e = i * 32 / N; e < (i + 1) * 32 / N; e++) {
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
            for (int e = i * 32 / N; e < (i + 1) * 32 / N; e++)
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

template <typename T, int NB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, NB <= 4 ? 2 : 1) void paged_many_kernel(PagedArgs g) {
    typedef Rows32<T, NB> R;
    constexpr int ROWS = WAVES * 32, THREADS = WAVES * 64, KEYS = UNIT, TILE = KEYS * R::PITCH;
    constexpr int LOADS = KEYS * R::CH / THREADS;
    extern __shared__ __attribute__((aligned(1024))) char lds[];  // [2] keys, [2] values; slots' sums of units, their requests
    const jx_attend_args& a = g.a;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const lds_ptr ring = (lds_ptr)lds;
    Shares sh;
    const bool any = sh.begin<ROWS, 1>(g, (int*)(lds + 4 * TILE), 0);
    sh.clear_rows<T>(g);
    if (!any) return;

    const int d = a.head_dim, page_mask = a.cache.page - 1;
    if (d < R::CH * 8)  // what lies behind a head meets zeros of the queries, so it has to be a number
        for (int i = tid; i < 4 * TILE / 16; i += THREADS) *(uint4*)(lds + i * 16) = make_uint4(0, 0, 0, 0);
    const uint32_t page_chunks = (uint32_t)(a.cache.page_stride / 8), token_chunks = (uint32_t)(a.cache.token_stride / 8);
    const float c = fmaxf(fabsf(a.scale) * LOG2E, __FLT_MIN__);  // a scale of 0 has to leave -infinity what it is
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
    while (sh.x0 < sh.x1) {
        const Segment e = sh.next<ROWS, 1>(g);
        const Tile& t = e.t;
        if (t.r < 0) return;
        const int work = sh.group, head = sh.head;
        const bool whole = e.whole();
        const int key0 = t.lo + e.u0 * KEYS, key1 = min(t.lo + e.u1 * KEYS, t.hi);

        // rows of this wavefront
        R x;
        x.begin();
        const int rows0 = ((wave + (g.n_work ? work : 0)) & (WAVES - 1)) * 32;  // tiles of few rows: the workgroups of a CU keep different SIMDs busy
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
        const uint32_t lane_row = lane / R::CH * token_chunks * 16, lane_chunk = lane % R::CH ^ mix<R::CH>(tid / R::CH);
        auto stage = [&](const char* from, int key, int ids, lds_ptr to) {
            if (g.near && !ballot(ids < 0)) {
                for (int i = 0; i < LOADS; i++) {
                    const int at = i * (THREADS / R::CH) + wave * (64 / R::CH), odd = mix<R::CH>(i * (THREADS / R::CH) & 15);
                    const uint64_t row = row_at(__builtin_amdgcn_readlane(ids, at), key + at);
                    const uint32_t off = lane_row + (lane_chunk ^ odd) * 16;
                    if (d == R::CH * 8) load_lds16(from + row * 16 + off, to + (i * THREADS + wave * 64) * 16);
                    else if ((lane_chunk ^ odd) * 8 < d)  // the other places are never written: see above
                        load_lds16(from + row * 16 + off, to + (i * THREADS + wave * 64) * 16);
                }
                return;
            }
            const uint64_t rows = row_at(max(ids, 0), key + lane);
#pragma unroll 1
            for (int i = 0; i < LOADS; i++) {
                const int at = i * (THREADS / R::CH) + tid / R::CH, chunk = tid % R::CH ^ mix<R::CH>(at);
                const char* p = from + ((uint64_t)shfl64((long long)rows, at) + chunk) * 16;
                load_lds16(__shfl(ids, at, 64) >= 0 && chunk * 8 < d ? p : (const char*)zero_chunk, to + (i * THREADS + wave * 64) * 16);
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
            part = sh.part(g, e.u0 == 0, NB) + rows0 / 32 * part_floats(NB);
            if (e.u0 == 0 && tid == 0) sh.name(g, t, sh.x0, e.units);
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
        sh.x0 += e.u1 - e.u0;
    }
}

template <typename T, int NB, int WAVES>
hipError_t launch(const PagedArgs& g, hipStream_t st) {
    constexpr int TILE = UNIT * Rows32<T, NB>::PITCH;
    const size_t lds = 4 * TILE + (g.n_work ? shares_bytes(g.a.n_req, g.slots) : 0);
    hipError_t e = hipFuncSetAttribute((const void*)paged_many_kernel<T, NB, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
    if (e != hipSuccess) return e;
    const unsigned blocks = g.n_work ? g.groups : (unsigned)(g.slots * g.a.n_kv_heads);
    paged_many_kernel<T, NB, WAVES><<<blocks ? blocks : 256, WAVES * 64, lds, st>>>(g);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_dim(const PagedArgs& g, int rows, hipStream_t st) {
    const bool wide = rows == 256;
    switch (blocks_of(g.a.head_dim)) {
        case 2: return wide ? launch<T, 2, 8>(g, st) : launch<T, 2, 4>(g, st);
        case 3: return wide ? launch<T, 3, 8>(g, st) : launch<T, 3, 4>(g, st);
        case 4: return wide ? launch<T, 4, 8>(g, st) : launch<T, 4, 4>(g, st);
        case 6: return launch<T, 6, 4>(g, st);
    }
    return launch<T, 8, 4>(g, st);
}

}  // namespace

hipError_t launch_paged_many(const PagedArgs& g, int rows, hipStream_t st) {
    return g.a.dtype == JX_BF16 ? launch_dim<__bf16>(g, rows, st) : launch_dim<_Float16>(g, rows, st);
}

}  // namespace jx
