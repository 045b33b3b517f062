// Paged attention of few rows for each request, above all of single tokens: tiles of 16 or 32 rows.
#include <limits.h>
#include <type_traits>
#include "paged_tiles.h"

namespace jx {

namespace {

template <typename T>
__device__ __forceinline__ f32x4 mul16(s16x8 a, s16x8 b, f32x4 c);
template <>
__device__ __forceinline__ f32x4 mul16<__bf16>(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Vec<__bf16>::x8, a), __builtin_bit_cast(Vec<__bf16>::x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x4 mul16<_Float16>(s16x8 a, s16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Vec<_Float16>::x8, a), __builtin_bit_cast(Vec<_Float16>::x8, b), c, 0, 0, 0);
}

// 16 bytes for each lane from from + off + step into LDS, zeros where off is OUTSIDE the 2 GiB after `from`.  A buffer load, not a
// global one: the compiler counts it, while with one of those on its way it waits for all that are where it wants the first.
constexpr uint32_t OUTSIDE = 0x80000000u;
__device__ __forceinline__ void load_lds16_at(const char* from, uint32_t off, uint32_t step, lds_ptr to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void*)from, 0, 0x7FFFFFFF, 0x00020000),
                                             (__attribute__((address_space(3))) void*)to, 16, off, step, 0, 0);
}

template <int N>
__device__ __forceinline__ void wait_loads() {  // until at most the N latest are on their way
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | 0x0F70 | (N >> 4) << 14);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The largest of two pairs of 16-bit values
__device__ __forceinline__ uint32_t max_pairs(uint32_t a, uint32_t b) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// S^T = K Q^T and O^T += V^T P^T as for many rows, by 16x16x32 matrix instructions.  Bound: the bytes of keys and values.  So every
// wavefront is a reader of its own, with a share of its own: it takes 32 keys at a time, K straight into registers, V into its own two
// places in LDS (where its transposed form is read), the next ones on their way while these are worked on, and waits for another
// only when its share is done.  Wavefronts that took a tile's keys in turn lost a fifth of the time where they met at its end.
// The shares of a workgroup follow each other, so that tiles which they cut are put together in LDS, and only those which the
// workgroup itself found begun or leaves open are left for join_kernel.  Few short tiles are a workgroup's own (g.own) and joined by it.
// 64 requests of up to 8,192 keys, 8 key heads of 128 elements: 138 us, 5.0 TB/s; 4 of up to 131,072: 255 us, 5.5 TB/s; one of 777: 8.
template <typename T, int NC, int RB, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void paged_few_kernel(PagedArgs g) {
    constexpr int ROWS = RB * 16, KEYS = 32, CH = NC <= 2 ? 8 : NC <= 4 ? 16 : 32, PITCH = CH * 16, TILE = KEYS * PITCH;
    constexpr int NV = KEYS * CH / 64, NK = 2 * NC, OB = 2 * NC;
    extern __shared__ __attribute__((aligned(1024))) char lds[];  // [WAVES][2] values, at last sums of open tiles; shares
    __shared__ float wave_m[WAVES][ROWS], wave_l[WAVES][ROWS];
    enum { CLOSED, BEGUN, WITHIN };  // how a share ends: with a tile, in one that it has begun, in one that it lies in
    __shared__ int wave_end[WAVES];
    const jx_attend_args& a = g.a;
    const int tid = threadIdx.x, lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, h = lane >> 4, d = a.head_dim;
    Shares sh;
    const bool any = sh.begin<ROWS, WAVES>(g, (int*)(lds + WAVES * 2 * TILE), wave);
    sh.clear_rows<T>(g);
    if (!any && !g.n_work) return;

    const int page_mask = a.cache.page - 1;
    const uint32_t page_chunks = (uint32_t)(a.cache.page_stride / 8), token_chunks = (uint32_t)(a.cache.token_stride / 8);
    const float c = fmaxf(fabsf(a.scale) * LOG2E, __FLT_MIN__);  // a scale of 0 has to leave -infinity what it is
    const uint32_t flip = a.scale < 0.0f ? 0x80008000u : 0u;
    const lds_ptr mine = (lds_ptr)lds + wave * 2 * TILE;
    // a lane's place in 16 keys; of a head that ends inside a block the last chunk is read once more, against zeros of the queries
    const uint32_t k_row = r16 * token_chunks * 16;
    auto k_chunk = [&](int i) { return (uint32_t)min(i * 4 + h, d / 8 - 1) * 16; };
    // a lane's place in the 64 / CH rows of one load of values
    const uint32_t v_row = lane / CH * token_chunks * 16, v_chunk = lane % CH ^ mix<CH>(lane / CH);
    auto v_off = [&](int i) {
        const uint32_t chunk = v_chunk ^ mix<CH>(i * (64 / CH) & 15);
        return v_row + min(chunk, (uint32_t)d / 8 - 1) * 16;
    };
    const int vr = 4 * h + (r16 >> 2), v_at = vr * PITCH + ((r16 >> 1 & 1) ^ mix<CH>(vr)) * 16 + (r16 & 1) * 8;

    const f32x8 none = {0, 0, 0, 0, 0, 0, 0, 0};
    Tile t;
    int head = 0, ends = CLOSED, units = 0;
    // a row of the tile, by its number
    auto row_of = [&](int row) {
        const int rr = t.first + min(row, t.count - 1), token = by_group(g, rr);
        return RowAt{row < t.count, head * g.group + rr - token * g.group, t.start + token, t.p0 + token - by_group(g, t.first)};
    };
    // the result of 16 rows; l: the weights' whole sum
    auto write_rows = [&](int b, const f32x4 (&o)[OB], float m, float l) {
        const RowAt row = row_of(b * 16 + r16);
        if (!row.mine) return;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        const long long at = (long long)row.token * a.n_heads + row.head;
        T* out = (T*)a.d_out + at * d + h * 4;
        for (int i = 0; i < OB; i++) {
            f32x4 w = o[i];
            for (int j = 0; j < 4; j++) w[j] *= inv;
            if (i * 16 + h * 4 < d) *(typename Vec<T>::x4*)(out + i * 16) = __builtin_convertvector(w, typename Vec<T>::x4);
        }
        if (h == 0 && a.d_lse) a.d_lse[at] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
    };
    auto write_part = [&](float* part, int b, const f32x4 (&o)[OB], float m, float l) {
        if (b * 16 + r16 >= t.count) return;
        for (int i = 0; i < OB; i++) *(f32x4*)(part + part_at(b * 16 + r16, i * 16 + h * 4)) = o[i];
        if (h < 2) part[NC * 1024 + h * 32 + b * 16 + r16] = h ? l : m;
    };
    while (sh.x0 < sh.x1) {
        const Segment e = sh.next<ROWS, WAVES>(g);
        t = e.t;
        if (t.r < 0) return;
        if (e.u0 == e.u1) break;  // more wavefronts than units
        head = sh.head;
        units = e.units;
        const int key0 = t.lo + e.u0 * UNIT, key1 = min(t.lo + e.u1 * UNIT, t.hi);
        const char* kb = (const char*)a.cache.d_k + head * a.cache.head_stride * 2;
        const char* vb = (const char*)a.cache.d_v + head * a.cache.head_stride * 2;
        const int32_t* table = a.d_table + (size_t)t.r * a.table_pages;
        const __attribute__((address_space(4))) int32_t* table_s = (const __attribute__((address_space(4))) int32_t*)table;

        // Keys key .. key + 15 lie in one page (a page has at least 16 tokens, and key is a multiple of 16); scalar reads
        struct Pages {
            int id[2];  // of 16 keys each
        };
        auto there = [&](int id) { return (uint32_t)id < (uint32_t)a.cache.n_pages; };
        auto pages_at = [&](int key) {
            Pages p;
            for (int b = 0; b < 2; b++) p.id[b] = key + b * 16 < key1 ? table_s[(key + b * 16) >> g.page_shift] : -1;
            return p;
        };
        auto row_at = [&](int id, int key) {  // page 0 stands for one that is not there
            return ((uint64_t)(there(id) ? id : 0) * page_chunks + (uint64_t)(uint32_t)(key & page_mask) * token_chunks) * 16;
        };
        s16x8 k[2][NC];
        auto load_keys = [&](int key, const Pages& p) {
            for (int b = 0; b < 2; b++) {
                const char* from = kb + row_at(p.id[b], key + b * 16);
                for (int i = 0; i < NC; i++) k[b][i] = *(const s16x8*)(from + k_row + k_chunk(i));
            }
        };
        // Zeros for values that are not there: their place is outside the range.  No branch: the loads that are on their way have to be as
        // many on every path for the compiler to count them.
        auto load_values = [&](int key, const Pages& p, lds_ptr to) {
            const int left = key1 - key - (int)(lane / CH);
            for (int b = 0; b < 2; b++) {
                const char* from = vb + row_at(p.id[b], key + b * 16);
                const int rows = there(p.id[b]) ? left : INT_MIN;
                for (int i = b * NV / 2; i < (b + 1) * NV / 2; i++)
                    load_lds16_at(from, i * (64 / CH) < rows ? v_off(i) : OUTSIDE, (i - b * NV / 2) * (64 / CH) * 16 * token_chunks, to + i * 1024);
            }
        };
        Pages here = pages_at(key0), next = pages_at(key0 + KEYS);
        load_keys(key0, here);
        load_values(key0, here, mine);

        int pos[RB];
        s16x8 q[RB][NC];
        for (int b = 0; b < RB; b++) {
            const RowAt row = row_of(b * 16 + r16);
            pos[b] = row.pos;
            const T* from = (const T*)a.d_q + (long long)row.token * a.q_token_stride + row.head * a.q_head_stride + h * 8;
            for (int i = 0; i < NC; i++) {
                uint4 w = i * 32 + h * 8 < d && row.mine ? *(const uint4*)(from + i * 32) : make_uint4(0, 0, 0, 0);
                w = make_uint4(w.x ^ flip, w.y ^ flip, w.z ^ flip, w.w ^ flip);
                q[b][i] = __builtin_bit_cast(s16x8, w);
            }
        }
        f32x4 o[RB][OB];
        float m[RB], l[RB];
        for (int b = 0; b < RB; b++) {
            m[b] = -INFINITY;
            l[b] = 0.0f;
            for (int i = 0; i < OB; i++) o[b][i] = (f32x4)0.0f;
        }
        uint32_t worst = 0;  // the largest pair of values, signs aside, where not every row looks
        // 32 keys; while they are worked on the next ones are on their way, the keys into the registers that the scores have been made of,
        // the values into the other place.  The compiler has to know that this is another: it would wait for it.
        auto work_on = [&](auto more, int key, const Pages& here, const Pages& next, const lds_ptr __restrict v,
                           const lds_ptr __restrict next_v) __attribute__((always_inline)) {
            if (more) load_values(key + KEYS, next, next_v);
            f32x4 s[RB][2];
            for (int b = 0; b < RB; b++)
                for (int x = 0; x < 2; x++) s[b][x] = (f32x4)0.0f;
            for (int i = 0; i < NC; i++)
                for (int x = 0; x < 2; x++)
                    for (int b = 0; b < RB; b++) s[b][x] = mul16<T>(k[x][i], q[b][i], s[b][x]);
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_keys(key + KEYS, next);
            // what is not seen, and the weights
            const bool all = key + KEYS <= key1 && there(here.id[0]) && there(here.id[1]) && key + KEYS - 1 <= t.p0 && (!a.window || key > t.p1 - a.window);
            s16x8 p[RB];
            for (int b = 0; b < RB; b++) {
                if (!all) {
                    const int last = min(pos[b], key1 - 1) - key - 4 * h, first = a.window ? max(pos[b] + 1 - a.window - key, 0) - 4 * h : -4 * h;
                    for (int x = 0; x < 2; x++) {
                        const int most = there(here.id[x]) ? last - x * 16 : INT_MIN;
                        for (int i = 0; i < 4; i++) s[b][x][i] = i <= most && i >= first - x * 16 ? s[b][x][i] : -INFINITY;
                    }
                }
                float top = -INFINITY;
                for (int i = 0; i < 8; i += 2) top = fmaxf(fmaxf(top, s[b][i >> 2][i & 3]), s[b][i >> 2][(i & 3) + 1]);
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64)) * c;
                if (ballot(top > m[b] + BELOW<T> + 8.0f)) {  // the running maximum moves only for a rise by more than 2^8, as for many rows
                    const float to = fmaxf(top - BELOW<T>, m[b]), keep = __builtin_amdgcn_exp2f(m[b] - (to == -INFINITY ? 0.0f : to));
                    m[b] = to;
                    l[b] *= keep;
                    for (int i = 0; i < OB; i++)
                        for (int j = 0; j < 4; j++) o[b][i][j] *= keep;
                }
                const float base = m[b] == -INFINITY ? 0.0f : m[b];
                f32x8 w;
                for (int i = 0; i < 8; i++) {
                    w[i] = __builtin_amdgcn_exp2f(fmaf(s[b][i >> 2][i & 3], c, -base));
                    l[b] += w[i];
                }
                p[b] = __builtin_bit_cast(s16x8, __builtin_convertvector(w, typename Vec<T>::x8));
            }
            if (more) wait_loads<NV + NK>();
            else wait_loads<0>();
            constexpr int AT_ONCE = RB == 1 ? OB : OB / 2;  // by the registers that are free
            for (int i0 = 0; i0 < OB; i0 += AT_ONCE) {
                s16x8 y[AT_ONCE];
                for (int i = 0; i < AT_ONCE; i++) {
                    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + (v_at ^ ((i0 + i) * 32))));
                    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(v + (v_at ^ ((i0 + i) * 32)) + 16 * PITCH));
                    y[i] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (!all)
                    for (int i = 0; i < AT_ONCE; i++) {
                        const uint4 w = __builtin_bit_cast(uint4, y[i]);
                        worst = max_pairs(worst, max_pairs(max_pairs(w.x & 0x7FFF7FFFu, w.y & 0x7FFF7FFFu), max_pairs(w.z & 0x7FFF7FFFu, w.w & 0x7FFF7FFFu)));
                    }
                for (int i = 0; i < AT_ONCE; i++)
                    for (int b = 0; b < RB; b++) o[b][i0 + i] = mul16<T>(y[i], p[b], o[b][i0 + i]);
            }
            __builtin_amdgcn_sched_barrier(0);  // the place has been read before it is filled again
        };
        if (key0 < key1) {
            int key = key0, buf = 0;
            for (; key + KEYS < key1; key += KEYS, buf ^= TILE) {
                const Pages then = pages_at(key + 2 * KEYS);
                work_on(std::true_type{}, key, here, next, mine + buf, mine + (buf ^ TILE));
                here = next;
                next = then;
            }
            work_on(std::false_type{}, key, here, next, mine + buf, mine + (buf ^ TILE));
        } else {
            wait_loads<0>();  // what was on its way for a tile without keys
        }

        // Results: of a whole tile, of a part that ends one, or of one that is open at the share's end
        const bool whole = e.whole(), open = !whole && (g.own || e.u1 < e.units);
        if (open) ends = e.u0 == 0 ? BEGUN : WITHIN;
        float* part = whole || open ? NULL : wave == 0 ? sh.part(g, false, NC) : sh.inner(g, sh.work, NC);
        float* sums = (float*)(lds + wave * 2 * TILE);  // [RB][OB][64][4], as the lanes hold them
        constexpr uint32_t ODD = __is_same(T, __bf16) ? 0x7F80u : 0x7C00u;  // infinities and what is not a number
        if (!ballot((worst & 0xFFFF) >= ODD || worst >> 16 >= ODD)) {
            for (int b = 0; b < RB; b++) {
                float sum = l[b] + __shfl_xor(l[b], 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                if (whole) {
                    write_rows(b, o[b], m[b], sum);
                } else if (!open) {
                    write_part(part, b, o[b], m[b], sum);
                } else {
                    for (int i = 0; i < OB; i++) *(f32x4*)(sums + ((b * OB + i) * 64 + lane) * 4) = o[b][i];
                    if (h == 0) {
                        wave_m[wave][b * 16 + r16] = m[b];
                        wave_l[wave][b * 16 + r16] = sum;
                    }
                }
            }
        } else {
            // A weight of 0 times such a value is not 0: these rows are done again, key by key
            const int c8 = lane % CH * 8;
            for (int i = 0; i < t.count; i++) {
                const RowAt row = row_of(i);
                f32x8 x = none;
                if (c8 < d) x = load8((const T*)a.d_q + (long long)row.token * a.q_token_stride + row.head * a.q_head_stride + c8);
                for (int j = 0; j < 8; j++) x[j] *= a.scale * LOG2E;
                const int k0 = a.window ? max(key0, row.pos + 1 - a.window) : key0, k1 = min(key1, row.pos + 1);
                Softmax s = walk_keys<T, CH>((const T*)kb, (const T*)vb, x, c8 < d, k0, k1, [&](long long at) {
                    const int id = table[at >> g.page_shift];
                    return there(id) ? (long long)row_at(id, (int)at) / 2 : -1ll;
                });
                s = gather<CH>(s);
                const long long out = (long long)row.token * a.n_heads + row.head;
                if (whole) {
                    const float inv = s.l == 0.0f ? 0.0f : 1.0f / s.l;
                    for (int j = 0; j < 8; j++) s.acc[j] *= inv;
                    if (lane < CH && c8 < d) store8((T*)a.d_out + out * d + c8, s.acc);
                    if (lane == 0 && a.d_lse) a.d_lse[out] = s.l == 0.0f ? -INFINITY : (s.m + __builtin_amdgcn_logf(s.l)) * LN2;
                } else if (!open) {
                    if (lane < CH && c8 < d)
                        for (int j = 0; j < 8; j++) part[part_at(i, c8 + j)] = s.acc[j];
                    if (lane == 0) {
                        part[NC * 1024 + i] = s.m;
                        part[NC * 1024 + 32 + i] = s.l;
                    }
                } else {
                    if (lane < CH && c8 < OB * 16)
                        for (int j = 0; j < 8; j++) sums[((i / 16 * OB + c8 / 16) * 64 + ((c8 + j) / 4 & 3) * 16 + i % 16) * 4 + (j & 3)] = s.acc[j];
                    if (lane == 0) {
                        wave_m[wave][i] = s.m;
                        wave_l[wave][i] = s.l;
                    }
                }
            }
        }
        if (open) break;  // the share's last
        sh.x0 += e.u1 - e.u0;
    }
    if (!g.n_work && !g.own) return;

    // Tiles that shares of this workgroup have cut: the first of them takes what the others have added
    if (lane == 0) wave_end[wave] = ends;
    __syncthreads();
    if (ends == CLOSED || (ends == WITHIN && wave > 0)) return;
    for (int b = 0; b < RB; b++) {
        f32x4 o[OB];
        for (int i = 0; i < OB; i++) o[i] = *(const f32x4*)(lds + wave * 2 * TILE + ((b * OB + i) * 64 + lane) * 16);
        float m = wave_m[wave][b * 16 + r16], l = wave_l[wave][b * 16 + r16];
        auto add = [&](float pm, float pl, auto sums_of) {
            const float top = fmaxf(m, pm), base = top == -INFINITY ? 0.0f : top;
            const float keep = __builtin_amdgcn_exp2f(m - base), w = __builtin_amdgcn_exp2f(pm - base);
            m = top;
            l = l * keep + pl * w;
            for (int i = 0; i < OB; i++) {
                const f32x4 y = sums_of(i);
                for (int j = 0; j < 4; j++) o[i][j] = fmaf(y[j], w, o[i][j] * keep);
            }
        };
        int w = wave + 1;
        for (; w < sh.active && wave_end[w] == WITHIN; w++)
            add(wave_m[w][b * 16 + r16], wave_l[w][b * 16 + r16],
                [&](int i) { return *(const f32x4*)(lds + w * 2 * TILE + ((b * OB + i) * 64 + lane) * 16); });
        const bool ended = w < sh.active;  // its share begins with the tile's end
        if (ended && b * 16 + r16 < t.count) {
            const float* part = sh.inner(g, sh.work + w - wave, NC);
            add(part[NC * 1024 + b * 16 + r16], part[NC * 1024 + 32 + b * 16 + r16],
                [&](int i) { return *(const f32x4*)(part + part_at(b * 16 + r16, i * 16 + h * 4)); });
        }
        if (ends == BEGUN && (ended || g.own)) write_rows(b, o, m, l);
        else write_part(sh.part(g, ends == BEGUN, NC), b, o, m, l);
        if (ends == BEGUN && !ended && !g.own && b == 0 && lane == 0) sh.name(g, t, sh.x0, units);
    }
}

template <typename T, int NC, int RB>
hipError_t launch(const PagedArgs& g, hipStream_t st) {
    constexpr int WAVES = FEW_WAVES(NC), CH = NC <= 2 ? 8 : NC <= 4 ? 16 : 32;
    const size_t lds = WAVES * 2 * 32 * CH * 16 + (g.n_work ? shares_bytes(g.a.n_req, g.slots) : 0);
    hipError_t e = hipFuncSetAttribute((const void*)paged_few_kernel<T, NC, RB, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, 150 * 1024);
    if (e != hipSuccess) return e;
    const unsigned tiles = (unsigned)(g.slots * g.a.n_kv_heads), blocks = g.n_work ? g.groups : g.own ? tiles : (tiles + WAVES - 1) / WAVES;
    paged_few_kernel<T, NC, RB, WAVES><<<blocks ? blocks : 256, WAVES * 64, lds, st>>>(g);
    return hipGetLastError();
}

template <typename T, int RB>
hipError_t launch_dim(const PagedArgs& g, hipStream_t st) {
    switch (blocks_of(g.a.head_dim)) {
        case 2: return launch<T, 2, RB>(g, st);
        case 3: return launch<T, 3, RB>(g, st);
        case 4: return launch<T, 4, RB>(g, st);
        case 6: return launch<T, 6, RB>(g, st);
    }
    return launch<T, 8, RB>(g, st);
}

}  // namespace

hipError_t launch_paged_few(const PagedArgs& g, int rows, hipStream_t st) {
    if (g.a.dtype == JX_BF16) return rows == 16 ? launch_dim<__bf16, 1>(g, st) : launch_dim<__bf16, 2>(g, st);
    return rows == 16 ? launch_dim<_Float16, 1>(g, st) : launch_dim<_Float16, 2>(g, st);
}

}  // namespace jx
