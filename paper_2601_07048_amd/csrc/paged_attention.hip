// Attention of a step's new tokens over a paged cache: which kernel, and the join of tiles that workgroups shared.
#include <algorithm>
#include <type_traits>
#include "paged_tiles.h"

namespace jx {

namespace {

// Threads of a workgroup: a wavefront for eight elements of a tile's rows.  Small ones, since most of those of a launch have nothing to
// join, and a tile of many pieces is read by as many CUs
constexpr int JOIN_THREADS = 256;

// The parts of a tile whose keys several workgroups share, as one: the tile that workgroup blockIdx.x began and did not end;
// blockIdx.y: which 32 rows.  A wavefront takes 8 elements, as the lanes held them when the parts were written, and of few rows
// two or four pieces side by side.  Bound: the time that a chain of reads takes, hence PIECES at once, but two or four where there
// are no more (8 always: 27 and not 16 us for a chunk of 4,096 tokens): single tokens of 64 requests 4.8 us, 40 MB of parts of
// 256 elements 15.2.
template <typename T, int NB>
__global__ __launch_bounds__(JOIN_THREADS) void join_kernel(PagedArgs g) {
    constexpr int PIECES = 8;
    const jx_attend_args& a = g.a;
    const int lane = lane_id(), e0 = (int)((blockIdx.z * blockDim.x + threadIdx.x) >> 6) * 8, d = a.head_dim;
    const Join j = g.joins[blockIdx.x];
    const int count = j.pieces ? j.count - (int)blockIdx.y * 32 : 0;
    if (count <= 0 || e0 >= d) return;
    const int wide = count <= 8 ? 16 : count <= 16 ? 32 : 64, side = 64 / wide;  // lanes of a piece, pieces side by side
    const int row = lane & (wide / 2 - 1), half = lane / (wide / 2) & 1;
    const float* parts = g.part + blockIdx.y * part_floats(NB);
    const int to_s = part_at(row, e0 + half * 4), to_m = NB * 1024 + row;
    float m = -INFINITY, l = 0.0f;
    f32x4 s = {0, 0, 0, 0};
    // A piece is one by its number, not by its largest score: that of scores which are not numbers is -infinity, and they have to
    // reach the result.  One without keys adds zeros.
    auto take = [&](auto at_once, int i0) {
        constexpr int N = at_once;
        float pm[N], pl[N], top = m;
        f32x4 y[N];
        for (int u = 0; u < N; u++) {
            const int i = min(i0 + u * side, j.pieces - 1);
            const float* p = parts + (size_t)(2 * (blockIdx.x + i) + (i == 0)) * g.part_rows * part_floats(NB);
            pm[u] = p[to_m];
            pl[u] = p[to_m + 32];
            y[u] = *(const f32x4*)(p + to_s);
        }
        for (int u = 0; u < N; u++) {
            if (i0 + u * side >= j.pieces) pm[u] = -INFINITY;
            top = fmaxf(top, pm[u]);
        }
        const float base = top == -INFINITY ? 0.0f : top, keep = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= keep;
        for (int e = 0; e < 4; e++) s[e] *= keep;
        for (int u = 0; u < N; u++) {
            const float w = __builtin_amdgcn_exp2f(pm[u] - base);
            const bool counts = i0 + u * side < j.pieces;
            l = counts ? fmaf(pl[u], w, l) : l;
            for (int e = 0; e < 4; e++) s[e] = counts ? fmaf(y[u][e], w, s[e]) : s[e];
        }
    };
    const int i0 = lane / wide;
    if (j.pieces <= 2 * side) take(std::integral_constant<int, 2>(), i0);
    else if (j.pieces <= 4 * side) take(std::integral_constant<int, 4>(), i0);
    else
        for (int i = 0; i < j.pieces; i += PIECES * side) take(std::integral_constant<int, PIECES>(), i0 + i);
    float top = m;
    for (int x = wide; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float keep = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    l *= keep;
    for (int e = 0; e < 4; e++) s[e] *= keep;
    for (int x = wide; x < 64; x *= 2) {
        l += __shfl_xor(l, x, 64);
        for (int e = 0; e < 4; e++) s[e] += __shfl_xor(s[e], x, 64);
    }
    if (lane >= wide || row >= count) return;
    const int rr = j.first + (int)blockIdx.y * 32 + row, token = by_group(g, rr);
    const long long o = (j.start + (long long)token) * a.n_heads + j.head * g.group + rr - token * g.group;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    for (int i = 0; i < 4; i++) s[i] *= inv;
    const int e = e0 + half * 4;
    if (e < d) *(typename Vec<T>::x4*)((T*)a.d_out + o * d + e) = __builtin_convertvector(s, typename Vec<T>::x4);
    if (e0 == 0 && half == 0 && a.d_lse) a.d_lse[o] = l == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * LN2;
}

struct Plan {
    int rows;  // of a tile: 16, 32: few rows, 64, 128, 256: many
    int slots, groups, n_work, columns, part_rows, own;
    int64_t joins, total;  // bytes before the joins, in all
};

Plan make_plan(const jx_attend_args& a, bool coded) {
    const int nb = blocks_of(a.head_dim);
    Plan p = {};
    const long long rows = a.n_tokens * (a.n_heads / a.n_kv_heads);
    // Few rows: the 16 neighbouring keys that a load takes have to lie in one page.  16 for what is mostly single tokens; 32 where the
    // cache has little room for each request, since a request of more rows reads its keys once for every tile (32 or 128 rows: 64
    // requests of up to 8 tokens, 4 heads, up to 300 keys 20 or 31 us; 32 of up to 16 tokens, 4,000 keys 69 or 55).
    // Many rows: 256 where most tiles are full (256 or 128 rows: a chunk of 4,096 over 16,384 keys 967 or 1,080 us; eight
    // chunks of up to 512 152 or 131).  One height for all requests, by their mean: 256 single tokens of 4,000 keys and a chunk of 512
    // are all taken 16 rows at a time, in 877 us; 735 and 68 apart.
    const bool pages = a.cache.page >= 16 && a.cache.token_stride < (1 << 25);
    const bool little = (int64_t)a.cache.n_pages * a.cache.page <= 512ll * a.n_req;
    const long long full = a.n_req == 1 ? 512 : 2048;
    if (pages && rows <= 16ll * a.n_req) p.rows = 16;
    else if (pages && little && rows <= 32ll * a.n_req) p.rows = 32;
    else p.rows = nb <= 4 && rows >= full * a.n_req ? 256 : 128;
    // Of codes with a key head for each query head, 64 of up to 64 elements, where requests have as many on the mean: a conversion serves few rows then,
    // and what waits for it is hidden by more workgroups on a CU.  Means of up to 64 rows, 4 to 16 heads, 12 to 100 requests: tiles of 128 take
    // 1.07 of the time (0.76 to 1.39), alike chunks without a window 1.16 (60 of 64 tokens, 600 keys, 16 heads 46 or 59 us).  65 to 128: alike chunks 0.82 to 0.97
    // (20 of 128 over 3,000 keys 92 or 76), mixes 0.96 to 1.03 (33 of 1 to 509, most of them short, over 500 to 8,000 keys with a window of 1,024: 69 or
    // 77, without 128 or 139).  129 to 192: 0.94 to 1.01 (50 of 1 to 256 over 2,000 keys 131 or 122).  4 or 2 query heads to a key head, 64 chunks of up
    // to 33 over 1,000 keys: 42 or 39.
    // Four workgroups of 64 rows have room on a CU while what each holds of the requests for the shares fits into the rest of its quarter of the LDS
    // (with more tiles than are shared out it holds nothing). Beyond that three do, and a fourth of the shares runs after the others: requests
    // of 1 to 79 tokens, up to 600 keys, 440 of them with 8 heads 108 us or, of 128 rows, 122, 460 of them with 4 heads 73 or 81; 480 of them with
    // 8 heads 180 or 136, with 4 heads 117 or 81.
    const int low = (int)(rows / 64 + a.n_req);
    const bool four = low > MAX_SLOTS || (int64_t)shares_bytes(a.n_req, low) <= MANY_LDS / MANY_PER_CU(2, 64) - 4 * UNIT * 128;
    if (coded && nb == 2 && a.n_heads == a.n_kv_heads && p.rows == 128 && rows <= 64ll * a.n_req && four) p.rows = 64;
    p.part_rows = (p.rows + 31) / 32;
    p.slots = a.n_req ? (int)(rows / p.rows + a.n_req) : 0;
    // Few tiles of few rows and few keys (a table with little room, a short window): a workgroup a tile, which its wavefronts put
    // together, and no second launch.  The host has the room, not the lengths: neither this nor 32 rows is taken where pool and table
    // are sized for more than the step's requests hold.  128 elements, 8 key heads, 16 requests of up to 256 or 512 keys: 8.9 or 12.7 us, shared out
    // 11.1 or 12.5; 64 requests 18 or 16.  64 elements, 16 key heads, 16 requests of up to 1,024 keys: 10.9, shared out 18.4.
    const int64_t room = (int64_t)a.table_pages * a.cache.page, keys = a.window ? std::min<int64_t>(room, (int64_t)a.window + 16) : room;
    const int64_t tiles = (int64_t)p.slots * a.n_kv_heads, few = 1024 / (nb <= 2 ? 1 : nb);
    p.own = p.rows < 64 && tiles <= 384 && keys <= few;
    // Of codes also where there are tiles for most CUs: 8 key heads of 128, single tokens of 250 / 500 / 1,000 keys, a request 10.0 / 11.7 / 14.7 us
    // (shared out 10.4 / 10.5 / 11.9), 4 requests 10.3 / 12.2 / 15.1 (11.5 / 12.0 / 13.2), 16 requests 10.5 / 12.4 / 16.0 (13.7 / 18.9 / 21.2).
    if (coded && p.rows < 64 && tiles <= 256) p.own = p.own || keys <= std::min(4 * few, tiles * 64 / nb);
    const double units = ((double)a.table_pages * a.cache.page / (coded ? UNIT / 2 : UNIT) + 1) * p.slots * a.n_kv_heads;  // at most
    // as many shares as the card holds workgroups (many rows) or wavefronts (few) at a time
    if (p.slots && !p.own && p.slots <= MAX_SLOTS && units < 2e9) {
        p.groups = 256 * (p.rows >= 64 ? MANY_PER_CU(nb, p.rows) : nb <= 2 ? 2 : 1);
        p.n_work = p.rows >= 64 ? p.groups : p.groups * FEW_WAVES(nb);
    }
    p.columns = 1;
    if (coded && p.rows < 64)
        while (p.columns < 4 && a.n_kv_heads % (2 * p.columns) == 0) p.columns *= 2;
    auto up = [](int64_t x) { return (x + 255) & ~(int64_t)255; };
    p.joins = up(((int64_t)2 * p.groups * p.columns * p.part_rows + (p.rows >= 64 ? 0 : p.n_work)) * part_floats(nb) * 4);
    p.total = p.joins + up((int64_t)p.groups * p.columns * sizeof(Join));
    return p;
}

template <typename T, int NB>
void join(const PagedArgs& g, hipStream_t st) {
    join_kernel<T, NB><<<dim3(g.groups * g.columns, g.part_rows, NB * 256 / JOIN_THREADS), JOIN_THREADS, 0, st>>>(g);
}

template <typename T>
void join_dim(const PagedArgs& g, hipStream_t st) {
    switch (blocks_of(g.a.head_dim)) {
        case 2: return join<T, 2>(g, st);
        case 3: return join<T, 3>(g, st);
        case 4: return join<T, 4>(g, st);
        case 6: return join<T, 6>(g, st);
    }
    join<T, 8>(g, st);
}

}  // namespace

namespace {

hipError_t launch(const jx_attend_args& a, const jx_kv_scales* s, uint8_t* work, hipStream_t st) {
    const Plan p = make_plan(a, s != NULL);
    const int rows = (a.head_dim <= 64 ? 8 : a.head_dim <= 128 ? 4 : 2) * (s ? 2 : 1);  // that a load of a wavefront takes
    const int near = a.cache.page >= rows && a.cache.token_stride * rows < (1 << 29);
    const int group = a.n_heads / a.n_kv_heads, bits = group == 1 ? 1 : log2_of(group - 1) + 1;
    const uint32_t mul = (uint32_t)(((1ull << (31 + bits)) + group - 1) / group);
    const Scales scales = s ? Scales{s->d_k, s->d_v, log2_of(s->block), a.cache.page / s->block} : Scales{};
    const PagedArgs g = {a, scales, log2_of(a.cache.page), group, mul, (uint32_t)bits - 1, near, p.slots, p.groups, p.n_work, p.columns, p.part_rows, p.own,
                         (float*)work, (Join*)(work + p.joins)};
    hipError_t e = p.rows >= 64 ? (s ? launch_paged_many8 : launch_paged_many)(g, p.rows, st) : (s ? launch_paged_few8 : launch_paged_few)(g, p.rows, st);
    if (e != hipSuccess || !p.n_work) return e;
    if (a.dtype == JX_BF16) join_dim<__bf16>(g, st);
    else join_dim<_Float16>(g, st);
    return hipGetLastError();
}

}  // namespace

int64_t paged_attention_bytes(const jx_attend_args& a) { return make_plan(a, false).total; }
int64_t paged_attention8_bytes(const jx_attend_args& a) { return make_plan(a, true).total; }

hipError_t launch_paged_attention(const jx_attend_args& a, uint8_t* work, hipStream_t st) { return launch(a, NULL, work, st); }
hipError_t launch_paged_attention8(const jx_attend_args& a, const jx_kv_scales& s, uint8_t* work, hipStream_t st) { return launch(a, &s, work, st); }

}  // namespace jx
