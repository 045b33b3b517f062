// Attention of a step's new tokens over a paged cache: which kernel, and the join of tiles that workgroups shared.
#include "paged_tiles.h"

namespace jx {

namespace {

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
                const float* p = parts + (size_t)(2 * (work + i) + (i == 0)) * g.part_rows * part_floats(NB);
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
    int rows;  // of a tile: 16, 32: few rows, 128: many
    int slots, n_work, part_rows;
    int64_t joins, total;  // bytes before the joins, in all
};

Plan make_plan(const jx_attend_args& a) {
    const int nb = blocks_of(a.head_dim);
    Plan p = {};
    const long long rows = a.n_tokens * (a.n_heads / a.n_kv_heads);
    // few rows: those of 16 neighbouring keys have to lie in one page
    const bool pages = a.cache.page >= 16 && a.cache.token_stride < (1 << 25);
    p.rows = pages && rows <= 16ll * a.n_req ? 16 : pages && rows <= 32ll * a.n_req ? 32 : 128;
    p.part_rows = p.rows == 128 ? 4 : 1;
    p.slots = a.n_req ? (int)(rows / p.rows + a.n_req) : 0;
    const double units = ((double)a.table_pages * a.cache.page / UNIT + 1) * p.slots * a.n_kv_heads;  // at most
    // as many workgroups as the card holds at a time
    if (p.slots && p.slots <= MAX_SLOTS && units < 2e9) p.n_work = a.head_dim <= (p.rows == 128 ? 128 : 64) ? 512 : 256;
    auto up = [](int64_t x) { return (x + 255) & ~(int64_t)255; };
    p.joins = up((int64_t)2 * p.n_work * p.part_rows * part_floats(nb) * 4);
    p.total = p.joins + up((int64_t)p.n_work * sizeof(Join));
    return p;
}

template <typename T>
void join(const PagedArgs& g, hipStream_t st) {
    const int nb = blocks_of(g.a.head_dim);
    const dim3 grid(g.n_work, (g.a.head_dim + 31) / 32);
    switch (nb) {
        case 2: join_kernel<T, 2><<<grid, 256, 0, st>>>(g); break;
        case 3: join_kernel<T, 3><<<grid, 256, 0, st>>>(g); break;
        case 4: join_kernel<T, 4><<<grid, 256, 0, st>>>(g); break;
        case 6: join_kernel<T, 6><<<grid, 256, 0, st>>>(g); break;
        default: join_kernel<T, 8><<<grid, 256, 0, st>>>(g);
    }
}

}  // namespace

int64_t paged_attention_bytes(const jx_attend_args& a) { return make_plan(a).total; }

hipError_t launch_paged_attention(const jx_attend_args& a, uint8_t* work, hipStream_t st) {
    const Plan p = make_plan(a);
    const int rows = a.head_dim <= 64 ? 8 : a.head_dim <= 128 ? 4 : 2;
    const int near = a.cache.page >= rows && a.cache.token_stride * rows < (1 << 29);
    const int group = a.n_heads / a.n_kv_heads, bits = group == 1 ? 1 : log2_of(group - 1) + 1;
    const uint32_t mul = (uint32_t)(((1ull << (31 + bits)) + group - 1) / group);
    const PagedArgs g = {a, log2_of(a.cache.page), group, mul, (uint32_t)bits - 1, near, p.slots, p.n_work, p.part_rows, (float*)work,
                         (Join*)(work + p.joins)};
    hipError_t e = p.rows == 128 ? launch_paged_many(g, st) : launch_paged_few(g, p.rows, st);
    if (e != hipSuccess || !p.n_work) return e;
    if (a.dtype == JX_BF16) join<__bf16>(g, st);
    else join<_Float16>(g, st);
    return hipGetLastError();
}

}  // namespace jx
