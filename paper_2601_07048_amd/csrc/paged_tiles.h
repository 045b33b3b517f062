// Tiles of a paged attention call: what they are, how they are shared out over workgroups, how rows lie in LDS.
#pragma once
#include <atomic>
#include "attend_walk.h"
#include "codes8.h"

namespace jx {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int MAX_SLOTS = 1024;  // tiles that are shared out by keys, see Shares

// A tile whose keys several workgroups share: part 2 group + 1 of the first of them, 2 group of the pieces - 1 that follow.  0 pieces: none
struct __attribute__((aligned(16))) Join {
    int pieces, head, first, count;  // of the tile: key head, first row and number of rows
    int start, unused[3];            // of the request: its first row of q
};

struct PagedArgs {
    jx_attend_args a;
    Scales scales;          // of keys and values in 8 bits
    int page_shift, group;  // group: query heads of a key head
    uint32_t group_mul, group_shift;  // see by_group
    int near;               // whether the rows that one load of a wavefront takes lie in one page, less than 2^31 bytes apart
    int slots;              // tiles at most
    int groups, n_work;     // workgroups, and shares of all tiles (1 or FEW_WAVES for each workgroup); 0 = a share a tile
    int columns;            // of few rows: key heads that the wavefronts of a workgroup share between them, see Shares; each has parts of its own
    int part_rows;          // tiles' rows / 32
    int own;                // few rows, n_work = 0: whether a workgroup takes a tile, not a wavefront
    float* part;            // [2 groups columns][part_rows], and [n_work] of few rows inside workgroups: of 32 rows, over a part of a tile's
                            // keys, sums [NB][4][64][4], largest scores and weights' sums [2][32]; the sums as a wavefront holds
                            // them, see part_at
    Join* joins;            // [columns][groups]
};

hipError_t launch_paged_many(const PagedArgs& g, int rows, hipStream_t st);  // rows: of a tile, 128, or 256 up to 128 elements
hipError_t launch_paged_few(const PagedArgs& g, int rows, hipStream_t st);  // rows: of a tile, 16 or 32
hipError_t launch_paged_many8(const PagedArgs& g, int rows, hipStream_t st);  // over keys and values in 8 bits; 64 too up to 64 elements
hipError_t launch_paged_few8(const PagedArgs& g, int rows, hipStream_t st);

// wavefronts of a workgroup that takes few rows, by blocks of 32 elements: as many as have room for their values in LDS
constexpr int FEW_WAVES(int nb) { return nb <= 4 ? 8 : 4; }

// workgroups for many rows that a CU holds, by their registers, and its LDS
constexpr int MANY_LDS = 160 * 1024;
constexpr int MANY_PER_CU(int nb, int rows) { return nb <= 2 && rows == 64 ? 4 : nb <= 4 && rows == 128 ? 2 : 1; }

// blocks of 32 elements that hold a head: those for which there is a kernel
inline int blocks_of(int head_dim) { return head_dim <= 64 ? 2 : head_dim <= 96 ? 3 : head_dim <= 128 ? 4 : head_dim <= 192 ? 6 : 8; }

// Lets a kernel have `bytes` of LDS that its launches ask for, once for each device: the call takes as long as a fifth of a launch
template <auto Kernel>
hipError_t allow_lds(int bytes) {
    static std::atomic<uint64_t> done{0};
    int device = 0;
    if (hipError_t e = hipGetDevice(&device); e != hipSuccess) return e;
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && done.load(std::memory_order_relaxed) & bit) return hipSuccess;
    const hipError_t e = hipFuncSetAttribute((const void*)Kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess && device < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

namespace {

__device__ __attribute__((aligned(16))) const uint32_t zero_chunk[4] = {0, 0, 0, 0};

// n / group for 0 <= n < 2^31, by a product with the reciprocal rounded up to 32 bits: group_mul = ceil(2^(31 + b) / group),
// 2^(b - 1) < group <= 2^b, is too large by less than 1 / 2^31 of itself.
__device__ __forceinline__ int by_group(const PagedArgs& g, int n) {
    return g.group == 1 ? n : (int)(__umulhi((uint32_t)n, g.group_mul) >> g.group_shift);
}

// Weights are 2^(score - m), m = the running maximum less BELOW, and rounded to the element type for their product with the values:
// two parts of a weight would take half as many matrix instructions again, which bound chunks.  What that costs, against 64 bits: 0.0023
// of the result's size in bfloat16 and 0.00029 in binary16, where 32-bit weights and the rounding of the result have 0.0017 and 0.00021.
// binary16 has nothing under 2^-25: with weights of up to 1, 2^8 after a rise that leaves m alone, the values of keys 18 and
// more nats under the largest vanish from the sum while their weights stay in the divisor (of 60,000 such keys beside one that has
// the maximum 98 % of what they add).  So they go up to 2^7, 2^15 after a rise, and what is lost of a key is at most 2^-32 of the
// largest weight.  bfloat16 has the exponents of 32 bits.
template <typename T>
constexpr float BELOW = __is_same(T, _Float16) ? 7.0f : 0.0f;

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

// The cache holds elements of type T, or codes (C = uint8_t)
template <typename C>
constexpr bool CODED = sizeof(C) == 1;

// Eight codes of one row, times its scale, as chunk c of the row
template <typename T, int CH>
__device__ __forceinline__ void put_codes(uint32_t a, uint32_t b, float scale, lds_ptr tile, int row, int c) {
    *(__attribute__((address_space(3))) u32x4*)(tile + (row * CH + (c ^ mix<CH>(row))) * 16) =
        (u32x4){codes_pair<T, false>(a, scale), codes_pair<T, true>(a, scale), codes_pair<T, false>(b, scale), codes_pair<T, true>(b, scale)};
}

// A query row over keys i0 .. i1 - 1 by a wavefront, LPR lanes a row with eight elements each, q times scale * log2 e; where(i): chunks of 16
// bytes from k and v to the row of key i, < 0 where it is masked; scale_at(i): its block among the scales
template <typename T, typename C, int LPR, typename Where, typename ScaleAt>
__device__ __forceinline__ Softmax one_row(const PagedArgs& g, const char* k, const char* v, f32x8 q, bool inside, int i0, int i1, Where where, ScaleAt scale_at) {
    if constexpr (CODED<C>) {
        float x[8];
        for (int e = 0; e < 8; e++) x[e] = q[e];
        SoftmaxCodes<8> s = walk_codes<LPR, 8>((const uint8_t*)k, (const uint8_t*)v, x, inside, i0, i1, [&](long long i) {
            const long long at = where((int)i);
            if (at < 0) return RowCodes{-1, 0.0f, 0.0f};
            const long long b = scale_at((int)i);
            return RowCodes{at * 16, scale_value(g.scales.k[b]), scale_value(g.scales.v[b])};
        });
        gather_codes<LPR>(s);
        Softmax r = {s.m, s.l, {0, 0, 0, 0, 0, 0, 0, 0}};
        for (int e = 0; e < 8; e++) r.acc[e] = s.acc[e];
        return r;
    } else {
        return gather<LPR>(walk_keys<T, LPR>((const T*)k, (const T*)v, q, inside, i0, i1, [&](long long i) { const long long at = where((int)i); return at < 0 ? -1ll : at * 8; }));
    }
}

__device__ __forceinline__ void load_lds16(const void* from, lds_ptr to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}

// Element e of row r (of 32) among the sums that a wavefront leaves for join_kernel; elements 4 i .. 4 i + 3 are together
__device__ __forceinline__ int part_at(int r, int e) { return ((e >> 3) * 64 + r + (e >> 2 & 1) * 32) * 4 + (e & 3); }
constexpr int part_floats(int nb) { return nb * 1024 + 64; }

// ---- tiles shared out ---------------------------------------------------------------------------------------------------
// All tiles of all key heads, UNIT keys of one a unit (32 where few rows meet codes, whose shares are shorter), are cut into equal shares, whatever the lengths of the requests are, one for each
// workgroup (many rows) or wavefront (few); where a cut falls into a tile, its parts are joined afterwards.  Every workgroup finds its
// shares for itself: from the first rows and lengths of all requests (8 bytes each) it counts the units of every slot and adds them up
// in LDS.  With more than MAX_SLOTS slots there are tiles enough to fill the card, and each is a share: that holds for like lengths (1,000
// single tokens of up to 512 keys, 4 heads a group: 251 us), while one long request among so many is read by a wavefront alone (one
// of 131,072 keys: 10.6 ms).
constexpr int UNIT = 64;

struct Segment {  // units u0 .. u1 - 1 of the tile's
    Tile t;
    int u0, u1, units;
    __device__ __forceinline__ bool whole() const { return u0 == 0 && u1 == units; }
};

__host__ __device__ inline size_t shares_bytes(int n_req, int slots) { return (size_t)(n_req + 1) * 8 + (size_t)(slots + 1) * 4 + (size_t)slots * 2; }

template <int U>
__device__ __forceinline__ int units_of(const Tile& t) { return max((t.hi - t.lo + U - 1) / U, 1); }  // results have to be written

struct Shares {
    int *starts, *lens;  // [n_req + 1]
    int* cum;            // [slots + 1] units before each slot
    uint16_t* req;       // [slots]
    // Units x0 .. x1 - 1 are this workgroup's.  The first `rem` shares are `each` + 1 units, the others `each`; the launch has seen to it that
    // there are less than 2^31 in all.
    uint32_t x0, x1, per_head, each, rem;
    int head, slot;
    int group, per, work, active;  // workgroup in the order of the shares, shares of each, this share, shares that this workgroup has
    int columns, column, first;    // see begin; the first share's wavefront of this column

    // For share `sub` of up to PER of the workgroup, by all of it.  false: there is no such share
    template <int ROWS, int PER, int U>
    __device__ __forceinline__ bool begin(const PagedArgs& g, int* lds, int sub) {
        const jx_attend_args& a = g.a;
        const int tid = threadIdx.x, lane = lane_id(), THREADS = (int)blockDim.x;
        x0 = 0;
        x1 = 1;
        columns = 1;
        column = first = 0;
        if (!g.n_work) {
            work = sub;
            const uint32_t i = g.own ? blockIdx.x : blockIdx.x * PER + sub;
            head = (int)(i % a.n_kv_heads);
            slot = g.slots - 1 - (int)(i / a.n_kv_heads);  // long ones first where there is one request
            return slot >= 0;
        }
        starts = lds;
        lens = starts + a.n_req + 1;
        cum = lens + a.n_req + 1;
        req = (uint16_t*)(cum + g.slots + 1);
        for (int i = tid; i <= a.n_req; i += THREADS) {
            starts[i] = a.d_q_start[i];
            lens[i] = i < a.n_req ? a.d_kv_len[i] : 0;
        }
        __syncthreads();
        for (int s = tid; s < g.slots; s += THREADS) {
            int lo = 0, hi = a.n_req;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_slot<ROWS>(starts[mid], mid, g) <= s) lo = mid;
                else hi = mid;
            }
            const Tile t = make_tile<ROWS>(g, lo, s, starts[lo], starts[lo + 1], lens[lo]);
            cum[s + 1] = t.r < 0 ? 0 : units_of<U>(t);
            req[s] = (uint16_t)lo;
        }
        if (tid == 0) cum[0] = 0;
        __syncthreads();
        if (tid < 64) {
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
        const uint32_t units = per_head * a.n_kv_heads;
        // With enough units each of `columns` neighbouring key heads has wavefronts of its own in every workgroup, which then reads the same
        // tokens of all of them: rows of 128 bytes that lie side by side, about the same time.  64 single tokens of up to 8,192 keys, 8 key
        // heads of 128 codes, a call: 83 us with four heads a workgroup, 86 with two, 92 with one; eight, 83, leave more to join (4 tokens of
        // up to 131,072: 137 us with four, 143 with eight, 160 with one).
        columns = PER == 1 || units < (uint32_t)g.n_work ? 1 : g.columns;
        const int of_column = PER / columns, at = sub % of_column;
        column = sub / of_column;
        first = column * of_column;
        const uint32_t all = units / columns, shares = min((uint32_t)g.n_work / columns, all);  // of a column; none is empty
        // shares of a workgroup follow each other; consecutive workgroups stay on one XCD's cache, few are spread over all
        per = PER == 1 ? 1 : (int)((shares + g.groups - 1) / g.groups);
        group = units < (uint32_t)g.n_work ? (int)blockIdx.x : (int)(blockIdx.x % 8) * (g.groups / 8) + (int)(blockIdx.x / 8);
        const int share = group * per + at;
        work = group * PER + sub;
        active = min(per, (int)shares - group * per);
        if (tid < g.columns) g.joins[tid * g.groups + group].pieces = 0;
        if (at >= active) {
            x1 = 0;
            return false;
        }
        each = all / shares;
        rem = all - each * shares;
        x0 = share * each + min((uint32_t)share, rem);
        x1 = x0 + each + ((uint32_t)share < rem);
        head = (int)(x0 / per_head);
        slot = -1;
        return true;
    }

    // Heads are counted in their column
    __device__ __forceinline__ int key_head() const { return head * columns + column; }

    // Rows that belong to no request: zeros and -infinity, by all workgroups, after begin
    template <typename T>
    __device__ __forceinline__ void clear_rows(const PagedArgs& g) const {
        const jx_attend_args& a = g.a;
        const int n = (int)a.n_tokens;
        int b = n, e = n;
        if (a.n_req) {
            b = clamp_rows(__builtin_amdgcn_readfirstlane(g.n_work ? starts[0] : a.d_q_start[0]), a);
            e = clamp_rows(__builtin_amdgcn_readfirstlane(g.n_work ? starts[a.n_req] : a.d_q_start[a.n_req]), a);
        }
        const int chunks = a.n_heads * (a.head_dim / 8), outside = b + max(n - max(b, e), 0);
        for (int i = blockIdx.x; i < outside; i += gridDim.x) {
            const long long t = i < b ? i : i - b + max(b, e);
            for (int c = threadIdx.x; c < chunks; c += blockDim.x) ((uint4*)a.d_out)[t * chunks + c] = make_uint4(0, 0, 0, 0);
            if (a.d_lse)
                for (int h = threadIdx.x; h < a.n_heads; h += blockDim.x) a.d_lse[t * a.n_heads + h] = -INFINITY;
        }
    }

    // The segment that begins with unit x0
    template <int ROWS, int PER, int U>
    __device__ __forceinline__ Segment next(const PagedArgs& g) {
        const jx_attend_args& a = g.a;
        Segment e;
        if (!g.n_work) {
            const int r = last_before(a.n_req, [&](int i) { return first_slot<ROWS>(a.d_q_start[i], i, g) <= slot; });
            e.t = make_tile<ROWS>(g, r, slot, a.d_q_start[r], a.d_q_start[r + 1], a.d_kv_len[r]);
            e.u0 = 0;
            e.u1 = e.units = e.t.r < 0 ? 1 : units_of<U>(e.t);
            if (PER > 1 && g.own) {
                active = min(PER, e.units);
                e.u0 = (int)((long long)e.units * min(work, active) / active);
                e.u1 = (int)((long long)e.units * min(work + 1, active) / active);
            }
            x1 = x0 + e.u1 - e.u0;
            return e;
        }
        if (x0 >= (head + 1) * per_head) {
            head++;
            slot = -1;
        }
        const int at = (int)(x0 - head * per_head);
        if (slot < 0 && at) {
            slot = last_before(g.slots, [&](int i) { return cum[i] <= at; });
        } else {
            do slot++;
            while (cum[slot + 1] <= at);
        }
        slot = __builtin_amdgcn_readfirstlane(slot);
        e.u0 = at - cum[slot];
        e.units = cum[slot + 1] - cum[slot];
        e.u1 = (int)min((uint32_t)e.units, e.u0 + (x1 - x0));
        const int r = req[slot];
        e.t = make_tile<ROWS>(g, r, slot, starts[r], starts[r + 1], lens[r]);
        return e;
    }

    // Where a workgroup leaves its part of a tile that it shares with others: of the tile that it begins and does not end (`begun`) or
    // that it found begun
    __device__ __forceinline__ float* part(const PagedArgs& g, bool begun, int nb) const {
        return g.part + (size_t)(2 * (column * g.groups + group) + begun) * g.part_rows * part_floats(nb);
    }
    // ... and a wavefront its part of a tile that others of its workgroup have begun
    __device__ __forceinline__ float* inner(const PagedArgs& g, int of_work, int nb) const {
        return g.part + (size_t)(2 * g.groups * g.columns + of_work) * part_floats(nb);
    }

    // The first workgroup of those that share a tile, which began with unit x of all, says who they are
    __device__ __forceinline__ void name(const PagedArgs& g, const Tile& t, uint32_t x, int units) const {
        const uint32_t end = x + units - 1, large = rem * (each + 1);  // the tile's last unit, and whose it is
        const int last = (int)(end < large ? end / (each + 1) : rem + (end - large) / each);
        g.joins[column * g.groups + group] = {last / per - group + 1, key_head(), t.first, t.count, t.start, {0, 0, 0}};
    }
};

// A lane's row: whether there is one, its query head, its token's row of q, its position
struct RowAt {
    bool mine;
    int head, token, pos;
};

}  // namespace

}  // namespace jx
