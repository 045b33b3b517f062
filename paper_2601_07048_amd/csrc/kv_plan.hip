// Bookkeeping of a paged key-value cache on the GPU: pages for the new tokens of a step, their positions and slots; pages
// given back.
#include "attend.h"
#include "jx_device.h"

namespace jx {

namespace {

constexpr int PLAN_THREADS = 1024;

// Sum over the workgroup of everything before the calling thread; *total = over all threads.  `part` has a place per wavefront.
__device__ __forceinline__ long long block_before(long long v, long long* part, long long* total) {
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    long long s = v;
    for (int d = 1; d < 64; d *= 2) {
        const long long o = __shfl_up(s, d, 64);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = s;
    __syncthreads();
    long long before = 0, all = 0;
    for (int w = 0; w < PLAN_THREADS / 64; w++) {
        const long long p = part[w];
        if (w < wave) before += p;
        all += p;
    }
    *total = all;
    return before + s - v;
}

// Two sums over the requests decide everything: of the new tokens (where a request's rows begin) and of the pages they
// need, and a token finds its own place from those.  Every workgroup takes the sums for itself (8 bytes a request, from the
// second-level cache after the first) and writes PLAN_THREADS tokens, so nothing passes between workgroups and one launch is
// enough; the first one also writes what there is once per request.  A page's entry in the table is written by the token
// at its first position, which knows the page's place among the free ones; only tokens that go on in a page begun earlier read
// the table, and those entries nobody writes.
// Bound: a chain of dependent reads (lengths, sums, table or free page), not bytes: 6 us for 64 requests of a token, 8 for 1,000
// requests of up to 512.
__global__ __launch_bounds__(PLAN_THREADS) void kv_plan_kernel(KvPlanArgs a) {
    extern __shared__ int32_t places[];  // [n_req + 1] first row, [n_req] pages asked for before this request, -1 = no room
    __shared__ long long part[PLAN_THREADS / 64];
    int32_t* row = places;
    int32_t* before = places + a.n_req + 1;
    const int tid = threadIdx.x, page = 1 << a.page_shift;
    const bool first_block = blockIdx.x == 0;
    const long long n_free = min(max((long long)*a.n_free, 0ll), (long long)a.n_pages);
    long long tokens = 0, pages = 0, taken = 0;
    for (int r0 = 0; r0 < a.n_req; r0 += PLAN_THREADS) {
        const int r = r0 + tid;
        long long len = 0, add = 0, need = 0, end = 0;
        if (r < a.n_req) {
            len = max(a.len[r], 0);
            add = max(a.add[r], 0);
            end = (len + add + page - 1) >> a.page_shift;
            need = end - ((len + page - 1) >> a.page_shift);
        }
        long long all_tokens, all_pages;
        const long long t = tokens + block_before(add, part, &all_tokens);
        const bool fits = r < a.n_req && end <= a.table_pages && t + add <= a.n_tokens;
        if (!fits) need = 0;  // asks for nothing: what is granted has to be one piece at the end of the free pages
        const long long p = pages + block_before(need, part, &all_pages);
        const bool room = fits && (!need || p + need <= n_free);
        if (r < a.n_req) {
            row[r] = (int32_t)min(t, a.n_tokens);
            before[r] = room ? (int32_t)p : -1;  // p + need <= n_free, or unused
            if (room && !need) before[r] = 0;
            if (first_block) {
                a.q_start[r] = row[r];
                a.kv_len[r] = room ? (int32_t)(len + add) : 0;
            }
        }
        long long got;
        block_before(room ? need : 0, part, &got);
        taken += got;
        tokens += all_tokens;
        pages += all_pages;
    }
    if (tid == 0) {
        row[a.n_req] = (int32_t)min(tokens, a.n_tokens);
        if (first_block) {
            a.q_start[a.n_req] = row[a.n_req];
            *a.n_free_out = (int32_t)(n_free - taken);
        }
    }
    __syncthreads();
    const long long t = (long long)blockIdx.x * PLAN_THREADS + tid;
    if (t >= a.n_tokens) return;
    int32_t pos = -1;
    int64_t slot = -1;
    if (t < row[a.n_req]) {
        int lo = 0, hi = a.n_req;  // the last request that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (row[mid] <= t) lo = mid;
            else hi = mid;
        }
        const int32_t p0 = before[lo];
        if (p0 >= 0) {
            const int32_t len = max(a.len[lo], 0);
            pos = len + (int32_t)(t - row[lo]);
            const int at = pos >> a.page_shift, begun = (int)(((long long)len + page - 1) >> a.page_shift);
            int32_t* entry = a.table + (size_t)lo * a.table_pages + at;
            int32_t id;
            if (at < begun) {
                id = *entry;
            } else {
                id = a.free_pages[n_free - 1 - ((long long)p0 + at - begun)];
                if ((pos & (page - 1)) == 0) *entry = id;
            }
            if ((uint32_t)id < (uint32_t)a.n_pages) slot = ((int64_t)id << a.page_shift) + (pos & (page - 1));
        }
    }
    a.pos[t] = pos;
    a.slot[t] = slot;
}

// One workgroup: a wavefront counts the pages that a request gives back, the counts become places, and a second walk writes them, in
// the order of requests and pages whatever the timing.  Bound: for a few requests latency, as for the plan (7 us for a row of 640
// entries), for many what one CU reads, the table twice (26 us for 64 such rows, 1.5 ms for 1,000 of 2,000 entries).
__global__ __launch_bounds__(PLAN_THREADS) void kv_release_kernel(const int32_t* first, const int32_t* end, int n_req, int32_t* table,
                                                                 int table_pages, int32_t* free_pages, int32_t* n_free, int n_pages) {
    extern __shared__ int32_t places[];  // [n_req] pages given back, then their place
    __shared__ long long part[PLAN_THREADS / 64];
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const long long have = min(max((long long)*n_free, 0ll), (long long)n_pages);
    long long total = 0;
    for (int write = 0; write < 2; write++) {
        for (int r = wave; r < n_req; r += PLAN_THREADS / 64) {
            int32_t* row = table + (size_t)r * table_pages;
            const int p1 = min(end[r], table_pages);
            long long n = write ? have + places[r] : 0;
            for (int p0 = max(first[r], 0); p0 < p1; p0 += 64) {
                const int32_t id = p0 + lane < p1 ? row[p0 + lane] : -1;
                const bool held = (uint32_t)id < (uint32_t)n_pages;
                const uint64_t m = ballot(held);
                if (write && held) {
                    const long long at = n + prefix_count(m);
                    if (at < n_pages) free_pages[at] = id;
                    row[p0 + lane] = -1;
                }
                n += __popcll(m);
            }
            if (!write && lane == 0) places[r] = (int32_t)n;
        }
        if (write) break;
        __syncthreads();
        for (int r0 = 0; r0 < n_req; r0 += PLAN_THREADS) {
            const int r = r0 + (int)threadIdx.x;
            long long all;
            const long long at = total + block_before(r < n_req ? places[r] : 0, part, &all);
            if (r < n_req) places[r] = (int32_t)at;
            total += all;
        }
        __syncthreads();
    }
    if (threadIdx.x == 0) *n_free = (int32_t)min(have + total, (long long)n_pages);
}

}  // namespace

hipError_t launch_kv_plan(const KvPlanArgs& a, hipStream_t st) {
    const unsigned blocks = (unsigned)((a.n_tokens + PLAN_THREADS - 1) / PLAN_THREADS);
    kv_plan_kernel<<<blocks ? blocks : 1, PLAN_THREADS, (size_t)(2 * a.n_req + 1) * 4, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_kv_release(const int32_t* first, const int32_t* end, int n_req, int32_t* table, int table_pages, int32_t* free_pages,
                             int32_t* n_free, int n_pages, hipStream_t st) {
    kv_release_kernel<<<1, PLAN_THREADS, (size_t)(n_req + 1) * 4, st>>>(first, end, n_req, table, table_pages, free_pages, n_free, n_pages);
    return hipGetLastError();
}

}  // namespace jx
