// page_map.hip -- block tables, slots and positions of a serving step from its
// requests' lengths (cola_page_map).
//
// Two prefix sums over the requests (new tokens, new pages) and two lookups per
// row and page.  A few KB of work: bound by latency, so one launch does it all.
// Every workgroup forms the sums of all requests itself (at most 4096, from L2)
// and keeps them in LDS; then the workgroups share out the rows and the new
// pages, each finding its request by bisection.  No workgroup waits for another:
// table entries that are read (pages of older tokens) and written (new pages) are
// different ones, and new pages are looked up in the free list again.
#include "serve.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;
constexpr int kMaxReq = COLA_PAGE_MAP_MAX_REQ;

struct Req {
    int old, fresh, have;
    int n;
};
__device__ __forceinline__ Req request(const PageMapArgs& a, int r) {
    const int kv = max(a.kv_len[r], 0);
    Req q;
    q.n = min(max(a.n_new[r], 0), kv);
    q.old = kv - q.n;
    const int64_t up = (int64_t(1) << a.lg_page) - 1;
    q.have = (int)min(((int64_t)q.old + up) >> a.lg_page, a.max_pages);
    q.fresh = (int)min(((int64_t)kv + up) >> a.lg_page, a.max_pages) - q.have;
    return q;
}

// Largest r with at[r] <= x (at ascending, at[0] = 0 <= x, n entries).
__device__ __forceinline__ int find(const int* at, int n, int x) {
    int lo = 0;
    while (n > 1) {
        const int h = n / 2;
        if (at[lo + h] <= x) {
            lo += h;
            n -= h;
        } else {
            n = h;
        }
    }
    return lo;
}

__global__ __launch_bounds__(NTHR) void page_map_kernel(const PageMapArgs a) {
    __shared__ int tok[kMaxReq];                        // first row of each request (saturating at 2^31 - 1)
    __shared__ int pg[kMaxReq];                         // new pages before each request
    __shared__ int old[kMaxReq];                        // tokens that it held before
    __shared__ int64_t wt[NTHR / 64];
    __shared__ int wp[NTHR / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int span = (a.n_req + NTHR - 1) / NTHR;       // requests of one thread, in order
    const int r0 = tid * span, r1 = min(r0 + span, a.n_req);
    int64_t st = 0;
    int sp = 0;
    for (int r = r0; r < r1; ++r) {
        const Req q = request(a, r);
        old[r] = q.old;
        st += q.n;
        sp += q.fresh;
    }
    int64_t it = st;
    int ip = sp;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t x = __shfl_up(it, d);
        const int y = __shfl_up(ip, d);
        if (lane >= d) {
            it += x;
            ip += y;
        }
    }
    if (lane == 63) {
        wt[wave] = it;
        wp[wave] = ip;
    }
    __syncthreads();
    int64_t total = 0, bt = it - st;
    int pages = 0, bp = ip - sp;
#pragma unroll
    for (int w = 0; w < NTHR / 64; ++w) {
        if (w < wave) {
            bt += wt[w];
            bp += wp[w];
        }
        total += wt[w];
        pages += wp[w];
    }
    for (int r = r0; r < r1; ++r) {
        const Req q = request(a, r);
        const int at = (int)min(bt, (int64_t)INT32_MAX);
        tok[r] = at;
        pg[r] = bp;
        if (blockIdx.x == 0) a.start[r] = at;
        bt += q.n;
        bp += q.fresh;
    }
    const int64_t first = a.free_at ? a.free_at[0] : 0;
    if (blockIdx.x == 0 && tid == 0) {
        a.start[a.n_req] = (int)min(total, (int64_t)INT32_MAX);
        a.free_next[0] = (int)min(first + pages, (int64_t)INT32_MAX);
    }
    __syncthreads();

    auto taken = [&](int64_t e) -> int {                // entry first + e of the free list
        const int64_t i = first + e;
        return i >= 0 && i < a.n_free ? a.free_pages[i] : -1;
    };
    const int64_t up = (int64_t(1) << a.lg_page) - 1;
    const int64_t step = (int64_t)gridDim.x * NTHR, me = (int64_t)blockIdx.x * NTHR + tid;
    for (int64_t e = me; e < pages; e += step) {
        const int r = find(pg, a.n_req, (int)e);
        const int64_t have = min(((int64_t)old[r] + up) >> a.lg_page, a.max_pages);
        a.table[r * a.max_pages + have + (e - pg[r])] = taken(e);
    }
    for (int64_t t = me; t < a.T; t += step) {
        int slot = -1, pos = 0;
        if (t < total) {
            const int r = find(tok, a.n_req, (int)t);
            const int64_t i = (int64_t)old[r] + (t - tok[r]);
            const int64_t have = min(((int64_t)old[r] + up) >> a.lg_page, a.max_pages), j = i >> a.lg_page;
            int page = -1;
            if (j < have) page = a.table[r * a.max_pages + j];
            else if (j < a.max_pages) page = taken(pg[r] + (j - have));
            const int64_t s = ((int64_t)page << a.lg_page) + (i & up);
            if (page >= 0 && s <= INT32_MAX) slot = (int)s;
            pos = (int)min(a.pos0 + i, (int64_t)INT32_MAX);
        }
        a.slots[t] = slot;
        a.positions[t] = pos;
    }
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t s) {
    int64_t n = (a.T + NTHR - 1) / NTHR;
    n = n < 1 ? 1 : (n > 1024 ? 1024 : n);
    page_map_kernel<<<dim3((unsigned)n), NTHR, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cola
