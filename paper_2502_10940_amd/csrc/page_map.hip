// page_map.hip -- block tables, slots and positions of a serving step from its
// requests' lengths (cola_page_map).
//
// Two prefix sums over the requests (new tokens, new pages) and two lookups per
// row and page.  A few KB to a few MB of work: bound by latency, so one launch does
// it all.  Every workgroup forms the sums of all requests itself (at most 4096,
// from L2) and keeps them in LDS; then the workgroups share out the rows, four
// neighbours to a thread where they are many, and the new pages, each finding its
// request by bisection.  No workgroup waits for another: table entries that are
// read (pages of older tokens) and written (new pages) are different ones, and new
// pages are looked up in the free list again.  96 requests of one new token 4.5 us
// (an empty launch takes 3.7); 263423 rows of 1024 requests 7.5 us.
#include "serve.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;
constexpr int kMaxReq = COLA_PAGE_MAP_MAX_REQ;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 loose4 __attribute__((aligned(4)));

struct Req {
    int old, fresh, n;
};
__device__ __forceinline__ Req request(const PageMapArgs& a, int len, int fresh) {
    const int kv = max(len, 0);
    Req q;
    q.n = min(max(fresh, 0), kv);
    q.old = kv - q.n;
    const int64_t up = (int64_t(1) << a.lg_page) - 1;
    q.fresh = (int)(min(((int64_t)kv + up) >> a.lg_page, a.max_pages) - min(((int64_t)q.old + up) >> a.lg_page, a.max_pages));
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

// ROWS neighbouring rows to a thread: four where they fill the chip (263423 rows of
// 1024 requests 7.6 us, 10.3 with one), one where latency counts (128 rows 4.5 us, 6.0
// with four).
template <int ROWS>
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
    constexpr int KEEP = 4;                             // requests that a thread keeps (1024 in all)
    Req kept[KEEP];
    if (span <= KEEP) {
        int len[KEEP], fresh[KEEP];
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            len[i] = r0 + i < r1 ? a.kv_len[r0 + i] : 0;
            fresh[i] = r0 + i < r1 ? a.n_new[r0 + i] : 0;
        }
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            kept[i] = request(a, len[i], fresh[i]);
            st += kept[i].n;
            sp += kept[i].fresh;
        }
    } else {
        for (int r = r0; r < r1; ++r) {
            const Req q = request(a, a.kv_len[r], a.n_new[r]);
            st += q.n;
            sp += q.fresh;
        }
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
    auto keep = [&](int r, const Req& q) {
        const int at = (int)min(bt, (int64_t)INT32_MAX);
        old[r] = q.old;
        tok[r] = at;
        pg[r] = bp;
        if (blockIdx.x == 0) a.start[r] = at;
        bt += q.n;
        bp += q.fresh;
    };
    if (span <= KEEP) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            if (r0 + i < r1) keep(r0 + i, kept[i]);
    } else {
        for (int r = r0; r < r1; ++r) keep(r, request(a, a.kv_len[r], a.n_new[r]));
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
    for (int64_t t0 = ROWS * me; t0 < a.T; t0 += ROWS * step) {
        int slot[ROWS], pos[ROWS];
        int r = t0 < total ? find(tok, a.n_req, (int)t0) : 0;
        int64_t page[ROWS], i[ROWS];
#pragma unroll
        for (int x = 0; x < ROWS; ++x) {
            const int64_t t = t0 + x;
            page[x] = -1;
            i[x] = 0;
            slot[x] = -1;
            pos[x] = 0;
            if (t >= total || t >= a.T) continue;
            while (r + 1 < a.n_req && tok[r + 1] <= t) ++r;
            i[x] = (int64_t)old[r] + (t - tok[r]);
            const int64_t have = min(((int64_t)old[r] + up) >> a.lg_page, a.max_pages), j = i[x] >> a.lg_page;
            if (j < have) page[x] = a.table[r * a.max_pages + j];
            else if (j < a.max_pages) page[x] = taken(pg[r] + (j - have));
            pos[x] = (int)min(a.pos0 + i[x], (int64_t)INT32_MAX);
        }
#pragma unroll
        for (int x = 0; x < ROWS; ++x) {
            const int64_t s = (page[x] << a.lg_page) + (i[x] & up);
            if (page[x] >= 0 && s <= INT32_MAX) slot[x] = (int)s;
        }
        if (ROWS == 4 && t0 + ROWS <= a.T) {
            *reinterpret_cast<loose4*>(a.slots + t0) = i32x4{slot[0], slot[1 % ROWS], slot[2 % ROWS], slot[3 % ROWS]};
            *reinterpret_cast<loose4*>(a.positions + t0) = i32x4{pos[0], pos[1 % ROWS], pos[2 % ROWS], pos[3 % ROWS]};
        } else {
#pragma unroll
            for (int x = 0; x < ROWS; ++x)
                if (t0 + x < a.T) {
                    a.slots[t0 + x] = slot[x];
                    a.positions[t0 + x] = pos[x];
                }
        }
    }
}

}  // namespace

hipError_t launch_page_map(const PageMapArgs& a, hipStream_t s) {
    const int rows = a.T > (1 << 16) ? 4 : 1;
    int64_t n = (a.T + rows * NTHR - 1) / (rows * NTHR);
    n = n < 1 ? 1 : (n > 1024 ? 1024 : n);
    if (rows == 4) page_map_kernel<4><<<dim3((unsigned)n), NTHR, 0, s>>>(a);
    else page_map_kernel<1><<<dim3((unsigned)n), NTHR, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cola
