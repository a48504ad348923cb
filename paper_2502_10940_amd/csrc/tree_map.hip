// tree_map.hip -- which drafted tokens each drafted token sees, and its position, from
// the tree's parents (cola_tree_map).
//
// mask_i = {i} + mask_parent(i), position = the request's older tokens + the number of
// i's ancestors.  A few KB: bound by latency, so one launch and few dependent steps: a
// workgroup to a request, a thread to a node, and ancestors taken in doubling steps
// (after k of them a node has its 2^k nearest, and knows the next one), as many as
// the tree's depth asks for.  Calls one after the other: 4 requests of up to 16 nodes 4.3
// us (an empty launch takes 3.7), 1000 of up to 201 (4 MB) 5.8.
#include "serve.hpp"

namespace cola {
namespace {

// W words of 64 nodes; trees of one word stay in one wave's registers.
template <int W>
__global__ __launch_bounds__(W == 1 ? 64 : 256) void tree_map_kernel(const TreeMapArgs a) {
    constexpr int NTHR = W == 1 ? 64 : 256;
    const int i = threadIdx.x, r = blockIdx.x;
    // rows of no request: those before the first, and behind the last
    const int64_t first = a.start ? min(max((int64_t)a.start[0], (int64_t)0), a.T) : 0;
    const int64_t last = a.start ? min(max((int64_t)a.start[a.n_req], (int64_t)0), a.T) : min((int64_t)a.n_req, a.T);
    auto clear = [&](int64_t t) __attribute__((always_inline)) {
#pragma unroll
        for (int w = 0; w < W; ++w) a.mask[t * W + w] = 0;
        a.positions[t] = 0;
    };
    for (int64_t t = (int64_t)r * NTHR + i; t < first; t += (int64_t)gridDim.x * NTHR) clear(t);
    for (int64_t t = last + (int64_t)r * NTHR + i; t < a.T; t += (int64_t)gridDim.x * NTHR) clear(t);
    if (r >= a.n_req) return;

    const int64_t lo = a.start ? max((int64_t)a.start[r], (int64_t)0) : r, hi = a.start ? (int64_t)a.start[r + 1] : r + 1;
    const int64_t n = max(hi - lo, (int64_t)0), here = max(min(hi, a.T) - lo, (int64_t)0);
    const int nodes = (int)min(here, (int64_t)a.max_new);
    for (int64_t j = a.max_new + i; j < here; j += NTHR) clear(lo + j);
    const int64_t old = (int64_t)a.kv_len[r] - n;
    int p = i < nodes ? a.parent[lo + i] : -1;
    if (p < 0 || p >= i) p = -1;
    uint64_t m[W];
#pragma unroll
    for (int w = 0; w < W; ++w) m[w] = i >> 6 == w ? uint64_t(1) << (i & 63) : 0;
    if constexpr (W == 1) {
        while (__ballot(p >= 0) != 0) {
            const int from = max(p, 0);
            const uint32_t x = __shfl((uint32_t)m[0], from), y = __shfl((uint32_t)(m[0] >> 32), from);
            const int up = __shfl(p, from);
            if (p >= 0) {
                m[0] |= (uint64_t)y << 32 | x;
                p = up;
            }
        }
    } else {
        __shared__ uint64_t seen[W][NTHR];
        __shared__ int next[NTHR];
        while (__syncthreads_or(p >= 0)) {
#pragma unroll
            for (int w = 0; w < W; ++w) seen[w][i] = m[w];
            next[i] = p;
            __syncthreads();
            if (p >= 0) {
#pragma unroll
                for (int w = 0; w < W; ++w) m[w] |= seen[w][p];
                p = next[p];
            }
        }
    }
    if (i >= nodes) return;
    int depth = -1;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        a.mask[(lo + i) * W + w] = m[w];
        depth += __popcll(m[w]);
    }
    a.positions[lo + i] = (int32_t)min(max(a.pos0 + old + depth, (int64_t)0), (int64_t)INT32_MAX);
}

}  // namespace

hipError_t launch_tree_map(const TreeMapArgs& a, hipStream_t s) {
    const unsigned grid = a.n_req > 0 ? a.n_req : 1;
    switch (a.words) {
        case 1: tree_map_kernel<1><<<grid, 64, 0, s>>>(a); break;
        case 2: tree_map_kernel<2><<<grid, 256, 0, s>>>(a); break;
        case 3: tree_map_kernel<3><<<grid, 256, 0, s>>>(a); break;
        case 4: tree_map_kernel<4><<<grid, 256, 0, s>>>(a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace cola
