// logits.hip -- penalties for repeated tokens, biases and grammar masks on the logits
// of a step (cola_logits_adjust).
//
// HBM bound: each logit is read once and written once, and few are changed.  A workgroup
// takes a chunk of the vocabulary for a run of rows: it counts the chunk's tokens in
// the request's history in LDS (whole numbers, so that the order of the additions does
// not matter), keeps the last bias of each token beside the counts, and sends the
// rows through, 16 bytes a load.  The rows of one request share the counts; each adds
// its own drafted tokens before its pass and takes them back after it.  A row's logits
// are on their way to registers while the history is read.
#include "rows.hpp"
#include "serve.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;
constexpr uint32_t kPrompt = 0x80000000u;               // in a count: the token is in the prompt

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 loose4 __attribute__((aligned(4)));

struct LogitsGrid {
    int rows;                                           // rows of a workgroup
};

// Largest r with start[r] <= t, or -1 (n entries that do not fall), by all lanes of a wave.
__device__ __forceinline__ int owner(const int32_t* start, int n, int64_t t) {
    const int lane = threadIdx.x & 63;
    if (start[0] > t) return -1;
    int lo = 0, len = n;
    while (len > 1) {
        const int step = (len + 63) / 64, at = lane * step;
        const uint64_t b = __ballot(at < len && start[lo + at] <= t);
        const int k = max(__popcll(b) - 1, 0) * step;
        lo += k;
        len = min(step, len - k);
    }
    return lo;
}

template <bool BF16, int NVEC>
__global__ __launch_bounds__(NTHR) void logits_kernel(const LogitsArgs a, const LogitsGrid g) {
    constexpr int PV = BF16 ? 8 : 4, C = NTHR * PV * NVEC;
    typedef Vec<BF16, PV> V;
    typedef typename V::E E;
    typedef typename V::G G;
    extern __shared__ uint32_t count[];                 // [C], then (with biases) the last entry of each token
    int32_t* last = reinterpret_cast<int32_t*>(count) + C;
    const int tid = threadIdx.x;
    const int64_t c0 = (int64_t)blockIdx.x * C;
    const int width = (int)min(a.V - c0, (int64_t)C);
    const int64_t t0 = (int64_t)blockIdx.y * g.rows, t1 = min(t0 + g.rows, a.T);
    const bool repeats = a.repetition || a.presence || a.frequency;
    const bool biases = a.bias_start != nullptr;
    const bool drafted = repeats && a.draft;
    int r = a.start ? owner(a.start, a.n_req, t0) : (int)t0;
    int held = -1;                                      // the request whose counts are in LDS
    uint32_t mine = 0;                                  // this thread's node in the counts: its place + 1

    for (int64_t t = t0; t < t1; ++t) {
        if (a.start) {
            if (r < 0 && a.start[0] <= t) r = owner(a.start, a.n_req, t);
            while (r >= 0 && r < a.n_req && a.start[r + 1] <= t) ++r;
            if (r < 0) continue;
        } else {
            r = (int)t;
        }
        if (r >= a.n_req) break;

        // this row's logits on their way
        const E* from = (const E*)a.logits + t * a.ldl + c0;
        V x[NVEC];
#pragma unroll
        for (int k = 0; k < NVEC; ++k) {
            const int v = (k * NTHR + tid) * PV;
            if (v + PV <= width) x[k].load(from + v);
        }
        float rep = 1.0f, pres = 0.0f, freq = 0.0f;
        if (a.repetition) rep = a.repetition[r];
        if (a.presence) pres = a.presence[r];
        if (a.frequency) freq = a.frequency[r];

        const bool fresh = r != held;
        if (fresh && (repeats || biases)) {
            if (held >= 0) __syncthreads();             // the row before has read its counts
            for (int i = tid; i < C; i += NTHR) {
                count[i] = 0;
                if (biases) last[i] = -1;
            }
            mine = 0;
            __syncthreads();
            if (repeats && a.hist_len) {
                const int64_t end = min(max((int64_t)a.hist_len[r], (int64_t)0), a.max_hist);
                const int64_t past = a.prompt_len ? min(max((int64_t)a.prompt_len[r], (int64_t)0), end) : 0;
                const int32_t* h = a.history + r * a.max_hist;
                auto note = [&](int32_t token, int64_t j) __attribute__((always_inline)) {
                    const int64_t at = (int64_t)token - c0;
                    if (at >= 0 && at < width) {
                        if (j < past) atomicOr(&count[at], kPrompt);
                        else atomicAdd(&count[at], 1u);
                    }
                };
                int64_t j = 4 * tid;
                for (; j + 4 <= end; j += 4 * NTHR) {
                    const i32x4 y = *reinterpret_cast<const loose4*>(h + j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) note(y[i], j + i);
                }
                for (; j < end; ++j) note(h[j], j);
            }
            if (biases) {
                const int64_t lo = min(max((int64_t)a.bias_start[r], (int64_t)0), a.n_bias);
                const int64_t hi = min(max((int64_t)a.bias_start[r + 1], lo), a.n_bias);
                for (int64_t j = lo + tid; j < hi; j += NTHR) {
                    const int64_t at = (int64_t)a.bias_token[j] - c0;
                    if (at >= 0 && at < width) atomicMax(&last[at], (int32_t)j);
                }
            }
            held = r;
            if (!drafted) __syncthreads();
        }
        if (drafted) {
            // the drafted tokens that this row sees, in place of those of the row before
            if (!fresh) __syncthreads();
            if (mine) atomicSub(&count[mine - 1], 1u);
            mine = 0;
            const int64_t lo = a.start ? max((int64_t)a.start[r], (int64_t)0) : t, hi = a.start ? min((int64_t)a.start[r + 1], a.T) : t + 1;
            if (tid < 64 * a.words && lo + tid < hi && (a.mask[t * a.words + (tid >> 6)] >> (tid & 63) & 1)) {
                const int64_t at = (int64_t)a.draft[lo + tid] - c0;
                if (at >= 0 && at < width) {
                    mine = (uint32_t)at + 1;
                    atomicAdd(&count[at], 1u);
                }
            }
            __syncthreads();
        }
        const uint32_t* ok = nullptr;
        if (a.allowed) {
            const int64_t s = a.allowed_row ? (int64_t)a.allowed_row[t] : t;
            if (s >= 0 && s < a.n_allowed) ok = a.allowed + s * a.lda + (c0 >> 5);
        }
        auto adjust = [&](float y, int v) __attribute__((always_inline)) {
            if (repeats) {
                const uint32_t n = count[v];
                if (n != 0) {
                    y = y > 0.0f ? y / rep : y * rep;
                    const uint32_t c = n & ~kPrompt;
                    if (c != 0) y = y - freq * (float)c - pres;
                }
            }
            if (biases && last[v] >= 0) y += a.bias[last[v]];
            return y;
        };
        G to = (G)a.out + t * a.ldo + c0;
#pragma unroll
        for (int k = 0; k < NVEC; ++k) {
            const int v = (k * NTHR + tid) * PV;
            if (v + PV <= width) {
                uint32_t any = 0;
#pragma unroll
                for (int e = 0; e < PV; ++e) {
                    if (repeats) any |= count[v + e];
                    if (biases) any |= (uint32_t)(last[v + e] + 1);
                }
                const uint32_t bits = ok ? ok[v >> 5] >> (v & 31) : ~0u;
                if (any != 0 || (~bits & ((1u << PV) - 1)) != 0) {
                    float y[PV];
                    x[k].get(y);
#pragma unroll
                    for (int e = 0; e < PV; ++e) {
                        if (any != 0) y[e] = adjust(y[e], v + e);
                        if (!(bits >> e & 1)) y[e] = -INFINITY;
                    }
                    x[k].put(y);
                }
                x[k].template store<false>(to + v);
            } else {
                for (int e = v; e < width; ++e) {
                    Vec<BF16, 1> z;
                    z.load(from + e);
                    float y[1];
                    z.get(y);
                    y[0] = adjust(y[0], e);
                    if (ok && !(ok[e >> 5] >> (e & 31) & 1)) y[0] = -INFINITY;
                    z.put(y);
                    z.template store<false>(to + e);
                }
            }
        }
    }
}

template <bool BF16, int NVEC>
hipError_t go(const LogitsArgs& a, const LogitsGrid& g, hipStream_t s) {
    constexpr int C = NTHR * (BF16 ? 8 : 4) * NVEC;
    const bool repeats = a.repetition || a.presence || a.frequency;
    const size_t lds = a.bias_start ? 8 * C : (repeats ? 4 * C : 0);
    const int64_t gy = (a.T + g.rows - 1) / g.rows;
    logits_kernel<BF16, NVEC><<<dim3((unsigned)((a.V + C - 1) / C), (unsigned)gy), NTHR, lds, s>>>(a, g);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_logits(bool bf16, const LogitsArgs& a, hipStream_t s) {
    LogitsGrid g{};
    g.rows = 1;
    while ((a.T + g.rows - 1) / g.rows > 65535) g.rows *= 2;
    return bf16 ? go<true, 4>(a, g, s) : go<false, 8>(a, g, s);
}

}  // namespace cola
