// logits.hip -- penalties for repeated tokens, biases and grammar masks on the logits
// of a step (cola_logits_adjust).
//
// HBM bound: each logit is read once and written once.  A workgroup takes a chunk of the
// vocabulary for a run of rows.  It counts the chunk's tokens in the request's history
// in LDS (whole numbers, so that the order of the additions does not matter) and turns
// the counts into what each logit gets: y = x f + shift, f = 1, or for tokens that were
// seen 1 / repetition or repetition by x's sign, and shift = bias - (frequency c +
// presence), -0 where there is nothing to add.  Then the rows go through, 16 bytes a
// load, a row ahead of the arithmetic; bits say which vectors anything happens to (a
// wave that read every shift would meet eight lanes on each bank of LDS).  The rows of one
// request share all that but for the drafted tokens: for each of those in the chunk a
// lane counts the nodes of the row's path that drafted it (the bits that two masks
// share) and writes the token's shift anew.  A wave has a part of the chunk to itself,
// so that no wave waits for another between the rows.
//
// 980 rows of 128003 bf16 logits of 40 requests, histories of up to 8000 tokens, 200 biases
// each and masks for the rows (533 MB): 141 us, 3.8 TB/s (three sets of tensors in turn);
// without rules 115 us, 4.4 TB/s: rows of 128003 begin off their lines.
// What is between is the counting (66 workgroups of a request read its history), the
// masks' bits and the vectors that hold tokens of the history, nearly all here (21 vector
// instructions a logit, which take 52 % of the launch).  One row of 32000 fp32 logits: 5.4
// us, a launch and five loads one after the other.  256 rows of requests of their own (138
// MB): 77 us, 1.8 TB/s: each of a row's 32 workgroups reads the request's history and builds
// its chunk's counts for one row; fp32 (269 MB) 91.
#include "rows.hpp"
#include "serve.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;
constexpr uint32_t kPrompt = 0x80000000u;               // in a count: the token is in the prompt
constexpr int kMaxRows = 16;                            // rows of a workgroup

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 loose4 __attribute__((aligned(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t loose_u16 __attribute__((aligned(1)));

// What a wave's loads go to where it has no logits.
__device__ const uint32_t kNowhere[4] = {0, 0, 0, 0};
__device__ const float kOne = 1.0f;
// A load from global memory, said so: a pointer picked among several loses its space.
template <class X>
__device__ __forceinline__ X global(const void* p) {
    return *(const __attribute__((address_space(1))) X*)p;
}

// An entry that is the same for a wave, of arrays that this kernel only reads: by the
// scalar unit, so that no wait for it is one for the rows in flight.
template <class X>
__device__ __forceinline__ X entry(const X* p, int64_t i) {
    return ((const __attribute__((address_space(4))) X*)p)[i];
}

// Largest r with start[r] <= t, or -1 (n entries that do not fall), by all lanes of a wave.
__device__ __forceinline__ int owner(const int32_t* start, int n, int64_t t) {
    const int lane = threadIdx.x & 63;
    if (entry(start, 0) > t) return -1;
    int lo = 0, len = n;
    while (len > 1) {
        const int step = (len + 63) / 64, at = lane * step;
        const uint64_t b = __ballot(at < len && start[lo + at] <= t);
        const int k = max(__popcll(b) - 1, 0) * step;
        lo += k;
        len = min(step, len - k);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// LDS: a count, then a shift, for each token of the chunk; a bit for each that was seen,
// and for each that changes; with biases the last entry of each token; with drafted
// tokens their nodes.
constexpr size_t lds_bytes(int C, bool biases, int words) {
    return 4 * C + 2 * (C / 8 + 16) + (biases ? 4 * C : 0) + 64 * words * 8 * (words + 2);
}
// Eight bits or less from `place` on.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int place) {
    const uint32_t* w = words + (place >> 5);
    return __builtin_amdgcn_alignbit(w[1], w[0], place & 31);
}
// All ones where bit e of x is set.
__device__ __forceinline__ uint32_t spread(uint32_t x, int e) { return (uint32_t)((int32_t)(x << (31 - e)) >> 31); }
__device__ __forceinline__ uint32_t pick(uint32_t m, uint32_t x, uint32_t y) { return (x & m) | (y & ~m); }

// A token that the request drafted: its place in the chunk (-1: another entry has it), the
// shift that it has without the row's path, and whether the history and the answer
// have it.
struct Draft {
    int32_t place;
    float shift;
    uint32_t seen, answer;
};

// PV NVEC elements of a row to a thread; PAST: results past the caches, which leaves them to
// the inputs (256 rows of 128003 bf16 logits, one to a request, 138 MB: 78 us against 85; 980
// rows of 32000: 56 against 60; 980 of 128000: 132 either way).  Where rows begin off their
// lines it costs more than it gives at larger sizes (980 of 128003: 142 against 138, fp32
// 235 against 225).
template <bool BF16, int NVEC, bool PAST>
__global__ __launch_bounds__(NTHR) void logits_kernel(const LogitsArgs a, const int rows, const int chunks, const int64_t base) {
    constexpr int PV = BF16 ? 8 : 4, CW = 64 * PV * NVEC, C = CW * NTHR / 64;
    constexpr int AHEAD = 4;                            // loads of the history that a thread has on their way, 4 tokens each
    typedef Vec<BF16, PV> V;
    typedef typename V::E E;
    typedef typename V::G G;
    extern __shared__ __attribute__((aligned(16))) uint32_t count[];
    float* shift = reinterpret_cast<float*>(count);
    uint32_t* seen = count + C;                         // [C / 32], and a word past the end
    uint32_t* changed = seen + C / 32 + 4;              // the same
    uint64_t* nodes = reinterpret_cast<uint64_t*>(changed + C / 32 + 4);
    Draft* drafts = reinterpret_cast<Draft*>(nodes + 64 * a.words * a.words);
    uint32_t* last = reinterpret_cast<uint32_t*>(drafts + 64 * a.words);
    __shared__ int n_drafts;
    __shared__ float value[NTHR];                       // of the first entries of the request's list
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t group = (base + blockIdx.x) / chunks;
    const int64_t c0 = (base + blockIdx.x - group * chunks) * C;
    const int width = (int)min(a.V - c0, (int64_t)C);
    // this wave's part of the chunk
    const int v0 = CW * wave, wide = min(max(width - v0, 0), CW);
    const int64_t t0 = group * rows;
    const int n_rows = (int)min((int64_t)rows, a.T - t0);
    const bool repeats = a.repetition || a.presence || a.frequency;
    const bool biases = a.bias_start != nullptr, changes = repeats || biases, drafted = repeats && a.draft;

    // A row: `head` logits up to where out is aligned, vectors, and what is left, with a
    // lane for each that no vector has.  All loads are made, by lanes that have nothing to
    // load from where another does: a branch would have the compiler wait for them.
    struct Row {
        V x[NVEC];
        Vec<BF16, 1> edge;
        uint32_t ok[NVEC], edge_ok;                     // allowed tokens: two bytes of the bits
        int head, full, state;
        __device__ __forceinline__ int at(int k, int lane) const { return head + (64 * k + lane) * PV; }
        __device__ __forceinline__ int edge_at(int lane) const { return lane < head ? lane : full + lane - head; }
    };
    const bool vectors = wide >= 2 * PV;
    // lane i has row i's place among the masks
    int64_t state = -1;
    if (a.allowed && lane < n_rows) state = a.allowed_row ? (int64_t)a.allowed_row[t0 + lane] : t0 + lane;
    if (state >= a.n_allowed) state = -1;
    // two bytes of the bits from here on end the masks' row
    const int last_bits = (int)(4 * a.lda - ((c0 + v0) >> 3)) - 2;
    auto bits_byte = [&](int v) __attribute__((always_inline)) { return min(v >> 3, last_bits); };
    auto load = [&](Row& w, int i) __attribute__((always_inline)) {
        const E* from = (const E*)a.logits + (t0 + i) * a.ldl + c0 + v0;
        const uint32_t off = (uint32_t)(uintptr_t)((E*)a.out + (t0 + i) * a.ldo + c0 + v0) / sizeof(E) % PV;
        w.head = vectors ? __builtin_amdgcn_readfirstlane((int)(off ? PV - off : 0)) : wide;
        w.full = w.head + (wide - w.head) / PV * PV;
        w.state = __builtin_amdgcn_readlane((int)state, i);
        const uint8_t* bits = w.state >= 0 && wide > 0 ? reinterpret_cast<const uint8_t*>(a.allowed + w.state * a.lda) + ((c0 + v0) >> 3)
                                                       : nullptr;
#pragma unroll
        for (int k = 0; k < NVEC; ++k) {
            const int v = min(w.at(k, lane), w.full - PV);
            w.x[k].r = global<typename V::Loose>(vectors ? (const void*)(from + v) : kNowhere);
            w.ok[k] = global<loose_u16>(vectors && bits ? (const void*)(bits + bits_byte(v)) : kNowhere);
        }
        const int v = min(w.edge_at(min(lane, max(w.head + wide - w.full, 1) - 1)), wide - 1);
        w.edge.r = global<typename Vec<BF16, 1>::Loose>(wide > 0 ? (const void*)(from + v) : kNowhere);
        w.edge_ok = global<uint8_t>(bits ? (const void*)(bits + (v >> 3)) : kNowhere);
    };
    bool built = false, own_drafts = false;             // shifts of a request are in LDS; drafted tokens in this wave's part
    float rep = 1.0f, inv = 1.0f, pres = 0.0f, freq = 0.0f;
    // One row from its registers, the next one on its way.
    auto step = [&](Row& now, Row& next, int i) __attribute__((always_inline)) {
        const int64_t t = t0 + i;
        load(next, min(i + 1, n_rows - 1));
        if (own_drafts) {
            const uint64_t* mask = a.mask + t * a.words;
            for (int j = lane; j < n_drafts; j += 64) {
                const Draft d = drafts[j];
                if (d.place < 0 || d.place / CW != wave) continue;
                int c = 0;
                for (int w = 0; w < a.words; ++w) c += __popcll(nodes[j * a.words + w] & entry(mask, w));
                shift[d.place] = c != 0 ? d.shift - fmaf(freq, (float)c, d.answer ? 0.0f : pres) : d.shift;
                const uint32_t bit = 1u << (d.place & 31);
                if (c != 0 || d.seen) atomicOr(&seen[d.place >> 5], bit);
                else atomicAnd(&seen[d.place >> 5], ~bit);
            }
            // the wave's own lanes read what it wrote
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
        auto adjust = [&](float y, float add, bool was) __attribute__((always_inline)) {
            return fmaf(y, was ? (y > 0.0f ? inv : rep) : 1.0f, add);
        };
        G to = (G)a.out + t * a.ldo + c0 + v0;
#pragma unroll
        for (int k = 0; k < NVEC; ++k) {
            const int v = now.at(k, lane);
            if (v >= now.full) continue;
            if (changes && (bits_at(changed, v0 + v) & ((1u << PV) - 1)) != 0) {
                const uint32_t was = bits_at(seen, v0 + v);
                float y[PV];
                now.x[k].get(y);
#pragma unroll
                for (int e = 0; e < PV; ++e) y[e] = adjust(y[e], shift[v0 + v + e], was >> e & 1);
                now.x[k].put(y);
            }
            if (now.state >= 0) {
                const uint32_t ok = now.ok[k] >> (v - 8 * bits_byte(v));
#pragma unroll
                for (int j = 0; j < V::N; ++j) {
                    if constexpr (BF16)
                        now.x[k].r[j] = pick(pick(0xffffu, spread(ok, 2 * j), spread(ok, 2 * j + 1)), now.x[k].r[j], 0xff80ff80u);
                    else
                        now.x[k].r[j] = pick(spread(ok, j), now.x[k].r[j], 0xff800000u);
                }
            }
            now.x[k].template store<PAST>(to + v);
        }
        if (lane < now.head + wide - now.full) {
            const int v = now.edge_at(lane);
            float y[1];
            now.edge.get(y);
            if (changes) y[0] = adjust(y[0], shift[v0 + v], seen[(v0 + v) >> 5] >> ((v0 + v) & 31) & 1);
            if (now.state >= 0 && !(now.edge_ok >> (v & 7) & 1)) y[0] = -INFINITY;
            now.edge.put(y);
            now.edge.template store<false>(to + v);
        }
    };

    Row x, y;
    load(x, 0);
    int r = a.start ? owner(a.start, a.n_req, t0) : (int)t0;
    for (int i = 0; i < n_rows;) {
        // the request of row i and the end of its rows
        const int64_t t = t0 + i;
        int stop = i + 1;
        if (a.start) {
            if (r < 0) r = owner(a.start, a.n_req, t);
            while (r >= 0 && r < a.n_req && entry(a.start, r + 1) <= t) ++r;
            if (r < 0) {
                load(x, min(i + 1, n_rows - 1));
                ++i;
                continue;
            }
            if (r < a.n_req) stop = (int)min((int64_t)entry(a.start, r + 1) - t0, (int64_t)n_rows);
        } else {
            r = (int)t;
        }
        if (r >= a.n_req) break;

        if (changes) {
            // The arguments that only this part needs, read here: held through the rows they
            // take scalar registers, which are spilled to and fetched from vector ones (256 rows
            // of requests of their own 86 us against 78, one row 6.2 against 5.4).
            const __attribute__((address_space(4))) LogitsArgs* here = (const __attribute__((address_space(4))) LogitsArgs*)__builtin_amdgcn_kernarg_segment_ptr();
            asm volatile("" : "+s"(here));
            const __attribute__((address_space(4))) LogitsArgs& z = *here;
            const bool counted = repeats && z.hist_len;
            const int32_t* h = z.history + (int64_t)r * z.max_hist;
            // The request's numbers, all on their way at once: those that are not there come
            // from a place that is.
            const int32_t* zero = reinterpret_cast<const int32_t*>(kNowhere);
            const float* one = &kOne;
            const int hist_len = entry(counted ? z.hist_len + r : zero, 0), prompt_len = entry(z.prompt_len ? z.prompt_len + r : zero, 0);
            const int bias_lo = entry(biases ? z.bias_start + r : zero, 0), bias_hi = entry(biases ? z.bias_start + r + 1 : zero, 0);
            const int first = entry(z.start ? z.start + r : zero, 0), past_last = entry(z.start ? z.start + r + 1 : zero, 0);
            rep = entry(z.repetition ? z.repetition + r : one, 0);
            pres = entry(z.presence ? z.presence + r : reinterpret_cast<const float*>(zero), 0);
            freq = entry(z.frequency ? z.frequency + r : reinterpret_cast<const float*>(zero), 0);
            const int end = min(max(hist_len, 0), (int)z.max_hist), past = min(max(prompt_len, 0), end);
            const int lo = min(max(bias_lo, 0), (int)z.n_bias), hi = min(max(bias_hi, lo), (int)z.n_bias);
            const int64_t n0 = z.start ? max(first, 0) : t, n1 = z.start ? min((int64_t)past_last, z.T) : t + 1;
            // A thread's first entries of the lists, on their way while LDS is cleared.  The
            // history goes four tokens a load; the last load ends with it.
            auto read = [&](i32x4 (&y)[AHEAD], int j0) __attribute__((always_inline)) {
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) y[k] = global<loose4>(h + min(j0 + 4 * k * NTHR, end - 4));
            };
            i32x4 y[AHEAD];
            if (end >= 4) read(y, 4 * tid);
            int token = -1, node = -1;
            float b = 0.0f;
            if (lo + tid < hi) {
                token = z.bias_token[lo + tid];
                b = z.bias[lo + tid];
            }
            if (drafted && tid < 64 * a.words && n0 + tid < n1) node = z.draft[n0 + tid];
            // a token's place in the chunk, `width` or more: it has none
            auto place_of = [&](int token) __attribute__((always_inline)) { return (uint32_t)token - (uint32_t)c0; };
            if (built) __syncthreads();                 // the request before has read its shifts
            for (int j = 4 * tid; j < C; j += 4 * NTHR) {
                *reinterpret_cast<u32x4*>(count + j) = u32x4{0, 0, 0, 0};
                if (biases) *reinterpret_cast<u32x4*>(last + j) = u32x4{0, 0, 0, 0};
            }
            if (tid == 0) n_drafts = 0;
            __syncthreads();
            auto note = [&](int token, int j) __attribute__((always_inline)) {
                const uint32_t at = place_of(token);
                if (at < (uint32_t)width) {
                    if (j < past) atomicOr(&count[at], kPrompt);
                    else atomicAdd(&count[at], 1u);
                }
            };
            if (end >= 4) {
                for (int j0 = 4 * tid;;) {
#pragma unroll
                    for (int k = 0; k < AHEAD; ++k) {
                        const int j = j0 + 4 * k * NTHR, from = min(j, end - 4);
                        if (j >= end) continue;
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (from + e >= j) note(y[k][e], from + e);
                    }
                    j0 += 4 * AHEAD * NTHR;
                    if (j0 >= end) break;
                    read(y, j0);
                }
            } else if (tid < end) {
                note(h[tid], tid);
            }
            // the last entry of each token, by its place in the list + 1
            for (int j = lo + tid; j < hi; j += NTHR) {
                const uint32_t at = place_of(token);
                if (at < (uint32_t)width) atomicMax(&last[at], (uint32_t)j + 1);
                if (j + NTHR < hi) token = z.bias_token[j + NTHR];
            }
            value[tid] = b;
            int mine = -1, place = 0;
            if (drafted && place_of(node) < (uint32_t)width) {
                place = (int)place_of(node);
                mine = atomicAdd(&n_drafts, 1);
                drafts[mine] = Draft{place, 0.0f, (uint32_t)tid, 0};
            }
            __syncthreads();
            if (drafted) {
                // The nodes that drafted this thread's token; the first of them keeps it.
                const int n = n_drafts;
                bool keep = mine >= 0;
                uint32_t held_count = 0;
                if (mine >= 0) {
                    held_count = count[place];
                    for (int w = 0; w < a.words; ++w) {
                        uint64_t m = 0;
                        for (int j = 0; j < n; ++j) {
                            const Draft d = drafts[j];
                            if (d.place != place) continue;
                            if ((int)d.seen < tid) keep = false;
                            if ((int)(d.seen >> 6) == w) m |= uint64_t(1) << (d.seen & 63);
                        }
                        nodes[mine * a.words + w] = m;
                    }
                }
                __syncthreads();
                if (mine >= 0) drafts[mine] = Draft{keep ? place : -1, 0.0f, held_count != 0, (held_count & ~kPrompt) != 0};
            }
            inv = 1.0f / rep;
#pragma unroll
            for (int j0 = 0; j0 < C; j0 += 8 * NTHR) {
                const int j = j0 + 8 * tid;
                if (C < 8 * NTHR && j >= C) break;
                uint32_t f = 0, g = 0;
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    u32x4 n = *reinterpret_cast<const u32x4*>(count + j + e), m = {0, 0, 0, 0};
                    if (biases) m = *reinterpret_cast<const u32x4*>(last + j + e);
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const uint32_t c = n[i4] & ~kPrompt;
                        f |= (uint32_t)(n[i4] != 0) << (e + i4);
                        float y = -0.0f;
                        if (m[i4]) y = (int)m[i4] - 1 - lo < NTHR ? value[m[i4] - 1 - lo] : z.bias[m[i4] - 1];
                        if (c != 0) y -= fmaf(freq, (float)c, pres);
                        n[i4] = __float_as_uint(y);
                        g |= (uint32_t)(n[i4] != 0x80000000u) << (e + i4);
                    }
                    *reinterpret_cast<u32x4*>(count + j + e) = n;
                }
                reinterpret_cast<uint8_t*>(seen)[j / 8] = (uint8_t)f;
                reinterpret_cast<uint8_t*>(changed)[j / 8] = (uint8_t)(f | g);
            }
            __syncthreads();
            if (drafted) {
                if (mine >= 0) {
                    drafts[mine].shift = shift[place];
                    atomicOr(&changed[place >> 5], 1u << (place & 31));
                }
                __syncthreads();
            }
            own_drafts = false;
            if (drafted) {
                for (int j = lane; j < n_drafts; j += 64) own_drafts |= drafts[j].place >= 0 && drafts[j].place / CW == wave;
                own_drafts = __ballot(own_drafts) != 0;
            }
            built = true;
        }
        for (; i + 1 < stop; i += 2) {
            step(x, y, i);
            step(y, x, i + 1);
        }
        if (i < stop) {
            step(x, y, i);
            x = y;
            ++i;
        }
    }
}

template <bool BF16, int NVEC>
hipError_t go(const LogitsArgs& a, int rows, bool past, hipStream_t s) {
    constexpr int C = NTHR * (BF16 ? 8 : 4) * NVEC;
    const bool repeats = a.repetition || a.presence || a.frequency;
    const size_t lds = a.bias_start || repeats ? lds_bytes(C, a.bias_start, a.words) : 0;
    const int chunks = (int)((a.V + C - 1) / C);
    const int64_t blocks = (a.T + rows - 1) / rows * chunks, most = int64_t(1) << 23;
    // more than a grid may have (2^32 threads) go into launches one after the other
    for (int64_t base = 0; base < blocks; base += most) {
        const unsigned grid = (unsigned)(blocks - base < most ? blocks - base : most);
        if (past) logits_kernel<BF16, NVEC, true><<<grid, NTHR, lds, s>>>(a, rows, chunks, base);
        else logits_kernel<BF16, NVEC, false><<<grid, NTHR, lds, s>>>(a, rows, chunks, base);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_logits(bool bf16, const LogitsArgs& a, hipStream_t s) {
    // Chunks of up to 4096 tokens (32 KB of LDS, four workgroups a CU) as large as leave 1024
    // workgroups of one row, and rows to a workgroup (of one request, so as many as it may
    // have) while there are 2048: the rows of a request share its counts (980 rows of 128003
    // of 40 requests, all rules, two sets of tensors in turn, chunks of 4096: 345 us with one
    // row, 158 with 4, 134 with 8, 130 with 16; chunks of 2048 361, 163, 134 and 130; 256 rows
    // of requests of their own 77 against 92).  max_new only bounds a request's rows: where
    // most have one, a workgroup counts for several requests in turn, which costs nothing
    // (980 requests of one row, none drafted, max_new 48: 284 us against 295 with max_new 1).
    const int pv = NTHR * (bf16 ? 8 : 4), most = bf16 ? 2 : 4;
    int nvec = 1;
    while (nvec < most && a.T * ((a.V + 2 * pv * nvec - 1) / (2 * pv * nvec)) >= 1024) nvec *= 2;
    const int64_t chunks = (a.V + pv * nvec - 1) / (pv * nvec);
    int64_t rows = a.T * chunks / 2048;
    const int64_t of_one = a.start ? (a.max_new > 1 ? a.max_new : 1) : 1;
    if (rows > of_one) rows = of_one;
    if (rows > kMaxRows) rows = kMaxRows;
    if (rows < 1) rows = 1;
    const bool past = (double)a.T * (double)a.V * (bf16 ? 2 : 4) > 48e6;
    if (bf16) return nvec == 1 ? go<true, 1>(a, (int)rows, past, s) : go<true, 2>(a, (int)rows, past, s);
    if (nvec == 1) return go<false, 1>(a, (int)rows, past, s);
    return nvec == 2 ? go<false, 2>(a, (int)rows, past, s) : go<false, 4>(a, (int)rows, past, s);
}

}  // namespace cola
