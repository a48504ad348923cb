// prefix_attn.hip -- attention of a batch whose requests share a prefix, over a
// paged cache (cola_prefix_attn).
//
// Row i of a request with n rows (query head h, key head h / g, g = heads_q /
// heads) sees the L tokens of the prefix and the request's own tokens 0 .. kv -
// n + i.  Softmax over the union splits into parts of the keys: with m the
// largest score of a part, l = sum exp(s - m) and o = sum exp(s - m) v, the whole
// is sum_p exp(m_p - M) o_p / sum_p exp(m_p - M) l_p, M = max m_p.  So the prefix
// is one matrix problem of all rows of the batch against shared keys, each
// request's own tokens another, both split along the keys where there are few
// rows, and a second launch joins the parts in a fixed order.
//
// A work item is (row tile, key head, part of the keys).  Its rows are (query,
// head of the group) pairs, the head running fastest; NT columns of 16 of them
// are the matrix instructions' n side.  The four waves of a workgroup take the
// part's blocks of 32 keys in turn, each with its own running maximum and sum, and
// join through LDS at the end.  A wave keeps everything in registers:
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16, K rows straight from the cache in the
//                 operand's layout (lane l: key l % 16, 8 elements at 8 (l / 16)),
//                 two tiles of 16 keys;
//   O^T += V^T P^T  lane l = 16 g + c holds P of column c for the keys 4 g .. 4 g
//                 + 3 of both tiles, which are the 8 values the instruction wants
//                 from it when the 32 keys are numbered in that order.  V is read
//                 to match: lane (g, c) loads those 8 keys' elements c D .. c D +
//                 D - 1 (D = head_dim / 16), and halves of pairs of keys are put
//                 together with one v_perm a pair.  Row m of output tile t is
//                 then element D m + t, so a lane ends with 4 D neighbouring
//                 elements of its row.
// The probabilities are rounded to bf16 for the second product only; the sum l is
// of the fp32 ones (the log-sum-exp needs them), each lane's own until the end.
// No LDS, no transposing pass, no barrier in the loop: key and value bytes go
// from memory to the matrix unit.
#include <math.h>

#include "serve.hpp"
#include "device_math.hpp"

namespace cola {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int NW = 4;                     // waves per workgroup
constexpr int KB = 32;                    // keys per block of a wave
constexpr int NTHR = 64 * NW;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Running maximum of a row that has seen nothing: finite, so that differences
// with it are.
constexpr float kNone = -3.0e38f;
// Probabilities may reach 2^kSlack against a stale maximum: the accumulators are
// rescaled only when a block exceeds it by more.
constexpr float kSlack = 8.0f;

struct Args {
    const uint16_t *q, *K, *V;
    const int32_t *prefix_table, *table, *kv_len, *start;
    uint16_t* out;
    float *lse, *part, *ml;
    int64_t ldq, ldo, rows, max_pages, n_pages, T;
    int n_req, hq, hk, g, lg_page;
    int prefix, max_kv, max_new;
    int64_t items, items_p;
    int tiles_p, splits_p, chunk_p;
    int tiles_s, splits_s, chunk_s;
    int direct;                           // one part in all, of the requests' own keys: the item writes the result
    float c;                              // scale log2 e
};

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// The maximum and the sum over lanes l, l ^ 16, l ^ 32, l ^ 48: a column's four.
__device__ __forceinline__ float column_max(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ float column_sum(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Request r, from whatever the arrays hold: its first row and how many (at most
// max_new), and of its own tokens the index of the first new one and the end.
struct Span {
    int row, n, first, end;
};
__device__ __forceinline__ Span span_of(const Args& a, int r) {
    Span s;
    int64_t all = r < a.T ? 1 : 0;
    s.row = r;
    if (a.start) {
        const int64_t lo = min(max((int64_t)a.start[r], (int64_t)0), a.T), hi = min((int64_t)a.start[r + 1], a.T);
        s.row = (int)lo;
        all = max(hi - lo, (int64_t)0);
    }
    s.n = (int)min(all, (int64_t)a.max_new);
    const int kv = a.max_kv > 0 ? max(a.kv_len[r], 0) : 0;
    s.first = (int)(kv - all);
    s.end = min(kv, a.max_kv);
    return s;
}

template <int HD, int NT>
struct Wave {
    static constexpr int KK = HD / 32;    // steps of the first product
    static constexpr int D = HD / 16;     // neighbouring head elements of a lane, and output tiles
    bf16x8 q[NT][KK];
    f32x4 o[D][NT];
    float m[NT], l[NT];                   // l: of this lane's keys
    int lim[NT];                          // keys that this lane's row sees

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            m[n] = kNone;
            l[n] = 0.0f;
#pragma unroll
            for (int t = 0; t < D; ++t) o[t][n] = f32x4{0, 0, 0, 0};
        }
    }
};

// Row `key` of V, this lane's D elements.
template <int D>
struct VRow;
template <>
struct VRow<8> { typedef u32x4 type; };
template <>
struct VRow<4> { typedef u32x2 type; };

__device__ __forceinline__ bool not_finite(uint32_t bf16) { return (bf16 & 0x7f80u) == 0x7f80u; }

// The value operand of output tile t: element t of the lane's 8 keys.
template <int D, class R>
__device__ __forceinline__ bf16x8 v_frag(const R (&v)[8], int t) {
    u32x4 f;
    const uint32_t sel = t & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
    for (int p = 0; p < 4; ++p) f[p] = __builtin_amdgcn_perm(v[2 * p + 1][t / 2], v[2 * p][t / 2], sel);
    return __builtin_bit_cast(bf16x8, f);
}

// One block of 32 keys from kb on.  MASK: some row does not see all of them, or
// a page is missing; keys from `end` on hold no tokens.
template <int HD, int NT, bool MASK>
__device__ __forceinline__ void block(Wave<HD, NT>& w, const Args& a, const int32_t* table, int head, int kb, int end,
                                      int lane) {
    constexpr int KK = HD / 32, D = HD / 16;
    typedef typename VRow<D>::type R;
    const int g = lane >> 4, c = lane & 15;
    int64_t base[2];
    bool there[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int k0 = kb + 16 * i;
        int64_t page = 0;
        there[i] = true;
        if (!MASK || k0 < end) page = table[k0 >> a.lg_page];
        else there[i] = false;
        if (page < 0 || page >= a.n_pages) {
            there[i] = false;
            page = 0;
        }
        base[i] = ((((page * a.hk + head) << a.lg_page) + (k0 & ((1 << a.lg_page) - 1)))) * HD;
    }
    u32x4 kf[2][KK];
    R v[8];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint16_t* p = a.K + base[i] + c * HD + 8 * g;
        const bool ok = !MASK || (there[i] && kb + 16 * i + c < end);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
            kf[i][kk] = ok ? *reinterpret_cast<const u32x4*>(p + 32 * kk) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint16_t* p = a.V + base[i] + 4 * g * HD + D * c;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool ok = !MASK || (there[i] && kb + 16 * i + 4 * g + j < end);
            R x{};
            if (ok) x = *reinterpret_cast<const R*>(p + j * HD);
            v[4 * i + j] = x;
        }
    }
    f32x4 s[2][NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i][n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) s[i][n] = mfma(__builtin_bit_cast(bf16x8, kf[i][kk]), w.q[n][kk], s[i][n]);
        }
    bf16x8 p[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        if constexpr (MASK) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!there[i] || kb + 16 * i + 4 * g + j >= w.lim[n]) s[i][n][j] = -INFINITY;
        }
        float mb = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) mb = fmaxf(mb, s[i][n][j]);
        mb = column_max(mb) * a.c;
        if (__ballot(mb > w.m[n] + kSlack) != 0) {
            const float mn = fmaxf(w.m[n], mb);
            const float alpha = exp2_hw(w.m[n] - mn);
#pragma unroll
            for (int t = 0; t < D; ++t) w.o[t][n] *= alpha;
            w.l[n] *= alpha;
            w.m[n] = mn;
        }
        u32x4 f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                e[j] = exp2_hw(fmaf(s[i][n][j], a.c, -w.m[n]));
                w.l[n] += e[j];
            }
            f[2 * i] = pack_bf16x2(e[0], e[1]);
            f[2 * i + 1] = pack_bf16x2(e[2], e[3]);
        }
        p[n] = __builtin_bit_cast(bf16x8, f);
    }
    // A key that some row of the tile sees and another does not must not reach the
    // second by 0 * inf: values that are not finite leave the product, and go to
    // the rows that see them by themselves.
    bool odd = false;
    if constexpr (MASK) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int x = 0; x < D / 2; ++x) odd |= not_finite(v[j][x] & 0xffffu) || not_finite(v[j][x] >> 16);
        odd = __ballot(odd) != 0;
        if (odd) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int x = 0; x < D / 2; ++x)
                    v[j][x] &= (not_finite(v[j][x] & 0xffffu) ? 0u : 0xffffu) |
                               (not_finite(v[j][x] >> 16) ? 0u : 0xffff0000u);
        }
    }
#pragma unroll
    for (int t = 0; t < D; ++t) {
        const bf16x8 vf = v_frag<D>(v, t);
#pragma unroll
        for (int n = 0; n < NT; ++n) w.o[t][n] = mfma(vf, p[n], w.o[t][n]);
    }
    if constexpr (MASK) {
        if (odd) {
#pragma unroll 1
            for (int k = 0; k < KB; ++k) {
                const int i = k / 16;
                if (!(i ? there[1] : there[0]) || kb + k >= end) continue;
                // this lane's elements of its rows: 4 D from 4 D g on
                const uint16_t* x = a.V + (i ? base[1] : base[0]) + (k - 16 * i) * HD + 4 * D * g;
#pragma unroll
                for (int e = 0; e < 4 * D; ++e) {
                    const uint32_t y = x[e];
                    if (!not_finite(y)) continue;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        if (kb + k < w.lim[n]) w.o[e % D][n][e / D] += bf16_to_f32(y);
                }
            }
        }
    }
}

// LDS of one wave's state on its way to another: accumulators, sum, maximum.
template <int HD, int NT>
constexpr int WAVES = HD * NT <= 128 ? 3 : 2;
template <int HD, int NT>
constexpr int kStateFloats = 64 * NT * (HD / 16 * 4 + 2);

template <int HD, int NT>
__device__ __forceinline__ void give(const Wave<HD, NT>& w, float* buf, int lane) {
    constexpr int D = HD / 16;
    f32x4* b = reinterpret_cast<f32x4*>(buf);
#pragma unroll
    for (int t = 0; t < D; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n) b[64 * (t * NT + n) + lane] = w.o[t][n];
    float* r = buf + 64 * 4 * D * NT;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        r[64 * (2 * n) + lane] = w.l[n];
        r[64 * (2 * n + 1) + lane] = w.m[n];
    }
}

template <int HD, int NT>
__device__ __forceinline__ void take(Wave<HD, NT>& w, const float* buf, int lane) {
    constexpr int D = HD / 16;
    const f32x4* b = reinterpret_cast<const f32x4*>(buf);
    const float* r = buf + 64 * 4 * D * NT;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float lo = r[64 * (2 * n) + lane], mo = r[64 * (2 * n + 1) + lane];
        const float mn = fmaxf(w.m[n], mo);
        const float x = exp2_hw(w.m[n] - mn), y = exp2_hw(mo - mn);
        w.m[n] = mn;
        w.l[n] = w.l[n] * x + lo * y;
#pragma unroll
        for (int t = 0; t < D; ++t) w.o[t][n] = w.o[t][n] * x + b[64 * (t * NT + n) + lane] * y;
    }
}

// One work item: rows rho = tile0 .. of the batch's row `row0` on (rho / g tokens
// further, head rho % g of the group), keys k0 .. of a table that ends at `end`.
// Row rho sees the keys up to first + rho / g, or all of them.
template <int HD, int NT, bool CAUSAL>
__device__ __forceinline__ void item(const Args& a, float* lds, const int32_t* table, int head, int row0, int tile0,
                                     int n_rows, int first, int end, int k0, int chunk, int slot) {
    constexpr int KK = HD / 32, D = HD / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, c = lane & 15;
    auto seen = [&](int rho) { return CAUSAL ? (int)min((int64_t)first + 1 + rho / a.g, (int64_t)end) : end; };
    Wave<HD, NT> w;
    w.clear();
    int64_t row[NT];
    int hh[NT];
    bool live[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int rho = tile0 + 16 * n + c;
        const int t = rho / a.g;
        live[n] = rho < n_rows;
        row[n] = row0 + t;
        hh[n] = head * a.g + (rho - t * a.g);
        w.lim[n] = live[n] ? seen(rho) : 0;
        const uint16_t* p = a.q + row[n] * a.ldq + hh[n] * HD + 8 * g;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            u32x4 x = {0, 0, 0, 0};
            if (live[n]) x = *reinterpret_cast<const u32x4*>(p + 32 * kk);
            w.q[n][kk] = __builtin_bit_cast(bf16x8, x);
        }
    }
    // keys that the tile's first row sees, and its last
    const int all = seen(tile0), any = min(seen(min(tile0 + 16 * NT, n_rows) - 1), k0 + chunk);
#pragma unroll 1
    for (int kb = k0 + KB * wave; kb < any; kb += KB * NW) {
        bool whole = kb + KB <= min(all, any);
        if (whole) {
            const int64_t p0 = table[kb >> a.lg_page], p1 = table[(kb + 16) >> a.lg_page];
            whole = p0 >= 0 && p0 < a.n_pages && p1 >= 0 && p1 < a.n_pages;
        }
        if (whole) block<HD, NT, false>(w, a, table, head, kb, any, lane);
        else block<HD, NT, true>(w, a, table, head, kb, any, lane);
    }
    // waves 2, 3 into 0, 1, then 1 into 0
    float* mine = lds + (wave & 1) * kStateFloats<HD, NT>;
    if (wave >= 2) give<HD, NT>(w, mine, lane);
    __syncthreads();
    if (wave < 2) take<HD, NT>(w, mine, lane);
    __syncthreads();
    if (wave == 1) give<HD, NT>(w, lds, lane);
    __syncthreads();
    if (wave != 0) return;
    take<HD, NT>(w, lds, lane);
    // lane (g, c): row c of each column, elements 4 D g .. 4 D g + 4 D - 1, the
    // element D (4 g + i) + t in o[t][i]
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const float l = column_sum(w.l[n]);
        if (!live[n]) continue;
        const int64_t id = row[n] * a.hq + hh[n];
        if (a.direct) {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            uint16_t* y = a.out + row[n] * a.ldo + hh[n] * HD + 4 * D * g;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < D; t += 4) {
                    const u32x2 x = {pack_bf16x2(w.o[t][n][i] * inv, w.o[t + 1][n][i] * inv),
                                     pack_bf16x2(w.o[t + 2][n][i] * inv, w.o[t + 3][n][i] * inv)};
                    *reinterpret_cast<u32x2*>(y + D * i + t) = x;
                }
            if (a.lse && g == 0) a.lse[hh[n] * a.T + row[n]] = l == 0.0f ? -INFINITY : (w.m[n] + log2f(l)) * kLn2;
        } else {
            float* y = a.part + (slot * a.rows + id) * HD + 4 * D * g;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < D; t += 4) {
                    const f32x4 x = {w.o[t][n][i], w.o[t + 1][n][i], w.o[t + 2][n][i], w.o[t + 3][n][i]};
                    *reinterpret_cast<f32x4*>(y + D * i + t) = x;
                }
            if (g == 0) *reinterpret_cast<float2*>(a.ml + 2 * (slot * a.rows + id)) = make_float2(w.m[n], l);
        }
    }
}

// Parts of the keys that a request of `end` own tokens has.
__device__ __forceinline__ int parts_of(const Args& a, int end) {
    return a.splits_s > 0 ? min((end + a.chunk_s - 1) / a.chunk_s, a.splits_s) : 0;
}

template <int HD, int NTP, int NTS>
__global__ __launch_bounds__(NTHR, 1) void prefix_attn_kernel(const Args a) {
    constexpr int NTM = NTP > NTS ? NTP : NTS;
    __shared__ __attribute__((aligned(16))) float lds[2 * kStateFloats<HD, NTM>];
    for (int64_t at = blockIdx.x; at < a.items; at += gridDim.x) {
        if (at != blockIdx.x) __syncthreads();          // the item before has left the LDS
        if (at < a.items_p) {
            int b = (int)at;
            const int tile = b % a.tiles_p;
            b /= a.tiles_p;
            const int head = b % a.hk, split = b / a.hk;
            // rows of the batch up to the last that holds a token
            const int64_t hi = a.start ? min(max((int64_t)a.start[a.n_req], (int64_t)0), a.T) : min((int64_t)a.n_req, a.T);
            const int tile0 = tile * 16 * NTP, n_rows = (int)hi * a.g;
            if (tile0 < n_rows)
                item<HD, NTP, false>(a, lds, a.prefix_table, head, 0, tile0, n_rows, 0, a.prefix, split * a.chunk_p,
                                     a.chunk_p, split);
        } else {
            int64_t b = at - a.items_p;
            const int tile = (int)(b % a.tiles_s);
            b /= a.tiles_s;
            const int head = (int)(b % a.hk);
            b /= a.hk;
            const int split = (int)(b % a.splits_s), r = (int)(b / a.splits_s);
            const Span s = span_of(a, r);
            const int tile0 = tile * 16 * NTS, n_rows = s.n * a.g;
            if (tile0 < n_rows && (a.direct || split < parts_of(a, s.end)))
                item<HD, NTS, true>(a, lds, a.table + r * a.max_pages, head, s.row, tile0, n_rows, s.first, s.end,
                                    split * a.chunk_s, a.chunk_s, a.splits_p + split);
        }
    }
}

// The parts of each row joined, in their order: a thread for four elements.
template <int HD>
__global__ __launch_bounds__(NTHR) void prefix_join_kernel(const Args a) {
    constexpr int TPR = HD / 4;
    for (int r = blockIdx.y; r < a.n_req; r += gridDim.y) {
        const Span s = span_of(a, r);
        const int parts = a.splits_p + parts_of(a, s.end);
        for (int64_t j = (int64_t)blockIdx.x * (NTHR / TPR) + threadIdx.x / TPR; j < (int64_t)s.n * a.hq;
             j += (int64_t)gridDim.x * (NTHR / TPR)) {
            const int64_t id = (int64_t)s.row * a.hq + j;
            const int e = 4 * (threadIdx.x % TPR);
            float M = kNone;
            for (int p = 0; p < parts; ++p) M = fmaxf(M, a.ml[2 * (p * a.rows + id)]);
            float l = 0.0f;
            f32x4 o = {0, 0, 0, 0};
            for (int p = 0; p < parts; ++p) {
                const float2 x = *reinterpret_cast<const float2*>(a.ml + 2 * (p * a.rows + id));
                const float f = exp2_hw(x.x - M);
                l += f * x.y;
                o += f * *reinterpret_cast<const f32x4*>(a.part + (p * a.rows + id) * HD + e);
            }
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const int64_t t = id / a.hq, h = id - t * a.hq;
            *reinterpret_cast<u32x2*>(a.out + t * a.ldo + h * HD + e) =
                u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
            if (a.lse && e == 0) a.lse[h * a.T + t] = l == 0.0f ? -INFINITY : (M + log2f(l)) * kLn2;
        }
    }
}

Args args_of(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t) {
    Args a{};
    a.q = t.q; a.K = t.K; a.V = t.V;
    a.prefix_table = t.prefix_table; a.table = t.table; a.kv_len = t.kv_len; a.start = t.start;
    a.out = t.out; a.lse = t.lse;
    const int64_t n = (p.splits_p + p.splits_s) * p.rows;
    a.ml = static_cast<float*>(t.ws);
    a.part = a.ml ? a.ml + (2 * n + 63) / 64 * 64 : nullptr;
    a.ldq = sh.ldq; a.ldo = sh.ldo; a.rows = p.rows; a.max_pages = sh.max_pages; a.n_pages = sh.n_pages; a.T = sh.T;
    a.n_req = (int)sh.n_req; a.hq = sh.hq; a.hk = sh.hk; a.g = sh.hq / sh.hk;
    a.lg_page = __builtin_ctzll((unsigned long long)sh.page_size);
    a.prefix = (int)sh.prefix; a.max_kv = (int)sh.max_kv; a.max_new = (int)sh.max_new;
    a.tiles_p = p.tiles_p; a.splits_p = p.splits_p; a.chunk_p = (int)p.chunk_p;
    a.tiles_s = p.tiles_s; a.splits_s = p.splits_s; a.chunk_s = (int)p.chunk_s;
    a.items_p = (int64_t)p.splits_p * p.tiles_p * sh.hk;
    a.items = a.items_p + sh.n_req * p.splits_s * p.tiles_s * sh.hk;
    a.direct = p.direct;
    a.c = (float)(sh.scale * (double)kLog2e);
    return a;
}

template <int HD>
hipError_t go(const PrefixAttnPlan& p, const Args& a, unsigned grid, hipStream_t s) {
    if (p.nt_p == 1) prefix_attn_kernel<HD, 1, 1><<<grid, NTHR, 0, s>>>(a);
    else if (p.nt_s == 1) prefix_attn_kernel<HD, 2, 1><<<grid, NTHR, 0, s>>>(a);
    else prefix_attn_kernel<HD, 2, 2><<<grid, NTHR, 0, s>>>(a);
    return hipGetLastError();
}

int columns(int64_t rows) { return rows <= 16 ? 1 : 2; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

PrefixAttnPlan plan_prefix_attn(const PrefixAttnShape& sh) {
    PrefixAttnPlan p{};
    const int64_t g = sh.hq / sh.hk;
    const int64_t new_rows = sh.max_new < sh.T ? sh.max_new : sh.T;
    p.rows = sh.T * sh.hq;
    p.nt_s = columns(new_rows * g);
    p.nt_p = columns(sh.T * g);                              // never below nt_s
    p.tiles_p = (int)ceil_div(sh.T * g, 16 * p.nt_p);
    p.tiles_s = (int)ceil_div(new_rows * g, 16 * p.nt_s);
    // Parts of the keys: about a thousand work items in all, none below 256 keys
    const int64_t base_p = (int64_t)p.tiles_p * sh.hk, base_s = sh.n_req * p.tiles_s * sh.hk;
    const int64_t blocks = base_p * ceil_div(sh.prefix, KB) + base_s * ceil_div(sh.max_kv, KB);
    int64_t chunk = ceil_div(blocks, 1024);
    if (chunk < 8) chunk = 8;
    // as many parts as that gives, of equal length
    auto parts = [&](int64_t keys, int* n, int64_t* len) {
        if (keys == 0) {
            *n = 0;
            *len = KB;
            return;
        }
        int64_t k = ceil_div(ceil_div(keys, KB), chunk);
        if (k > 64) k = 64;
        *len = ceil_div(ceil_div(keys, k), KB) * KB;
        *n = (int)ceil_div(keys, *len);
    };
    parts(sh.prefix, &p.splits_p, &p.chunk_p);
    parts(sh.max_kv, &p.splits_s, &p.chunk_s);
    const int64_t n = (p.splits_p + p.splits_s) * p.rows;
    p.direct = p.splits_p == 0 && p.splits_s == 1;
    p.ws_bytes = p.direct || n == 0 ? 0 : (size_t)((2 * n + 63) / 64 * 64 + n * sh.hd) * 4;
    return p;
}

hipError_t launch_prefix_attn(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t,
                              hipStream_t s) {
    const Args a = args_of(sh, p, t);
    if (a.items == 0) return hipSuccess;
    const int64_t grid = a.items < (1 << 22) ? a.items : (1 << 22);
    return sh.hd == 64 ? go<64>(p, a, (unsigned)grid, s) : go<128>(p, a, (unsigned)grid, s);
}

hipError_t launch_prefix_join(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t,
                              hipStream_t s) {
    if (p.direct) return hipSuccess;
    const Args a = args_of(sh, p, t);
    const int64_t new_rows = sh.max_new < sh.T ? sh.max_new : sh.T;
    int64_t gx = ceil_div(new_rows * sh.hq, NTHR / (sh.hd / 4));
    if (gx > 4096) gx = 4096;
    const dim3 grid((unsigned)gx, (unsigned)sh.n_req);
    if (sh.hd == 64) prefix_join_kernel<64><<<grid, NTHR, 0, s>>>(a);
    else prefix_join_kernel<128><<<grid, NTHR, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace cola
