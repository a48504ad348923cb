// prefix_attn.hpp -- attention of a batch whose requests share a prefix, over a
// paged cache: the kernels of cola_prefix_attn (prefix_attn.hip) and of
// cola_tree_attn (tree_attn.hip).
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
// A work item is (row tile, key head, part of the keys), one to a workgroup (a
// loop over items on the GPU held too many registers: two waves a SIMD where four
// to six fit).  Its rows are (query, head of the group) pairs, the head running
// fastest, so that heads that share keys share their reads.  Three kernels' worth
// of tiles, by the number of rows:
//
// 16 or 32 rows (single tokens, short chunks): bound by the keys' bytes, so the
// least may stand between memory and the matrix unit.  A wave keeps everything in
// registers, NT columns of 16 rows:
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
// No LDS, no transposing pass, no barrier in the loop.  The four waves of a
// workgroup take the part's blocks of 32 keys in turn, each with its own running
// maximum and sum, and join through LDS at the end; where single-token requests
// are many, a wave has an item of its own.  200 requests of 32 heads of 128 and up to
// 300 own tokens (490 MB): 96 us, 5.1 TB/s of the 6.2 that reading alone reaches.
//
// More rows: tiles of 128, bound by the softmax's arithmetic and the matrix
// products one after the other, keys staged in LDS once for all of them (below).  16
// chunks of up to 256 tokens, 32 heads of 64, behind 4096 + 1000 tokens (84 GFLOP):
// 138 us, 610 TFLOP/s; at a head of 64 the exponentials, maxima, sums and conversions
// take the vector unit 20 cycles a score and wave, the two products the matrix unit
// 16, and with two waves a SIMD neither is busy all the time (56 and 31 % of the
// launch).
//
// Trees (cola_tree_attn) use the same tiles: a block of keys that holds new tokens takes
// a word of each row's mask where causal rows take a limit, and all blocks before it are
// as they were.  32 requests of up to 4000 keys, trees of up to 32 nodes, 32 heads over 8
// of 128 (282 MB): 74 us with the keys still in the last-level cache, 81 without.
//
// Short prefixes: a request's own items read them along (the bytes come from L2),
// and neither partial rows nor a join are left.
//
// The probabilities are rounded to bf16 for the second product only (the matrix
// unit's type; half a step of 2^-8 each, which averages out over the keys); the sum
// l is of the fp32 ones (the log-sum-exp needs them), each lane's own until the end.
#pragma once

#include <math.h>

#include <type_traits>

#include "serve.hpp"
#include "device_math.hpp"

namespace cola {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lptr4_t;
typedef __attribute__((address_space(3))) void* lptr_t;

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
    int64_t blocks, items_p, base;        // workgroups' turns, those on the prefix, the launch's first
    int64_t units_p, units_s;             // (head, part) pairs of the prefix; (request, head, part) of the own keys
    int tiles_p, splits_p, chunk_p;
    int tiles_s, splits_s, chunk_s;
    int direct;                           // one part in all, of the requests' own keys: the item writes the result
    const uint64_t* mask;                 // trees: [T][words], which new tokens a row sees
    int words;
    int slots;                            // trees: workgroups that the own keys are cut for by their lengths (0: by chunk_s)
    int64_t work_p;                       // tiles and stages of the prefix
    int32_t* chunk;                       // where the first launch leaves the part's length for the second
    float c;                              // scale log2 e
};

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// exp2 by the hardware instruction alone: results that it flushes to zero are far
// below the resolution of what they are added to.
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

// An entry of the tables, lengths and starts, which no launch of this file writes:
// through the constant address space, so that it comes by the scalar unit and no
// wait for it is one for the vector loads in flight.
__device__ __forceinline__ int entry(const int32_t* p, int64_t i) {
    return ((const __attribute__((address_space(4))) int32_t*)p)[i];
}

// Wave-uniform values kept in scalar registers (a descriptor's parts must be).
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32 | (uint32_t)uniform((int)x));
}

// Request r, from whatever the arrays hold: its first row and how many there are (up
// to T, at most max_new), and of its own tokens the index of the first new one and
// the end.  Its new tokens are counted past T, too: those that have no row are the
// last ones of kv_len, and the rows that are there do not see them.
struct Span {
    int row, n, first, end;
};
__device__ __forceinline__ Span span_of(const Args& a, int r) {
    Span s;
    int64_t all = r < a.T ? 1 : 0, here = all;
    s.row = r;
    if (a.start) {
        const int64_t lo = max((int64_t)entry(a.start, r), (int64_t)0), hi = entry(a.start, r + 1);
        s.row = (int)min(lo, a.T);
        all = max(hi - lo, (int64_t)0);
        here = max(min(hi, a.T) - lo, (int64_t)0);
    }
    s.n = (int)min(here, (int64_t)a.max_new);
    const int kv = a.max_kv > 0 ? max(entry(a.kv_len, r), 0) : 0;
    s.first = (int)(kv - all);
    s.end = min(kv, a.max_kv);
    return s;
}

// Which of a table's keys a row sees: all; those up to its own; or all older ones and
// those new ones whose bits are set in its mask.
enum See : int { SEE_ALL = 0, SEE_CAUSAL = 1, SEE_TREE = 2 };

// Bit x: a row whose mask lies at `row` (its first word is w0) sees the key that is d + x
// tokens behind its request's first new one.  d is the same for a wave; only trees of
// more than 64 nodes read words here.
__device__ __forceinline__ uint64_t tree_bits(const uint64_t* row, uint64_t w0, int words, int d) {
    if (d <= -64) return ~uint64_t(0);
    if (d < 0) return ((uint64_t(1) << -d) - 1) | (w0 << -d);
    const int at = d >> 6, sh = d & 63;
    uint64_t x = 0;
    if (at < words) x = (at == 0 ? w0 : row[at]) >> sh;
    if (sh > 0 && at + 1 < words) x |= row[at + 1] << (64 - sh);
    return x;
}

template <int HD, int NT>
struct Wave {
    static constexpr int KK = HD / 32;    // steps of the first product
    static constexpr int D = HD / 16;     // neighbouring head elements of a lane, and output tiles
    bf16x8 q[NT][KK];
    f32x4 o[D][NT];
    float m[NT], l[NT];                   // l: of this lane's keys
    int lim[NT];                          // keys that this lane's row sees
    const uint64_t* mask[NT];             // trees: the row's mask, and its first word
    uint64_t mask0[NT];

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
// The top bit of each half of a pair that is not finite: its exponent plus one
// carries there and no further.
__device__ __forceinline__ uint32_t not_finite2(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
// The pair with those halves zero.
__device__ __forceinline__ uint32_t finite2(uint32_t x) { return x & ~((not_finite2(x) >> 15) * 0xffffu); }

// The value operand of output tile t: element t of the lane's 8 keys.
template <int D, class R>
__device__ __forceinline__ bf16x8 v_frag(const R (&v)[8], int t) {
    u32x4 f;
    const uint32_t sel = t & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
    for (int p = 0; p < 4; ++p) f[p] = __builtin_amdgcn_perm(v[2 * p + 1][t / 2], v[2 * p][t / 2], sel);
    return __builtin_bit_cast(bf16x8, f);
}

// The page of the 16 keys from k0 on; tiles that begin at or past `end` are looked
// up at the last one before it (their table entry may not exist).
__device__ __forceinline__ int page_of(const Args& a, const int32_t* table, int k0, int end) {
    const int k = min(k0, (end - 1) & ~15);
    return uniform(entry(table, k >> a.lg_page));
}
__device__ __forceinline__ bool in_cache(const Args& a, int page) { return (uint32_t)page < (uint32_t)a.n_pages; }
// Row of K and V (in units of HD) at which key k of a page lies.
__device__ __forceinline__ int64_t row_of(const Args& a, int page, int head, int k) {
    return (((int64_t)page * a.hk + head) << a.lg_page) + (k & ((1 << a.lg_page) - 1));
}
// Keys from k0 on, of 16, that lie in the cache and before `end`.
__device__ __forceinline__ int rows_in(bool there, int k0, int end) {
    return there && k0 < end ? (end - k0 < 16 ? end - k0 : 16) : 0;
}

// Descriptor of `rows` rows of HD from row `at` on; reads past them give zeros.
template <int HD>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_of(const uint16_t* base, int64_t at, int rows) {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(uniform64((int64_t)(base + at * HD))), (short)0,
                                             uniform(rows) * 2 * HD, 0x00020000);
}

// The keys and values of one block of 32 keys in a wave's registers; keys from
// `end` on and those of missing pages are zeros.
template <int HD>
struct Keys {
    static constexpr int KK = HD / 32, D = HD / 16;
    typedef typename VRow<D>::type R;
    bool there[2];
    u32x4 k[2][KK];
    R v[8];

    __device__ __forceinline__ void load(const Args& a, const int32_t* table, int head, int kb, int end, int lane) {
        const int g = lane >> 4, c = lane & 15;
        const int ko = 2 * (c * HD + 8 * g), vo = 2 * (4 * g * HD + D * c);
        __amdgpu_buffer_rsrc_t rv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int page = page_of(a, table, kb + 16 * i, end);
            there[i] = in_cache(a, page);
            const int rows = rows_in(there[i], kb + 16 * i, end);
            const int64_t at = row_of(a, page, head, kb + 16 * i);
            const __amdgpu_buffer_rsrc_t rk = rows_of<HD>(a.K, at, rows);
            rv[i] = rows_of<HD>(a.V, at, rows);
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) k[i][kk] = __builtin_amdgcn_raw_buffer_load_b128(rk, ko + 64 * kk, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (D == 8) v[4 * i + j] = __builtin_amdgcn_raw_buffer_load_b128(rv[i], vo + 2 * HD * j, 0, 0);
                else v[4 * i + j] = __builtin_amdgcn_raw_buffer_load_b64(rv[i], vo + 2 * HD * j, 0, 0);
            }
    }
};

// One block: the keys kb .. kb + 31, those from `end` on without a token.  `part`
// (wave-uniform): some row does not see all of them, or a page is missing.
// SEE: whether the rows see different keys; `first`: trees, the request's first new token.
template <int HD, int NT, int SEE>
__device__ __forceinline__ void block(Wave<HD, NT>& w, const Args& a, Keys<HD>& x, const int32_t* table, int head, int kb,
                                      int end, int first_new, bool part, int lane) {
    constexpr int KK = HD / 32, D = HD / 16;
    const int g = lane >> 4;
    f32x4 s[2][NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i][n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) s[i][n] = mfma16(__builtin_bit_cast(bf16x8, x.k[i][kk]), w.q[n][kk], s[i][n]);
        }
    // A key that some row of the tile sees and another does not must not reach the
    // second by 0 * inf: values that are not finite leave the product, and go to
    // the rows that see them by themselves.
    bool odd = false;
    uint32_t bits[NT];                                  // trees: which of the 32 keys a row sees
    if (part) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            bits[n] = SEE == SEE_TREE ? (uint32_t)tree_bits(w.mask[n], w.mask0[n], a.words, kb - first_new) : ~0u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int first = kb + 16 * i + 4 * g;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int lim = x.there[i] ? w.lim[n] : 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (first + j >= lim || (SEE == SEE_TREE && !(bits[n] >> (16 * i + 4 * g + j) & 1))) s[i][n][j] = -INFINITY;
            }
        }
        if constexpr (SEE != SEE_ALL) {
            uint32_t any = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int d = 0; d < D / 2; ++d) {
                    any |= not_finite2(x.v[j][d]);
                    x.v[j][d] = finite2(x.v[j][d]);
                }
            odd = __ballot(any != 0) != 0;
        }
    }
    bf16x8 p[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float mb = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 4; j += 2) mb = fmaxf(fmaxf(mb, s[i][n][j]), s[i][n][j + 1]);
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
#pragma unroll
    for (int t = 0; t < D; ++t) {
        const bf16x8 vf = v_frag<D>(x.v, t);
#pragma unroll
        for (int n = 0; n < NT; ++n) w.o[t][n] = mfma16(vf, p[n], w.o[t][n]);
    }
    if constexpr (SEE != SEE_ALL) {
        if (odd) {
#pragma unroll 1
            for (int k = 0; k < min(KB, end - kb); ++k) {
                const int page = page_of(a, table, kb + k, end);
                if (!in_cache(a, page)) continue;
                // this lane's elements of its rows: 4 D from 4 D g on
                const uint16_t* y = a.V + row_of(a, page, head, kb + k) * HD + 4 * D * g;
#pragma unroll
                for (int e = 0; e < 4 * D; ++e) {
                    const uint32_t z = y[e];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        w.o[e % D][n][e / D] += not_finite(z) && kb + k < w.lim[n] && (SEE != SEE_TREE || (bits[n] >> k & 1))
                                                    ? bf16_to_f32(z) : 0.0f;
                }
            }
        }
    }
}

// LDS of one wave's state on its way to another: accumulators, sum, maximum.
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
// Row rho sees the keys up to first + rho / g, or all of them, or (trees) those before
// `first` and some of the others.  KW = NW: the
// workgroup's waves share the keys and join through LDS; KW = 1: each wave has an
// item of its own.  ALONG: the prefix's keys come before them.  AHEAD: the next
// block's keys are on their way while one is used.
template <int HD, int NT, int KW, int SEE, bool ALONG, bool AHEAD>
__device__ __forceinline__ void item(const Args& a, float* lds, const int32_t* table, int head, int row0, int tile0,
                                     int n_rows, int first, int end, int k0, int chunk, int slot) {
    constexpr int KK = HD / 32, D = HD / 16;
    const int lane = threadIdx.x & 63, g = lane >> 4, c = lane & 15;
    const int wave = KW == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    auto seen = [&](int rho) { return SEE == SEE_CAUSAL ? (int)min((int64_t)first + 1 + rho / a.g, (int64_t)end) : end; };
    // keys that some row of the tile sees, and that all do
    const int any = uniform(a.n_pages > 0 ? min(seen(min(tile0 + 16 * NT, n_rows) - 1), k0 + chunk) : 0);
    const int all = uniform(min(SEE == SEE_TREE ? first : seen(tile0), any));
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
        if constexpr (SEE == SEE_TREE) {
            w.mask[n] = a.mask + (live[n] ? row[n] : row0) * a.words;
            w.mask0[n] = *w.mask[n];
        }
        const uint16_t* p = a.q + row[n] * a.ldq + hh[n] * HD + 8 * g;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            u32x4 x = {0, 0, 0, 0};
            if (live[n]) x = *reinterpret_cast<const u32x4*>(p + 32 * kk);
            w.q[n][kk] = __builtin_bit_cast(bf16x8, x);
        }
    }
    // The blocks kb, kb + KB KW, .. of one table.
    auto walk = [&](auto see, const int32_t* tab, int kb, int end_k, int all_k) __attribute__((always_inline)) {
        constexpr int C = decltype(see)::value;
        Keys<HD> x, y;
        if (AHEAD && kb < end_k) x.load(a, tab, head, kb, end_k, lane);
        auto step = [&](Keys<HD>& now, Keys<HD>& next) __attribute__((always_inline)) {
            const int nb = kb + KB * KW;
            if (!AHEAD) now.load(a, tab, head, kb, end_k, lane);
            else if (nb < end_k) next.load(a, tab, head, nb, end_k, lane);
            block<HD, NT, C>(w, a, now, tab, head, kb, end_k, first, kb + KB > all_k || !now.there[0] || !now.there[1], lane);
            kb = nb;
        };
#pragma unroll 1
        while (kb < end_k) {
            step(x, y);
            if (AHEAD && kb < end_k) step(y, x);
        }
    };
    int turn = wave;                                    // whose block is the first
    if constexpr (ALONG) {
        const int end_p = a.n_pages > 0 ? a.prefix : 0;
        int lim[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            lim[n] = w.lim[n];
            w.lim[n] = live[n] ? end_p : 0;
        }
        walk(std::integral_constant<int, SEE_ALL>{}, a.prefix_table, KB * wave, end_p, end_p);
#pragma unroll
        for (int n = 0; n < NT; ++n) w.lim[n] = lim[n];
        turn = (wave + KW - (end_p + KB - 1) / KB % KW) % KW;
    }
    walk(std::integral_constant<int, SEE>{}, table, k0 + KB * turn, any, all);
    if constexpr (KW > 1) {
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
    }
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

// ---------------------------------------------------------------------------
// Many rows: a tile of 128, 32 to a wave, against keys staged in LDS
// ---------------------------------------------------------------------------
//
// Stages of 64 keys, double buffered, loaded straight into LDS while the stage
// before is used; wave w loads the w-th 16 keys, which lie in one page.  A wave
// multiplies with v_mfma_f32_32x32x16_bf16: S^T = K Q^T leaves a lane 32 scores of
// one row (lane l, register v: key 8 (v / 4) + 4 (l / 32) + v % 4 of 32, row l %
// 32), and registers 8 i .. 8 i + 7 are the 8 probabilities that the second
// product O^T += V^T P^T wants from that lane when V's rows come in the same
// order, which the transposing LDS reads give.

constexpr int WROWS = 32 * NW;            // rows of a wide tile
constexpr int STG = 64;                   // keys of a stage (32: 5 to 10 % slower)

// A stage's keys or values in LDS: [STG][HD] bf16, 16-byte chunk c of row r at chunk
// c ^ swz(r).  The swizzle gives 16 rows of one chunk, and four neighbouring rows of
// 64 bytes, all 64 banks once: the reads of the two products.
template <int HD>
struct KeyTile {
    static constexpr int NB = STG / 32, TILES = STG / 16;
    static constexpr int ROW = 2 * HD, BYTES = STG * ROW;
    static constexpr int CPR = HD / 8;                 // chunks per row
    static constexpr int RPI = 64 / CPR;               // rows of a 1 KB load
    static constexpr int RW = STG / NW;                // rows that a wave loads, in NL loads
    static constexpr int NL = RW / RPI;
    __device__ static __forceinline__ int swz(int row) {
        const int x = HD == 128 ? row & 15 : (row >> 1) & 7;
        return HD == 128 ? ((x & 3) << 2) | (x >> 2) : ((x & 1) << 2) | (x >> 1);
    }
    __device__ static __forceinline__ int off(int row, int chunk) { return row * ROW + ((chunk ^ swz(row)) << 4); }
    // Load j of a wave: where this lane reads, from the first byte of its tile of 16.
    __device__ static __forceinline__ uint32_t from(int j, int wave, int lane) {
        const int row = RW * wave % 16 + RPI * j + lane / CPR;
        return row * ROW + (((lane % CPR) ^ swz(row)) << 4);
    }
    // K operand, step i: elements 16 i + 8 (lane / 32) .. of row lane % 32.
    __device__ static __forceinline__ int key_at(int i, int lane) { return off(lane & 31, 2 * i + (lane >> 5)); }
    // V^T operand of output tile t: element 32 t + lane % 32 of the rows 4 (lane /
    // 32) .. + 3 (x = 0) or 8 more (x = 1).  In each 16-lane group lanes 4 q .. 4 q +
    // 3 point at row q, four consecutive elements each; lane i gets column i.
    __device__ static __forceinline__ int val_at(int t, int x, int lane) {
        const int g = lane >> 4, i = lane & 15;
        const int m = 32 * t + 16 * (g & 1) + 4 * (i & 3);
        return off(8 * x + 4 * (g >> 1) + (i >> 2), m >> 3) + (m & 7) * 2;
    }
};

__device__ __forceinline__ bf16x8 lds_frag(const char* p) { return *reinterpret_cast<const bf16x8*>(p); }
__device__ __forceinline__ bf16x8 lds_frag_tr(const char* p, const char* q) {
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr4_t)p);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr4_t)q);
    const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    return __builtin_bit_cast(bf16x8, v);
}
// Element of a 32-row accumulator register.
__device__ __forceinline__ int acc_row(int v, int hh) { return 8 * (v >> 2) + 4 * hh + (v & 3); }

template <int HD>
struct WideWave {
    bf16x8 q[HD / 16];
    f32x16 o[HD / 32];
    float m, l;                                        // l: of this lane's keys
    int lim;                                           // keys that this lane's row sees
    const uint64_t* mask;                              // trees: the row's mask, and its first word
    uint64_t mask0;
    int key[HD / 16], val[HD / 32][2];                 // LDS addresses within a tile
};

// The keys kb .. of a stage (K at kt, V behind it): one online-softmax step of this
// lane's row.  `part` (wave-uniform): some row does not see all of them; TREE: nor
// those whose bits are not set.
template <int HD, bool TREE>
__device__ __forceinline__ void wide_block(WideWave<HD>& w, const char* kt, int kb, uint32_t there, bool part, uint64_t bits,
                                           float c, int hh) {
    typedef KeyTile<HD> Tile;
    constexpr int NB = Tile::NB;
    f32x16 s[NB] = {};
#pragma unroll
    for (int i = 0; i < HD / 16; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = mfma32(lds_frag(kt + w.key[i] + 32 * b * Tile::ROW), w.q[i], s[b]);
    if (part) {
        const uint64_t mine = bits >> (4 * hh);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int lim = there >> (2 * b + x) & 1 ? w.lim - kb - 4 * hh : 0;
#pragma unroll
                for (int v = 8 * x; v < 8 * x + 8; ++v)
                    if (32 * b + acc_row(v, 0) >= lim || (TREE && !(mine >> (32 * b + acc_row(v, 0)) & 1))) s[b][v] = -INFINITY;
            }
    }
    float mb = -INFINITY;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < 16; v += 2) mb = fmaxf(fmaxf(mb, s[b][v]), s[b][v + 1]);
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(mb), __float_as_uint(mb), false, false);
    mb = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) * c;
    if (__ballot(mb > w.m + kSlack) != 0) {
        const float mn = fmaxf(w.m, mb);
        const float alpha = exp2_hw(w.m - mn);
        w.l *= alpha;
#pragma unroll
        for (int t = 0; t < HD / 32; ++t) w.o[t] *= alpha;
        w.m = mn;
    }
    const char* vt = kt + Tile::BYTES;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float x = exp2_hw(fmaf(s[b][8 * i + 2 * j], c, -w.m)), y = exp2_hw(fmaf(s[b][8 * i + 2 * j + 1], c, -w.m));
                w.l += x + y;
                f[j] = pack_bf16x2(x, y);
            }
            const bf16x8 p = __builtin_bit_cast(bf16x8, f);
            const char* v0 = vt + (32 * b + 16 * i) * Tile::ROW;
#pragma unroll
            for (int t = 0; t < HD / 32; ++t) w.o[t] = mfma32(lds_frag_tr(v0 + w.val[t][0], v0 + w.val[t][1]), p, w.o[t]);
        }
}

// LDS of two stages of keys and values, and their flags.
template <int HD>
constexpr int kWideBytes = 4 * KeyTile<HD>::BYTES + 16;

// item() for a tile of 128 rows: the same rows, keys and results.
template <int HD, int SEE, bool ALONG>
__device__ __forceinline__ void wide_item(const Args& a, char* lds, const int32_t* table, int head, int row0, int tile0,
                                          int n_rows, int first, int end, int k0, int chunk, int slot) {
    typedef KeyTile<HD> Tile;
    constexpr int B = Tile::BYTES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), hh = lane >> 5;
    auto seen = [&](int rho) { return SEE == SEE_CAUSAL ? (int)min((int64_t)first + 1 + rho / a.g, (int64_t)end) : end; };
    const int rho = tile0 + 32 * wave + (lane & 31), t = rho / a.g;
    const bool live = rho < n_rows;
    const int64_t row = row0 + t;
    const int h = head * a.g + (rho - t * a.g);
    WideWave<HD> w;
    w.m = kNone;
    w.l = 0.0f;
    w.lim = live ? seen(rho) : 0;
    if constexpr (SEE == SEE_TREE) {
        w.mask = a.mask + (live ? row : (int64_t)row0) * a.words;
        w.mask0 = *w.mask;
    }
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) {
        w.o[i] = f32x16{};
        w.val[i][0] = Tile::val_at(i, 0, lane);
        w.val[i][1] = Tile::val_at(i, 1, lane);
    }
    const uint16_t* qp = a.q + row * a.ldq + h * HD + 8 * hh;
#pragma unroll
    for (int i = 0; i < HD / 16; ++i) {
        u32x4 x = {0, 0, 0, 0};
        if (live) x = *reinterpret_cast<const u32x4*>(qp + 16 * i);
        w.q[i] = __builtin_bit_cast(bf16x8, x);
        w.key[i] = Tile::key_at(i, lane);
    }
    uint32_t from[Tile::NL];
#pragma unroll
    for (int j = 0; j < Tile::NL; ++j) from[j] = Tile::from(j, wave, lane);
    const int w0 = tile0 + 32 * wave;
    // the last stage of each buffer that held values that are not finite
    int* odd = reinterpret_cast<int*>(lds + 4 * B);
    // The next stage has landed, and every wave has left this one.
    auto turn = [&]() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    // The keys k0 .. of one table: the tile's last row sees those up to `any`, its
    // first those up to `all`; this wave's rows up to w_any and w_all.
    auto walk = [&](auto see, const int32_t* table, int k0, int any, int all, int w_any, int w_all)
                    __attribute__((always_inline)) {
        constexpr int C = decltype(see)::value;
        const int n = any > k0 ? (any - k0 + STG - 1) / STG : 0;

        // The pages of stage i's tiles of 16, looked up a turn before they are used.
        int page[Tile::TILES] = {};
        auto look = [&](int i) __attribute__((always_inline)) {
            const int kb = k0 + STG * i;
            if (1 << a.lg_page >= STG) {                   // the stage lies in one page
                const int p = page_of(a, table, kb, any);
#pragma unroll
                for (int x = 0; x < Tile::TILES; ++x) page[x] = p;
            } else {
#pragma unroll
                for (int x = 0; x < Tile::TILES; ++x) page[x] = page_of(a, table, kb + 16 * x, any);
            }
        };
        constexpr uint32_t ALL = (1u << Tile::TILES) - 1;
        // Stage i into the buffer at `to`: keys from `any` on and missing pages arrive as
        // zeros (they lie past the descriptor's range).  Returns the pages that are there.
        auto load = [&](int i, char* to) __attribute__((always_inline)) -> uint32_t {
            uint32_t there = 0;
            int mine = page[0];
#pragma unroll
            for (int x = 0; x < Tile::TILES; ++x) {
                there |= (uint32_t)in_cache(a, page[x]) << x;
                if (x == Tile::RW * wave / 16) mine = page[x];
            }
            const int kb = k0 + STG * i + (Tile::RW * wave & ~15), rows = rows_in(in_cache(a, mine), kb, any);
            const int64_t at = row_of(a, mine, head, kb);
            to += Tile::RW * wave * Tile::ROW;
            const auto rk = rows_of<HD>(a.K, at, rows), rv = rows_of<HD>(a.V, at, rows);
#pragma unroll
            for (int j = 0; j < Tile::NL; ++j) {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lptr_t)(to + 1024 * j), 16, from[j], 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lptr_t)(to + B + 1024 * j), 16, from[j], 0, 0, 0);
            }
            return there;
        };
        uint32_t there = 0, next = 0;
        // Stage i from one buffer while the next is loaded into the other: the
        // __restrict parameters say that they don't overlap (without them the compiler
        // waits for the loads in flight before the first read).
        auto step = [&](char* __restrict to, char* __restrict kt, int i) __attribute__((always_inline)) {
            const int kb = k0 + STG * i;
            next = i + 1 < n ? load(i + 1, to) : 0;
            // A key that some row of the tile sees and another does not must not reach
            // the second by 0 * inf: values that are not finite leave the product,
            // and go to the rows that see them by themselves.
            const bool mixed = C != SEE_ALL && kb + STG > all;
            if (mixed) {
                char* mine = kt + B + Tile::RW * wave * Tile::ROW + 16 * lane;
                uint32_t any_odd = 0;
#pragma unroll
                for (int j = 0; j < Tile::NL; ++j) {
                    u32x4 x = *reinterpret_cast<const u32x4*>(mine + 1024 * j);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        any_odd |= not_finite2(x[e]);
                        x[e] = finite2(x[e]);
                    }
                    *reinterpret_cast<u32x4*>(mine + 1024 * j) = x;
                }
                if (any_odd) odd[i & 1] = i;
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            }
            const bool part = kb + STG > w_all || there != ALL;
            const uint64_t bits = C == SEE_TREE && part ? tree_bits(w.mask, w.mask0, a.words, kb - first) : ~uint64_t(0);
            if (kb < w_any) wide_block<HD, C == SEE_TREE>(w, kt, kb, there, part, bits, a.c, hh);
            if (mixed && odd[i & 1] == i) {
#pragma unroll 1
                for (int k = 0; k < min(STG, any - kb); ++k) {
                    if (!(there >> (k / 16) & 1)) continue;
                    const uint16_t* x = a.V + row_of(a, page_of(a, table, kb + k, any), head, kb + k) * HD;
#pragma unroll
                    for (int u = 0; u < HD / 32; ++u)
#pragma unroll
                        for (int v = 0; v < 16; ++v) {
                            const uint32_t y = x[32 * u + acc_row(v, hh)];
                            w.o[u][v] += not_finite(y) && kb + k < w.lim && (C != SEE_TREE || (bits >> k & 1)) ? bf16_to_f32(y) : 0.0f;
                        }
                }
            }
            there = next;
            if (i + 2 < n) look(i + 2);
        };
        if (threadIdx.x < 2) odd[threadIdx.x] = -1;
        if (n > 0) {
            look(0);
            there = load(0, lds);
            if (n > 1) look(1);
        }
        turn();
        // The queries have arrived, too; said in a way that the compiler sees, or it
        // waits for "them" (and so for the next stage) in every turn of the loop.
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) asm volatile("" : "+v"(w.q[i]));
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            step(lds + 2 * B * ((i + 1) & 1), lds + 2 * B * (i & 1), i);
            turn();
        }
    };
    if constexpr (ALONG) {
        const int end_p = uniform(a.n_pages > 0 ? a.prefix : 0), w_end = w0 < n_rows ? end_p : 0;
        const int lim = w.lim;
        w.lim = live ? end_p : 0;
        walk(std::integral_constant<int, SEE_ALL>{}, a.prefix_table, 0, end_p, end_p, w_end, w_end);
        w.lim = lim;
    }
    {
        const int any = uniform(a.n_pages > 0 ? min(seen(min(tile0 + WROWS, n_rows) - 1), k0 + chunk) : 0);
        const int all = uniform(min(SEE == SEE_TREE ? first : seen(tile0), any));
        const int w_any = uniform(w0 < n_rows ? min(seen(min(w0 + 32, n_rows) - 1), any) : 0);
        const int w_all = uniform(w0 < n_rows ? min(SEE == SEE_TREE ? first : seen(w0), any) : 0);
        walk(std::integral_constant<int, SEE>{}, table, k0, any, all, w_any, w_all);
    }
    // Lane (hh, row) has the elements 32 u + 8 j + 4 hh .. + 3 in o[u][4 j ..].  They go
    // out by way of LDS, a region for each wave, so that a store covers whole rows:
    // four elements at chunk c of row r lie at chunk c ^ (r % 16).
    constexpr int CH = HD / 4, RS = 64 / CH;           // chunks of a row, rows of a store
    float l = w.l + __shfl_xor(w.l, 32);
    f32x4* mine = reinterpret_cast<f32x4*>(lds) + 32 * CH * wave;
    const int rr = lane & 31;
    const float scale = a.direct ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
#pragma unroll
    for (int u = 0; u < HD / 32; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            mine[CH * rr + ((8 * u + 2 * j + hh) ^ (rr & 15))] =
                f32x4{w.o[u][4 * j], w.o[u][4 * j + 1], w.o[u][4 * j + 2], w.o[u][4 * j + 3]} * scale;
    const int64_t id = row * a.hq + h;
    if (live && hh == 0) {
        if (!a.direct) *reinterpret_cast<float2*>(a.ml + 2 * (slot * a.rows + id)) = make_float2(w.m, l);
        else if (a.lse) a.lse[h * a.T + row] = l == 0.0f ? -INFINITY : (w.m + log2f(l)) * kLn2;
    }
    const int c = lane % CH;
#pragma unroll
    for (int i = 0; i < 32; i += RS) {
        const int r = i + lane / CH;
        if (w0 + r >= n_rows) continue;
        const f32x4 x = mine[CH * r + (c ^ (r & 15))];
        const int t = (w0 + r) / a.g, hd = head * a.g + (w0 + r - t * a.g);
        if (a.direct)
            *reinterpret_cast<u32x2*>(a.out + (row0 + t) * a.ldo + hd * HD + 4 * c) =
                u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
        else
            *reinterpret_cast<f32x4*>(a.part + (slot * a.rows + (int64_t)(row0 + t) * a.hq + hd) * HD + 4 * c) = x;
    }
}

// Kinds of tiles: 16 or 32 rows whose keys a workgroup's waves share (ONE, TWO); 128
// rows against keys in LDS (WIDE); for trees 64 rows as ONE and TWO, too (FOUR).  On the
// requests' own keys, where each has one token, all rows of a tile see the same: ONE
// becomes FLAT, or SOLO with a tile to a wave.
// Behind a short prefix there are no tiles for it: each request's own items take its
// keys ALONG, and nothing is left to join.
enum Kind : int { ONE = 1, TWO = 2, SOLO = 3, FLAT = 4, ALONG = 5, FOUR = 6, WIDE = 8 };
constexpr int kind_rows(int k) { return k == SOLO || k == FLAT ? 16 : k == FOUR ? 64 : 16 * k; }
// Parts of `chunk` keys that a request of `end` own tokens has.
__device__ __forceinline__ int parts_of(const Args& a, int end, int chunk) {
    return a.splits_s > 0 ? min((end + chunk - 1) / chunk, a.splits_s) : 0;
}

// Tile `tile` of unit `unit` (a head and a part of the keys) from turn b of a range
// whose tiles of a unit read the same keys.  Workgroups go to the XCDs in turn, each
// of which has an L2 of its own: a unit's tiles are eight turns apart.  False past
// the last unit.
struct Turn {
    int64_t unit;
    int tile;
};
__device__ __forceinline__ Turn turn_of(int64_t b, int tiles) {
    const int64_t j = b >> 3;
    return {j / tiles * 8 + (b & 7), (int)(j % tiles)};
}
// Turns that `units` units of `tiles` tiles take.
__host__ __device__ constexpr int64_t turns(int64_t units, int tiles) { return tiles == 1 ? units : (units + 7) / 8 * 8 * tiles; }

// An item where the lengths decide (tiles of 128 rows of trees).  Every workgroup reads
// the lengths of all requests, at most 256, a wave's lanes four each, and comes to the
// same list: parts as long as gives a.slots workgroups, what they all do shared out
// evenly, with the half part that each tile ends with on the average, and no shorter
// than leaves the longest request as many as the workspace has room for; then the
// requests' items one after the other, a unit's tiles eight turns apart (turn_of).  So
// no workgroup is spent on parts that are not there, and max_kv decides how many parts
// there may be, not where they end (8 requests of up to 32000 keys, 64 nodes, 32 heads
// over 8 of 128: 166 us under a max_kv of 2^20, too, where 19 parts of it took 680).
constexpr int kCounted = 256;
constexpr int64_t kTreeOwn = 8;            // blocks of KB keys that such a part has at the least
struct Counted {
    int r, head, split, tile, chunk;       // r < 0: past the last item
};
__device__ __forceinline__ Counted counted_item(const Args& a, int64_t turn) {
    constexpr int PER = kCounted / 64;
    const int lane = threadIdx.x & 63;
    int tiles[PER], end[PER], all = 0, longest = 0;
    int64_t work = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const int r = PER * lane + q;
        const Span s = span_of(a, min(r, a.n_req - 1));
        tiles[q] = r < a.n_req ? (s.n * a.g + WROWS - 1) / WROWS : 0;
        end[q] = s.end;
        all += tiles[q];
        longest = max(longest, tiles[q] > 0 ? s.end : 0);
        work += (int64_t)tiles[q] * ((s.end + STG - 1) / STG);
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        work += __shfl_xor(work, d);
        all += __shfl_xor(all, d);
        longest = max(longest, __shfl_xor(longest, d));
    }
    work = uniform64(work) * a.hk + a.work_p;
    const int64_t parts = max(a.slots - (int64_t)uniform(all) * a.hk / 2, (int64_t)a.slots / 2);
    Counted c;
    const int least = max(((uniform(longest) + a.splits_s - 1) / a.splits_s + STG - 1) / STG * STG, a.chunk_s);
    c.chunk = (int)min(max((work + parts - 1) / parts * STG, (int64_t)least), (int64_t)1 << 30);
    int64_t items[PER], mine = 0;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const int units = parts_of(a, end[q], c.chunk) * a.hk;
        items[q] = turns(units, tiles[q]);
        mine += items[q];
    }
    int64_t upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t x = __shfl_up(upto, d);
        if (lane >= d) upto += x;
    }
    c.r = -1;
    int64_t at = upto - mine;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
        const uint64_t hit = __ballot(turn >= at && turn < at + items[q]);
        if (hit != 0) {
            const int l = __builtin_ctzll(hit);
            const int n = __builtin_amdgcn_readlane(tiles[q], l);
            const int units = parts_of(a, __builtin_amdgcn_readlane(end[q], l), c.chunk) * a.hk;
            const int64_t j = turn - uniform64(__shfl(at, l));
            const Turn t = n == 1 ? Turn{j, 0} : turn_of(j, n);
            if (t.unit < units) {
                c.r = PER * l + q;
                c.tile = t.tile;
                c.head = (int)t.unit % a.hk;
                c.split = (int)t.unit / a.hk;
            }
        }
        at += items[q];
    }
    return c;
}

template <int HD, int N>
constexpr int kLdsBytes = N == WIDE ? kWideBytes<HD> : (N == SOLO || N == ALONG ? 16 : 8 * kStateFloats<HD, kind_rows(N) / 16>);

// AHEAD costs registers: heads of 128 with 32 rows have none to spare, and beside
// wide tiles, which leave two workgroups a CU, the plain loop is faster (64 requests
// behind 32768 tokens 101 us against 114, 200 of 32 heads 123 against 140; one request
// behind 100 tokens 4.9 against 4.7, behind 1024 8.7 against 7.8).
template <int HD, int N, int NP>
constexpr bool kAhead = NP != WIDE && !(HD == 128 && N == TWO) && N != FOUR;

template <int HD, int N, int NP, int SEE>
__device__ __forceinline__ void any_item(const Args& a, char* lds, const int32_t* table, int head, int row0, int tile0,
                                         int n_rows, int first, int end, int k0, int chunk, int slot) {
    constexpr bool ALONG_P = NP == ALONG;
    if constexpr (N == WIDE)
        wide_item<HD, SEE, ALONG_P>(a, lds, table, head, row0, tile0, n_rows, first, end, k0, chunk, slot);
    else if constexpr (N == SOLO)
        item<HD, 1, 1, SEE_ALL, false, kAhead<HD, N, NP>>(a, nullptr, table, head, row0, tile0, n_rows, 0, min(first + 1, end), k0, chunk, slot);
    else if constexpr (N == FLAT)
        item<HD, 1, NW, SEE_ALL, ALONG_P, kAhead<HD, N, NP>>(a, reinterpret_cast<float*>(lds), table, head, row0, tile0, n_rows, 0, min(first + 1, end), k0,
                               chunk, slot);
    else
        item<HD, kind_rows(N) / 16, NW, SEE, ALONG_P, kAhead<HD, N, NP>>(a, reinterpret_cast<float*>(lds), table, head, row0, tile0, n_rows, first, end, k0, chunk, slot);
}

// NP, NS: kinds of the tiles on the prefix and on the requests' own keys.
// SEE: causal, or trees.  COUNTED: the own keys are cut by the lengths.  Wide tiles of trees
// at heads of 64 are held to 128 registers, four waves a SIMD (COUNTED at the price of two
// registers spilled, 12 bytes of scratch a lane).
template <int HD, int NP, int NS, int SEE, bool COUNTED>
__global__ __launch_bounds__(NTHR, (SEE == SEE_TREE && HD == 64 && NS == WIDE ? 4 : NP == WIDE || NS == WIDE || NS == FOUR ? 2 : 1)) void prefix_attn_kernel(const Args a) {
    constexpr int LDS = kLdsBytes<HD, NP> > kLdsBytes<HD, NS> ? kLdsBytes<HD, NP> : kLdsBytes<HD, NS>;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    const int64_t at = a.base + blockIdx.x;
    if (NP != ALONG && at < a.items_p) {
        const Turn t = a.tiles_p == 1 ? Turn{at, 0} : turn_of(at, a.tiles_p);
        if (t.unit >= a.units_p) return;
        const int tile = t.tile, head = (int)t.unit % a.hk, split = (int)t.unit / a.hk;
        // rows of the batch up to the last that holds a token
        const int64_t hi = a.start ? min(max((int64_t)entry(a.start, a.n_req), (int64_t)0), a.T) : min((int64_t)a.n_req, a.T);
        const int tile0 = tile * kind_rows(NP), n_rows = (int)hi * a.g;
        if constexpr (NP != ALONG)
            if (tile0 < n_rows)
                any_item<HD, NP, NP, SEE_ALL>(a, lds, a.prefix_table, head, 0, tile0, n_rows, 0, a.prefix, split * a.chunk_p,
                                        a.chunk_p, split);
    } else {
        int64_t b = at - a.items_p;
        if constexpr (COUNTED) {
            const Counted c = counted_item(a, b);
            if (b == 0 && threadIdx.x == 0) *a.chunk = c.chunk;
            if (c.r < 0) return;
            const Span s = span_of(a, c.r);
            any_item<HD, NS, NP, SEE>(a, lds, a.table + c.r * a.max_pages, c.head, s.row, c.tile * kind_rows(NS), s.n * a.g, s.first,
                                   s.end, c.split * c.chunk, c.chunk, a.splits_p + c.split);
            return;
        }
        if constexpr (NS == SOLO) b = b * NW + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        Turn t = a.tiles_s == 1 ? Turn{b, 0} : turn_of(b, a.tiles_s);
        if (NS == WIDE && a.n_req == 1) {
            // One prompt: its last tiles see most keys and go first, those of all heads
            // before the next (2000 tokens, 32 heads of 64: 46 us against 53; 8000, 8 heads:
            // 112 against 123).  Of several requests such tiles may be empty, and a
            // unit's tiles too far apart to share L2 (135 against 100).
            const int64_t units = (a.units_s + 7) / 8 * 8;
            t = {b % units, a.tiles_s - 1 - (int)(b / units)};
        }
        if (t.unit >= a.units_s) return;
        const int tile = t.tile, head = (int)(t.unit % a.hk);
        b = t.unit / a.hk;
        const int split = (int)(b % a.splits_s), r = (int)(b / a.splits_s);
        const Span s = span_of(a, r);
        const int tile0 = tile * kind_rows(NS), n_rows = s.n * a.g;
        if (tile0 < n_rows && (a.direct || split < parts_of(a, s.end, a.chunk_s)))
            any_item<HD, NS, NP, SEE>(a, lds, a.table + r * a.max_pages, head, s.row, tile0, n_rows, s.first, s.end,
                                   split * a.chunk_s, a.chunk_s, a.splits_p + split);
    }
}

// Workgroups of the wide kernels that the chip holds at once (two a CU at heads of 128,
// four at 64).
constexpr int64_t full_chip(int hd) { return hd == 128 ? 512 : 1024; }
// Whether a launch for trees cuts the own keys by the lengths: wide tiles, fewer than
// fill half of the chip, and as many requests as a workgroup counts in a few loads.
inline bool counts_lengths(const PrefixAttnShape& sh, int kind, int tiles) {
    return kind == WIDE && sh.n_req <= kCounted && sh.n_req * tiles * sh.hk < full_chip(sh.hd) / 2;
}

inline Args args_of(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t) {
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
    a.units_p = (int64_t)p.splits_p * sh.hk;
    a.units_s = sh.n_req * p.splits_s * sh.hk;
    a.items_p = turns(a.units_p, p.tiles_p);
    a.blocks = a.items_p + (p.kind_s == SOLO ? (a.units_s + NW - 1) / NW : turns(a.units_s, p.tiles_s));
    a.direct = p.direct;
    a.mask = t.mask;
    a.words = (int)((sh.max_new + 63) / 64);
    a.slots = t.mask && p.splits_s > 1 && counts_lengths(sh, p.kind_s, p.tiles_s) ? (int)full_chip(sh.hd) : 0;
    // parts as counted_item cuts them are at most the slots and one for each tile, and a
    // request's units are filled up to whole rounds of eight
    const int64_t base_s = sh.n_req * p.tiles_s * sh.hk;
    if (a.slots > 0 && a.chunk_s > kTreeOwn * KB) a.chunk_s = kTreeOwn * KB;
    if (a.slots > 0) a.blocks = a.items_p + a.slots + base_s + (p.tiles_s > 1 ? 8 * sh.n_req * p.tiles_s : 0);
    a.work_p = a.units_p / (p.splits_p > 0 ? p.splits_p : 1) * p.tiles_p * ((sh.prefix + STG - 1) / STG);
    a.chunk = reinterpret_cast<int32_t*>(a.part ? a.part + n * sh.hd : nullptr);
    a.c = (float)(sh.scale * (double)kLog2e);
    return a;
}

}  // namespace
}  // namespace cola
