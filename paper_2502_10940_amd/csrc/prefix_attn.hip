// prefix_attn.hip -- cola_prefix_attn: the plan of a call, its launches, and the
// launch that joins the parts of the keys.  The kernels are in prefix_attn.hpp.
#include "prefix_attn.hpp"

namespace cola {
namespace {

// The parts of each row joined, in their order, where they are few: a thread for
// four elements of a row, kFew parts in flight.
constexpr int kFew = 4;
template <int HD>
__global__ __launch_bounds__(NTHR) void prefix_join_few_kernel(const Args a) {
    constexpr int TPR = HD / 4;
    const int e = 4 * (threadIdx.x % TPR);
    for (int r = blockIdx.y; r < a.n_req; r += gridDim.y) {
        const Span s = span_of(a, r);
        const int parts = a.splits_p + parts_of(a, s.end, a.slots > 0 ? entry(a.chunk, 0) : a.chunk_s);
        for (int64_t j = (int64_t)blockIdx.x * (NTHR / TPR) + threadIdx.x / TPR; j < (int64_t)s.n * a.hq;
             j += (int64_t)gridDim.x * (NTHR / TPR)) {
            const int64_t id = (int64_t)s.row * a.hq + j;
            float M = kNone, l = 0.0f;
            f32x4 o = {0, 0, 0, 0};
            for (int p0 = 0; p0 < parts; p0 += kFew) {
                float2 x[kFew];
                f32x4 y[kFew];
                float m = M;
#pragma unroll
                for (int i = 0; i < kFew; ++i) {
                    x[i] = make_float2(kNone, 0.0f);
                    y[i] = f32x4{0, 0, 0, 0};
                    if (p0 + i < parts) {
                        x[i] = *reinterpret_cast<const float2*>(a.ml + 2 * ((p0 + i) * a.rows + id));
                        y[i] = *reinterpret_cast<const f32x4*>(a.part + ((p0 + i) * a.rows + id) * HD + e);
                    }
                    m = fmaxf(m, x[i].x);
                }
                const float f = exp2_hw(M - m);
                l *= f;
                o *= f;
                M = m;
#pragma unroll
                for (int i = 0; i < kFew; ++i) {
                    const float g = exp2_hw(x[i].x - m);
                    l += g * x[i].y;
                    o += g * y[i];
                }
            }
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const uint32_t t = (uint32_t)id / (uint32_t)a.hq, h = (uint32_t)id - t * (uint32_t)a.hq;
            *reinterpret_cast<u32x2*>(a.out + (int64_t)t * a.ldo + h * HD + e) =
                u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
            if (a.lse && e == 0) a.lse[h * a.T + t] = l == 0.0f ? -INFINITY : (M + log2f(l)) * kLn2;
        }
    }
}

// The same where they are many: a wave to a row.  Lane p holds the
// statistics of parts p and p + 64 (there are at most 128) and forms their
// weights; then LP lanes take four elements each of every 64 / LP-th part.
template <int HD>
__global__ __launch_bounds__(NTHR) void prefix_join_kernel(const Args a) {
    constexpr int LP = HD / 4, PP = 64 / LP;           // lanes of a part, parts at once
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int sub = lane / LP, e = 4 * (lane % LP);
    for (int r = blockIdx.y; r < a.n_req; r += gridDim.y) {
        const Span s = span_of(a, r);
        const int parts = a.splits_p + parts_of(a, s.end, a.slots > 0 ? entry(a.chunk, 0) : a.chunk_s);
        for (int64_t j = (int64_t)blockIdx.x * NW + wave; j < (int64_t)s.n * a.hq; j += (int64_t)gridDim.x * NW) {
            const int64_t id = (int64_t)s.row * a.hq + j;
            float m[2] = {kNone, kNone}, l[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (lane + 64 * i < parts) {
                    const float2 x = *reinterpret_cast<const float2*>(a.ml + 2 * ((lane + 64 * i) * a.rows + id));
                    m[i] = x.x;
                    l[i] = x.y;
                }
            float M = fmaxf(m[0], m[1]);
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
            const float f[2] = {exp2_hw(m[0] - M), exp2_hw(m[1] - M)};
            float L = f[0] * l[0] + f[1] * l[1];
#pragma unroll
            for (int d = 32; d >= 1; d >>= 1) L += __shfl_xor(L, d);
            f32x4 o = {0, 0, 0, 0};
            const float* from = a.part + id * HD + e;
            for (int p0 = 0; p0 < parts; p0 += 4 * PP) {
                f32x4 x[4];
                float y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int p = p0 + i * PP + sub;
                    const float lo = __shfl(f[0], p & 63), hi = __shfl(f[1], p & 63);
                    y[i] = p < 64 ? lo : hi;
                    x[i] = f32x4{0, 0, 0, 0};
                    if (p < parts) x[i] = *reinterpret_cast<const f32x4*>(from + p * a.rows * HD);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (p0 + i * PP + sub < parts) o += y[i] * x[i];
            }
#pragma unroll
            for (int d = 32; d >= LP; d >>= 1)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += __shfl_xor(o[i], d);
            const float inv = L == 0.0f ? 0.0f : 1.0f / L;
            const int64_t t = id / a.hq, h = id - t * a.hq;
            if (sub == 0)
                *reinterpret_cast<u32x2*>(a.out + t * a.ldo + h * HD + e) =
                    u32x2{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv)};
            if (a.lse && lane == 0) a.lse[h * a.T + t] = L == 0.0f ? -INFINITY : (M + log2f(L)) * kLn2;
        }
    }
}

template <int HD>
hipError_t go(const PrefixAttnPlan& p, const Args& a, unsigned grid, hipStream_t s) {
#define COLA_GO(P, S) \
    if (p.kind_p == P && p.kind_s == S) prefix_attn_kernel<HD, P, S, SEE_CAUSAL, false><<<grid, NTHR, 0, s>>>(a)
    COLA_GO(ALONG, ONE);
    else COLA_GO(ALONG, TWO);
    else COLA_GO(ALONG, FLAT);
    else COLA_GO(ALONG, WIDE);
    else COLA_GO(ONE, ONE);
    else COLA_GO(ONE, FLAT);
    else COLA_GO(ONE, SOLO);
    else COLA_GO(TWO, ONE);
    else COLA_GO(TWO, FLAT);
    else COLA_GO(TWO, TWO);
    else COLA_GO(WIDE, ONE);
    else COLA_GO(WIDE, FLAT);
    else COLA_GO(WIDE, SOLO);
    else COLA_GO(WIDE, TWO);
    else COLA_GO(WIDE, WIDE);
    else return hipErrorInvalidValue;
#undef COLA_GO
    return hipGetLastError();
}

// Batches of so many (request, key head) pairs keep the chip busy with a wave to
// each: 200 requests of 32 heads 97 us against 105 with four waves to a pair; 1024
// pairs 36 us against 23, 512 pairs of 2000 keys 79 against 67.
constexpr int64_t kSoloItems = 4096;
// Parts up to which a thread reads all of a row's four elements (2 to 8 parts: the
// same time as a wave to a row, or less; 3 parts of 70112 rows 13 us against 83).
constexpr int64_t kJoinFew = 8;
// Threads of that kind from which on parts don't matter: those that a loose max_kv
// allows and no request has cost a wave to a row its 64 lanes (16 chunks of up to 256,
// 32 heads of 64, behind 4096 + 1000 keys, 12 parts allowed and 2 there: 142 us against
// 218 in all; 16 requests of up to 4000 keys, 21 allowed, 3 there: 68 against 91), and
// 16 that are there take as long either way (128 requests behind 60000 keys, 32 heads
// of 128: 156 and 159).
constexpr int64_t kJoinThreads = 1 << 17;
// Keys that a request's item takes along at most, and bytes of prefix that all
// requests read again.  One request of 8 heads of 64 with 200 keys of its own: 5.1
// us against 8.0 behind 64 keys, 7.4 against 8.1 behind 512, 10.0 against 8.5 behind
// 1024; 64 requests: 9.4 against 12.1 at 34 MB, 12.0 against 12.4 at 67 MB.
constexpr int64_t kAlongKeys = 640, kAlongBytes = 40000000;
// The same of tiles of 128 rows, whose partial rows are more.  64 requests with 64
// queries of 16 heads over 2, 256 + 256 keys: 18.3 us against 37.6; of 16 over 4, 200
// + 700 keys: 27.9 against 39.0; of 8 heads of 128, 512 + 64 keys, 134 MB: 25.1
// against 31.9.  1000 + 100 keys take 23.0 against 18.2, 512 + 1000 keys 32.1 against
// 28.8.
constexpr int64_t kWideAlongKeys = 1024, kWideAlongBytes = 150000000;
constexpr int64_t kWideOwn = 48;           // blocks of KB own keys in a part of several requests' chunks
constexpr int64_t kWideOwnBytes = 128000000;  // of partial rows, where these parts are more than the chip needs
constexpr int64_t kWideOwnTurns = 1 << 16;   // workgroups up to which there are such parts: 1.3 ns for each that has no rows
constexpr int64_t kPrefixOwn = 32;         // least blocks of a part of the prefix that is cut against a loose max_kv
constexpr int64_t kMaxGrid = 1 << 23;      // workgroups (2^32 threads are the limit)
constexpr int kRound = 64;                 // parts end where a stage of any kernel does
// Trees of heads of 64 have one more kind, 64 rows in registers, where tiles are few: its
// waves share the keys, so that a tile takes a fourth of the turns (one request of 60
// nodes and 300 keys, 8 heads: 10.2 us against 12.9 in a tile of 128; two of 3000 keys 14.7
// against 18.6; 8 of up to 40 nodes over 8000 keys, 16 heads, 41.0 against 39.8; 24 of up to
// 48 over 1500, 32 heads, 37.5 against 34.2).
constexpr int64_t kFourTiles = 64;
int kind_of(int64_t rows, bool four) {
    if (rows <= 32) return rows <= 16 ? ONE : TWO;
    return four && rows <= 64 ? FOUR : WIDE;
}
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

PrefixAttnPlan plan_of(const PrefixAttnShape& sh, bool tree) {
    PrefixAttnPlan p{};
    const int64_t g = sh.hq / sh.hk;
    const int64_t new_rows = sh.max_new < sh.T ? sh.max_new : sh.T;
    p.rows = sh.T * sh.hq;
    p.kind_s = kind_of(new_rows * g, tree && sh.hd == 64 && sh.n_req * sh.hk <= kFourTiles);
    p.kind_p = kind_of(sh.T * g, p.kind_s == FOUR);   // never below kind_s
    p.tiles_p = (int)ceil_div(sh.T * g, kind_rows(p.kind_p));
    p.tiles_s = (int)ceil_div(new_rows * g, kind_rows(p.kind_s));
    if (p.kind_s == ONE && sh.max_new == 1 && !tree)
        p.kind_s = sh.n_req * sh.hk >= kSoloItems && (sh.prefix == 0 || p.kind_p == WIDE) ? SOLO : FLAT;
    // without a prefix, the kernel whose prefix part asks for least
    if (sh.prefix == 0) p.kind_p = p.kind_s == TWO || p.kind_s == FOUR || p.kind_s == WIDE ? p.kind_s : ONE;
    // Short prefixes and few requests: the prefix's bytes come from L2 for each of them,
    // which costs less than a launch that joins.
    auto along = [&](bool wide) {
        return sh.prefix > 0 && sh.prefix + sh.max_kv <= (wide ? kWideAlongKeys : kAlongKeys) && p.kind_s != SOLO &&
               sh.n_req * p.tiles_s * sh.prefix * sh.hk * sh.hd * 4 <= (wide ? kWideAlongBytes : kAlongBytes);
    };
    // FOUR beside wide tiles of a prefix leaves its kernel half the waves (24 trees of up to
    // 48 nodes behind 2048 tokens, 32 heads: 62.7 us against 59.9)
    if (p.kind_s == FOUR && p.kind_p == WIDE && !along(false)) p.kind_s = WIDE;
    const bool wide = p.kind_s == WIDE;
    if (along(wide)) {
        p.kind_p = ALONG;
        p.tiles_p = 1;
        p.chunk_p = kRound;
        p.splits_s = 1;
        p.chunk_s = ceil_div(sh.max_kv < 1 ? 1 : sh.max_kv, kRound) * kRound;
        p.direct = true;
        return p;
    }
    // Parts of the keys: as many work items in all as the chip holds at once of the
    // wide kernels (two workgroups a CU at 128, four at 64), none below 256 keys.
    // More parts cost more partial rows: 64 requests behind 32768 tokens take 100 us
    // with 512 items, 106 with 768, 116 with 1024; chunks of heads of 64 take 154, 151
    // and 141.
    const int64_t base_p = (int64_t)p.tiles_p * sh.hk, base_s = sh.n_req * p.tiles_s * sh.hk;
    const int64_t blocks_p = base_p * ceil_div(sh.prefix, KB), blocks_s = base_s * ceil_div(sh.max_kv, KB);
    const int64_t items = full_chip(sh.hd);
    int64_t chunk = ceil_div(blocks_p + blocks_s, items);
    if (chunk < 8) chunk = 8;
    // The prefix's length is known, max_kv only bounds the requests': their keys count
    // for at most twice the prefix's where its parts are cut, or a bound far above the
    // lengths would leave it too few to fill the chip (64 requests of up to 2000 keys
    // behind 32768, 32 heads over 8 of 128, max_kv 32768: 97 us against 640; 200 of up
    // to 300 behind 4001: 42 against 92).  No shorter than 1024 keys on that account
    // (200 behind 3000, 16 heads of 64: 28.6 us against 30.2 with 512; 64 behind 8192:
    // 34.0 against 30.2, and 51 with 2048).
    int64_t chunk_p = ceil_div(3 * blocks_p, items);
    if (chunk_p < kPrefixOwn) chunk_p = kPrefixOwn;
    if (chunk_p > chunk) chunk_p = chunk;
    // As many parts as that gives, of equal length.  Without a prefix, less than two
    // parts' worth of own keys is one: a call without a join (111 requests of up to 538
    // keys, 52 queries of 16 heads over 2: 25.7 us against 42.6; 7 requests of up to 353
    // keys, 29 queries: 7.0 against 9.7).
    auto parts = [&](int64_t keys, int64_t chunk, bool one, int* n, int64_t* len) {
        if (keys == 0) {
            *n = 0;
            *len = KB;
            return;
        }
        int64_t k = ceil_div(ceil_div(keys, KB), chunk);
        if (one && k == 2) k = 1;
        if (k > 64) k = 64;
        *len = ceil_div(ceil_div(keys, k), kRound) * kRound;
        *n = (int)ceil_div(keys, *len);
    };
    // Requests differ in length, and the bounds say nothing of it: where several have
    // tiles of 128 rows, no part of their keys is long enough to be what the others
    // wait for (16 requests, 128 queries of 20 heads over 4, up to 4000 keys: 67 us
    // against 94; 8 behind 4096 + 4000 keys, 256 queries: 172 against 209; two requests
    // 85 against 82, one 299 against 250).  Not at any price: max_kv may be a server's
    // context length, and each part is a row of fp32 for every row of the batch.  So
    // the partial rows stay within kWideOwnBytes and the workgroups, which a request
    // has whether it has rows or not, within kWideOwnTurns, or there are no more parts
    // than the chip needs (4 requests of 8192 rows in all, 32 heads over 8 of 128, max_kv
    // 131072: one part, where 64 would ask for 8.7 GB).  At 64, 128 MB and without
    // bound, max_kv 32768: 16 requests of up to 4000 keys 101, 68, 68 us; 32 of up to
    // 3000, 16 heads over 4, 139, 105, 124; 5 of up to 30000, 512 queries, 803, 756, 832;
    // 8 behind 4096 + 4000 134, 146, 127; 5 of up to 3000, 512 queries, 88, 111, 125.
    parts(sh.prefix, chunk_p, false, &p.splits_p, &p.chunk_p);
    int64_t own = chunk;
    // Few requests' trees are cut by their lengths on the GPU (counted_item); these parts
    // say how many the workspace has room for.  8 requests of up to
    // 32000 keys, 64 nodes of 32 heads over 8 of 128: 175 us against 205 with parts of 1536;
    // 4 of up to 8000, 200 nodes: 71 against 78.  Where the tiles fill half of the chip as
    // they are it costs more than it gives (32 of up to 4000, 32 nodes: 75 against 72).
    const int64_t kv_blocks = ceil_div(sh.max_kv, KB);
    const bool counted = tree && counts_lengths(sh, p.kind_s, p.tiles_s);
    const int64_t least = counted ? kTreeOwn : kWideOwn;
    if (counted || (wide && sh.n_req >= 4 && chunk > least)) {
        int64_t fit = kWideOwnBytes / (p.rows * (sh.hd + 2) * 4) - p.splits_p;
        if (fit > kWideOwnTurns / base_s) fit = kWideOwnTurns / base_s;
        own = ceil_div(kv_blocks, fit < 1 ? 1 : fit);
        if (own < least) own = least;
        if (own > chunk && !counted) own = chunk;
    }
    parts(sh.max_kv, own, sh.prefix == 0, &p.splits_s, &p.chunk_s);
    const int64_t n = (p.splits_p + p.splits_s) * p.rows;
    p.direct = p.splits_p == 0 && p.splits_s == 1;
    p.ws_bytes = p.direct || n == 0 ? 0 : (size_t)((2 * n + 63) / 64 * 64 + n * sh.hd) * 4;
    if (counted && p.ws_bytes > 0 && p.splits_s > 1) p.ws_bytes += 64;
    return p;
}

}  // namespace

PrefixAttnPlan plan_prefix_attn(const PrefixAttnShape& sh) { return plan_of(sh, false); }
PrefixAttnPlan plan_tree_attn(const PrefixAttnShape& sh) { return plan_of(sh, true); }

hipError_t launch_prefix_attn(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t,
                              hipStream_t s) {
    Args a = args_of(sh, p, t);
    // more turns than a grid may have go into launches one after the other
    for (a.base = 0; a.base < a.blocks; a.base += kMaxGrid) {
        const unsigned grid = (unsigned)(a.blocks - a.base < kMaxGrid ? a.blocks - a.base : kMaxGrid);
        const hipError_t e = t.mask ? start_tree_attn(sh.hd, p, &a, grid, s) : sh.hd == 64 ? go<64>(p, a, grid, s) : go<128>(p, a, grid, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_prefix_join(const PrefixAttnShape& sh, const PrefixAttnPlan& p, const PrefixAttnPtrs& t,
                              hipStream_t s) {
    if (p.direct) return hipSuccess;
    const Args a = args_of(sh, p, t);
    const int64_t new_rows = sh.max_new < sh.T ? sh.max_new : sh.T;
    // A thread for four elements while its loads of all parts fit a few rounds, or where
    // the rows fill the chip with such threads; a wave to a row beyond.
    const bool few = p.splits_p + p.splits_s <= kJoinFew || p.rows * (sh.hd / 4) >= kJoinThreads;
    int64_t gx = ceil_div(new_rows * sh.hq, few ? NTHR / (sh.hd / 4) : NW);
    if (gx > 4096) gx = 4096;
    const dim3 grid((unsigned)gx, (unsigned)sh.n_req);
    if (few) {
        if (sh.hd == 64) prefix_join_few_kernel<64><<<grid, NTHR, 0, s>>>(a);
        else prefix_join_few_kernel<128><<<grid, NTHR, 0, s>>>(a);
    } else {
        if (sh.hd == 64) prefix_join_kernel<64><<<grid, NTHR, 0, s>>>(a);
        else prefix_join_kernel<128><<<grid, NTHR, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace cola
