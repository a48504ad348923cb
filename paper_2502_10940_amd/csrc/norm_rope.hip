// norm_rope.hip -- norms of q and k for each head with the rotation in the same pass,
// forward, backward, and on the way into a paged cache (cola_norm_rope_fwd,
// cola_norm_rope_bwd, cola_norm_append).
//
// A head x of D elements with gain g:  n = x r, r = 1 / sqrt(mean(x^2) + eps),
// y = R(p) (n g) with the rotation R of rope.hip.  With dz = R^T dy and w = dz g:
//   dg = sum over rows and heads of dz n,   dx = r (w - n mean(w n)).
// HBM bound: forward reads x and writes y, backward reads x and dy and writes dx.  32768
// rows of 32 + 32 heads of 64 (537 MB, 805 MB): forward 106 us, backward 164 us, 5.1 and 4.9
// TB/s, where a large copy reaches 5.1; 8191 rows of 32 + 8 heads of 128 of which half turn,
// interleaved (252 MB): backward 67 us, 3.8 TB/s, the vector unit busy for 40 % of it (the
// row's cosines, formed by every group, are a third of its work), and the last quarter
// of its workgroups alone on the chip; 1536 rows of 32 + 8 into the cache (37 MB): 11.9 us.
// fp32: gradients of 8191 rows of 32 + 8 heads of 128 (503 MB) 104 us, 4.9 TB/s; 6001 such
// rows into the cache (295 MB) 70 us, 4.2 TB/s.  256 rows: 5.2 us forward, a launch;
// backward 12, two of them.
//
// A head is a group of L lanes (a power of two, 64 at most), a lane one unit of it as
// in rope.hip (MU of them where a head has more than 64): a pair of vectors that turn
// into each other, so that the rotation stays in the lane and the mean is the only
// thing that the group exchanges (log2 L steps between registers).  Heads that are no
// power of two leave lanes idle, three of eight at 80, two at 96: 16000 rows of 20 + 5
// heads of 80 (128 MB, 192 MB) take 34 us forward, 3.8 TB/s, and 69 backward, 2.8.  The
// rest is the rotation's: a row's groups share out its heads, loads of several heads are
// in flight before the cosines are formed.
//
// dg is summed in a fixed order: a thread over its rows and heads, the groups of a
// workgroup, and the workgroups (at most kParts of them) in a second launch.
#include "rows.hpp"
#include "serve.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;

// The sum over the groups of L lanes; L is the same for all lanes.
__device__ __forceinline__ float group_sum(float x, int L) {
    auto dpp = [](float v, auto ctrl) __attribute__((always_inline)) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    if (L > 1) x += dpp(x, std::integral_constant<int, 0xB1>{});        // lane ^ 1
    if (L > 2) x += dpp(x, std::integral_constant<int, 0x4E>{});        // lane ^ 2
    if (L > 4) x += dpp(x, std::integral_constant<int, 0x141>{});       // mirrored in 8 lanes: the other four's sum
    if (L > 8) x += dpp(x, std::integral_constant<int, 0x140>{});       // mirrored in 16 lanes
    if (L > 16) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if (L > 32) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    return x;
}

// The sum over a wave's groups of L lanes: lanes of one place in their group.
__device__ __forceinline__ float across_groups(float x, int L) {
    auto ror = [](float v, auto n) __attribute__((always_inline)) {
        return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + decltype(n)::value, 0xf, 0xf, true));
    };
    if (L < 64) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if (L < 32) {
        const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    }
    if (L < 16) x += ror(x, std::integral_constant<int, 8>{});
    if (L < 8) x += ror(x, std::integral_constant<int, 4>{});
    if (L < 4) x += ror(x, std::integral_constant<int, 2>{});
    if (L < 2) x += ror(x, std::integral_constant<int, 1>{});
    return x;
}

// 1 / sqrt(x): the hardware's (1 ulp) under a bf16 result, the rounded one under fp32.
template <bool BF16>
__device__ __forceinline__ float inv_sqrt(float x) {
    if constexpr (BF16) return __builtin_amdgcn_rsqf(x);
    else return 1.0f / sqrtf(x);
}

// A lane's part of a head: MU units of NV vectors.
template <bool BF16, int PV, bool INTER, int MU>
struct Part {
    typedef Vec<BF16, PV> V;
    typedef typename V::E E;
    typedef typename V::G G;
    static constexpr int NV = INTER ? 1 : 2;            // vectors of a unit
    static constexpr int NP = INTER ? PV / 2 : PV;      // its pairs

    // Where the lane's units lie, as in rope.hip: `turning` ones first, the rest copies
    // (here: is scaled without a turn).
    struct At {
        int at[MU][2];
        bool turning[MU], one[MU], two[MU], whole[MU];
        __device__ __forceinline__ void set(const RopeArgs& a, int u0, int L) {
#pragma unroll
            for (int m = 0; m < MU; ++m) {
                const int u = u0 + m * L;
                turning[m] = u < a.turning;
                if (INTER) {
                    at[m][0] = PV * u;
                    at[m][1] = a.hd;
                } else if (turning[m]) {
                    at[m][0] = PV * u;
                    at[m][1] = at[m][0] + a.rot / 2;
                } else {
                    at[m][0] = a.rot + PV * (u - a.turning);
                    at[m][1] = at[m][0] + PV * (a.units - a.turning);
                }
                one[m] = u < a.units && at[m][0] < a.hd;
                two[m] = u < a.units && at[m][1] < a.hd;
                whole[m] = at[m][0] + PV <= a.hd;
            }
        }
    };
    V x[MU][NV];

    __device__ __forceinline__ void load(const E* p, const At& w) {
#pragma unroll
        for (int m = 0; m < MU; ++m)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                x[m][v].r = 0;
                if (!(v ? w.two[m] : w.one[m])) continue;
                if (PV == 1 || !INTER || w.whole[m]) x[m][v].load(p + w.at[m][v]);
                else x[m][v].load_first(p + w.at[m][v]);
            }
    }
    __device__ __forceinline__ void store(G p, const At& w, bool past) const {
#pragma unroll
        for (int m = 0; m < MU; ++m)
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (!(v ? w.two[m] : w.one[m])) continue;
                if (PV > 1 && INTER && !w.whole[m]) x[m][v].store_first(p + w.at[m][v]);
                else if (past) x[m][v].template store<true>(p + w.at[m][v]);
                else x[m][v].template store<false>(p + w.at[m][v]);
            }
    }
    // Elements past the head's end are zeros, or (gains) what does not reach a result.
    __device__ __forceinline__ void get(float (&f)[MU][NV][PV]) const {
#pragma unroll
        for (int m = 0; m < MU; ++m)
#pragma unroll
            for (int v = 0; v < NV; ++v) x[m][v].get(f[m][v]);
    }
    __device__ __forceinline__ void put(const float (&f)[MU][NV][PV]) {
#pragma unroll
        for (int m = 0; m < MU; ++m)
#pragma unroll
            for (int v = 0; v < NV; ++v) x[m][v].put(f[m][v]);
    }
};

// Cosines and sines of a row's position for a lane's pairs.
template <bool BF16, int MU, int NP>
struct Turn {
    float c[MU][NP], s[MU][NP];
    template <class At>
    __device__ __forceinline__ void set(const RopeArgs& a, const At& w, int u0, int L, int64_t t) {
        const int64_t p = a.pos ? (int64_t)a.pos[t] : (a.seq_len > 0 ? t % a.seq_len : t);
#pragma unroll
        for (int m = 0; m < MU; ++m)
            if (w.turning[m]) {
#pragma unroll
                for (int e = 0; e < NP; ++e) {
                    const double turns = (double)p * a.rev[NP * (u0 + m * L) + e];
                    turn<BF16>((float)(turns - rint(turns)), c[m][e], s[m][e]);
                    c[m][e] *= a.mscale;
                    s[m][e] *= a.mscale * a.sign;
                }
            }
    }
    template <bool INTER, int NV, int PV, class At>
    __device__ __forceinline__ void apply(float (&f)[MU][NV][PV], const At& w) const {
#pragma unroll
        for (int m = 0; m < MU; ++m)
            if (w.turning[m]) {
#pragma unroll
                for (int e = 0; e < NP; ++e) {
                    float& x = INTER ? f[m][0][(2 * e) % PV] : f[m][0][e % PV];
                    float& y = INTER ? f[m][0][(2 * e + 1) % PV] : f[m][NV - 1][e % PV];
                    const float x0 = x;
                    x = x0 * c[m][e] - y * s[m][e];
                    y = y * c[m][e] + x0 * s[m][e];
                }
            }
    }
};

template <int MU, int NV, int PV>
__device__ __forceinline__ float dot(const float (&a)[MU][NV][PV], const float (&b)[MU][NV][PV]) {
    float s = 0.0f;
#pragma unroll
    for (int m = 0; m < MU; ++m)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int e = 0; e < PV; ++e) s = fmaf(a[m][v][e], b[m][v][e], s);
    return s;
}

// Row t's place of head h: q, then k, then (with a cache) v.
template <class E, bool CACHE>
__device__ __forceinline__ const E* source(const RopeArgs& a, int64_t t, int h) {
    if (h < a.hq) return (const E*)a.q + t * a.ldq + (int64_t)h * a.hd;
    const int hk = h - a.hq;
    if (CACHE && hk >= a.hk) return (const E*)a.v + t * a.ldv + (int64_t)(hk - a.hk) * a.hd;
    return (const E*)a.k + t * a.ldk + (int64_t)hk * a.hd;
}

template <bool BF16, int PV, bool INTER, bool CACHE, int MU>
__global__ __launch_bounds__(NTHR) void norm_rope_kernel(const NormRopeArgs a) {
    typedef Part<BF16, PV, INTER, MU> P;
    typedef typename P::E E;
    typedef typename P::G G;
    constexpr int NV = P::NV, NP = P::NP;
    constexpr int CH = MU > 1 ? 1 : 8 / NV;             // heads whose loads a thread has in flight
    const int L = a.group, per = a.lanes * L;           // threads of one row
    int rem = (int)(blockIdx.y * NTHR + threadIdx.x);
    const int tl = rem / per;
    rem -= tl * per;
    const int hl = rem / L, u0 = rem & (L - 1);
    typename P::At w;
    w.set(a, u0, L);
    P gq, gk;
    if (a.gq) gq.load((const E*)a.gq, w);
    if (a.gk) gk.load((const E*)a.gk, w);
    const int H = a.hq + a.hk + (CACHE ? a.hk : 0);
    for (int64_t t = (int64_t)blockIdx.x * a.tpw + tl; t < a.T; t += (int64_t)gridDim.x * a.tpw) {
        P x[CH];
        auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < CH; ++j)
                if (h0 + j * a.lanes < H) x[j].load(source<E, CACHE>(a, t, h0 + j * a.lanes), w);
        };
        load(hl);
        Turn<BF16, MU, NP> turn;
        turn.set(a, w, u0, L, t);
        int64_t place = -1;                             // this row's place in the cache, less the head's part
        if constexpr (CACHE) {
            const int64_t slot = a.slots[t];
            if (slot >= 0 && slot < a.n_slots) {
                const int64_t page = slot >> a.lg_page, off = slot & ((int64_t(1) << a.lg_page) - 1);
                place = ((page * a.hk) << a.lg_page) + off;
            }
        }
        for (int h0 = hl; h0 < H; h0 += CH * a.lanes) {
            if (h0 != hl) load(h0);
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int h = h0 + j * a.lanes;
                if (h >= H) continue;                   // the same for a group
                if (!CACHE || h < a.hq + a.hk) {
                    float f[MU][NV][PV];
                    x[j].get(f);
                    const float r = inv_sqrt<BF16>(fmaf(group_sum(dot(f, f), L), a.inv_hd, a.eps));
                    const bool is_q = h < a.hq;
                    const bool scaled = (is_q ? a.gq : a.gk) != nullptr;
#pragma unroll
                    for (int m = 0; m < MU; ++m)
#pragma unroll
                        for (int v = 0; v < NV; ++v) {
                            typename P::V g;
                            g.r = is_q ? gq.x[m][v].r : gk.x[m][v].r;
                            float y[PV];
                            g.get(y);
#pragma unroll
                            for (int e = 0; e < PV; ++e) f[m][v][e] = f[m][v][e] * r * (scaled ? y[e] : 1.0f);
                        }
                    turn.template apply<INTER>(f, w);
                    x[j].put(f);
                }
                G dst;
                if (h < a.hq) {
                    dst = (G)a.qo + t * a.ldqo + (int64_t)h * a.hd;
                } else if constexpr (CACHE) {
                    if (place < 0) continue;
                    const int hk = h - a.hq;
                    const bool val = hk >= a.hk;
                    dst = (G)(val ? a.V : a.K) + (place + ((int64_t)(val ? hk - a.hk : hk) << a.lg_page)) * a.hd;
                } else {
                    dst = (G)a.ko + t * a.ldko + (int64_t)(h - a.hq) * a.hd;
                }
                x[j].store(dst, w, a.past);
            }
        }
    }
}

// Backward: q, k as in the forward, their gradients' rows dqo, dko, results into qo, ko
// (at q's and k's pitches), and this workgroup's sums of dg in part.
template <bool BF16, int PV, bool INTER, int MU>
__global__ __launch_bounds__(NTHR) void norm_rope_bwd_kernel(const NormRopeArgs a) {
    typedef Part<BF16, PV, INTER, MU> P;
    typedef typename P::E E;
    typedef typename P::G G;
    constexpr int NV = P::NV, NP = P::NP;
    constexpr int CH = MU > 1 ? 1 : 4 / NV;
    extern __shared__ float sums[];                     // [NTHR / 64][2][hd]
    const int L = a.group, per = a.lanes * L;
    int rem = (int)(blockIdx.y * NTHR + threadIdx.x);
    const int tl = rem / per;
    rem -= tl * per;
    const int hl = rem / L, u0 = rem & (L - 1);
    typename P::At w;
    w.set(a, u0, L);
    P gq, gk;
    if (a.gq) gq.load((const E*)a.gq, w);
    if (a.gk) gk.load((const E*)a.gk, w);
    float dgq[MU][NV][PV] = {}, dgk[MU][NV][PV] = {};
    for (int64_t t = (int64_t)blockIdx.x * a.tpw + tl; t < a.T; t += (int64_t)gridDim.x * a.tpw) {
        Turn<BF16, MU, NP> turn;
        // This group's heads of q, or of k: one after the other, for each has its own gain.
        auto heads = [&](const E* from, const E* grad, G to, int H, const P& gain, bool scaled, float (&dg)[MU][NV][PV],
                         auto first) __attribute__((always_inline)) {
            P x[CH], y[CH];
            auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    const int h = h0 + j * a.lanes;
                    if (h >= H) continue;
                    x[j].load(from + (int64_t)h * a.hd, w);
                    y[j].load(grad + (int64_t)h * a.hd, w);
                }
            };
            load(hl);
            if constexpr (decltype(first)::value) turn.set(a, w, u0, L, t);
            for (int h0 = hl; h0 < H; h0 += CH * a.lanes) {
                if (h0 != hl) load(h0);
#pragma unroll
                for (int j = 0; j < CH; ++j) {
                    const int h = h0 + j * a.lanes;
                    if (h >= H) continue;
                    float n[MU][NV][PV], z[MU][NV][PV];
                    x[j].get(n);
                    y[j].get(z);
                    turn.template apply<INTER>(z, w);   // back: the sine has its sign
                    const float r = inv_sqrt<BF16>(fmaf(group_sum(dot(n, n), L), a.inv_hd, a.eps));
#pragma unroll
                    for (int m = 0; m < MU; ++m)
#pragma unroll
                        for (int v = 0; v < NV; ++v) {
                            float s[PV];
                            gain.x[m][v].get(s);
#pragma unroll
                            for (int e = 0; e < PV; ++e) {
                                n[m][v][e] *= r;
                                dg[m][v][e] = fmaf(z[m][v][e], n[m][v][e], dg[m][v][e]);
                                if (scaled) z[m][v][e] *= s[e];
                            }
                        }
                    const float mean = group_sum(dot(n, z), L) * a.inv_hd;
#pragma unroll
                    for (int m = 0; m < MU; ++m)
#pragma unroll
                        for (int v = 0; v < NV; ++v)
#pragma unroll
                            for (int e = 0; e < PV; ++e) z[m][v][e] = r * fmaf(-mean, n[m][v][e], z[m][v][e]);
                    x[j].put(z);
                    x[j].store(to + (int64_t)h * a.hd, w, a.past);
                }
            }
        };
        heads((const E*)a.q + t * a.ldq, (const E*)a.dqo + t * a.ldqo, (G)a.qo + t * a.ldq, a.hq, gq, a.gq != nullptr, dgq, std::true_type{});
        heads((const E*)a.k + t * a.ldk, (const E*)a.dko + t * a.ldko, (G)a.ko + t * a.ldk, a.hk, gk, a.gk != nullptr, dgk, std::false_type{});
    }
    // The groups of each wave, then the waves.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int m = 0; m < MU; ++m)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int e = 0; e < PV; ++e) {
                    const float x = across_groups(k ? dgk[m][v][e] : dgq[m][v][e], L);
                    const int at = w.at[m][v] + e;
                    if (lane < L && (v ? w.two[m] : w.one[m]) && at < a.hd) sums[(wave * 2 + k) * a.hd + at] = x;
                }
    __syncthreads();
    float* part = a.part + (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * 2 * a.hd;
    for (int i = threadIdx.x; i < 2 * a.hd; i += NTHR) {
        float x = 0.0f;
#pragma unroll
        for (int v = 0; v < NTHR / 64; ++v) x += sums[v * 2 * a.hd + i];
        part[i] = x;
    }
}

// dg of q and k from the workgroups' sums: COLS columns a workgroup, 1024 / COLS
// threads to each.
constexpr int COLS = 16;
__global__ __launch_bounds__(1024) void norm_gain_kernel(const float* part, int parts, int hd, float* dgq, float* dgk) {
    __shared__ float sums[1024];
    constexpr int SL = 1024 / COLS;
    const int col = blockIdx.x * COLS + threadIdx.x % COLS, slice = threadIdx.x / COLS;
    float x = 0.0f;
    if (col < 2 * hd)
        for (int p0 = slice; p0 < parts; p0 += 8 * SL) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = p0 + i * SL < parts ? part[(int64_t)(p0 + i * SL) * 2 * hd + col] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x += y[i];
        }
    sums[threadIdx.x] = x;
    __syncthreads();
    for (int d = SL / 2; d >= 1; d >>= 1) {
        if (slice < d) sums[threadIdx.x] += sums[threadIdx.x + d * COLS];
        __syncthreads();
    }
    if (slice == 0 && col < 2 * hd) {
        float* to = col < hd ? dgq : dgk;
        if (to) to[col < hd ? col : col - hd] = sums[threadIdx.x];
    }
}

template <bool BF16, int PV, bool INTER>
hipError_t start(NormKind kind, const NormRopeArgs& a, dim3 grid, hipStream_t s) {
    const size_t lds = kind == NORM_BWD ? (size_t)(NTHR / 64) * 2 * a.hd * 4 : 0;
#define COLA_GO(MU)                                                                                  \
    if (kind == NORM_BWD) norm_rope_bwd_kernel<BF16, PV, INTER, MU><<<grid, NTHR, lds, s>>>(a);      \
    else if (kind == NORM_APPEND) norm_rope_kernel<BF16, PV, INTER, true, MU><<<grid, NTHR, 0, s>>>(a); \
    else norm_rope_kernel<BF16, PV, INTER, false, MU><<<grid, NTHR, 0, s>>>(a)
    if (a.units <= 64) {
        COLA_GO(1);
    } else {
        // 512 elements in units of NV PV: bf16 vectors of 8 never come here
        if constexpr (!(BF16 && PV == 8)) { COLA_GO(4); }
    }
#undef COLA_GO
    return hipGetLastError();
}

template <bool BF16, int PV>
hipError_t go(NormKind kind, const NormRopeArgs& a, dim3 grid, hipStream_t s) {
    if (!a.interleaved) return start<BF16, PV, false>(kind, a, grid, s);
    if constexpr (PV > 1) return start<BF16, PV, true>(kind, a, grid, s);
    return hipErrorInvalidValue;
}

// Vectors, units and threads of a row, and the grid.
dim3 shape(bool bf16, NormKind kind, NormRopeArgs& a) {
    // as in rope.hip: the widest vector that divides the rotated part's vectors and the head
    int pv = bf16 ? 8 : 4;
    const int turned = a.interleaved ? a.rot : a.rot / 2, least = a.interleaved ? 2 : 1;
    while (pv > least && (turned % pv != 0 || a.hd % pv != 0)) pv /= 2;
    a.pv = pv;
    a.turning = turned / pv;
    const int copied = (a.hd - a.rot + pv - 1) / pv;
    a.units = a.turning + (a.interleaved ? copied : (copied + 1) / 2);
    a.group = 1;
    while (a.group < a.units && a.group < 64) a.group *= 2;
    // the heads that a row's groups share out: backward those of q, then those of k
    const int H = kind == NORM_BWD ? (a.hq > a.hk ? a.hq : a.hk) : a.hq + (kind == NORM_APPEND ? 2 : 1) * a.hk;
    const int CH = a.units > 64 ? 1 : (kind == NORM_BWD ? 4 : 8) / (a.interleaved ? 1 : 2);
    const int es = bf16 ? 2 : 4;
    // large results past the caches, as in rope.hip
    const int64_t pq = kind == NORM_BWD ? a.ldq : a.ldqo, pk = kind == NORM_BWD ? a.ldk : a.ldko;
    a.past = ((pq * es | pk * es | (int64_t)(uintptr_t)a.qo | (int64_t)(uintptr_t)a.ko) & 63) == 0 &&
             (double)a.T * (a.hq + a.hk) * a.hd * es > 48e6;
    // Groups of a row: as many as leave each two rounds of loads, for every group forms the
    // row's cosines again (16000 rows of 20 + 5 heads of 80: 34 us against 40 with one round,
    // backward 68 against 74), up to a head each where rows are few (2^18 threads fill the
    // chip), in powers of two (1536 rows into the cache: 12.5 us with 16, 14.8 with 22).
    int64_t lanes = 1;
    while (2 * lanes <= (int64_t(1) << 18) / (a.T * a.group) + 1) lanes *= 2;
    if (lanes < (H + 2 * CH - 1) / (2 * CH)) lanes = (H + 2 * CH - 1) / (2 * CH);
    if (lanes > H) lanes = H;
    // Rows of many heads take whole workgroups each (some groups then have no head), or the
    // rows that fill them would ask for a grid past its second axis.
    if (lanes * a.group > 8 * NTHR) lanes = (lanes + NTHR / a.group - 1) / (NTHR / a.group) * (NTHR / a.group);
    a.lanes = (int)lanes;
    // as many rows as fill whole workgroups: the groups of a row may lie in two (20 heads of
    // 80: 5 groups of 8 lanes a row, 32 rows in 5 workgroups; with the rest of each workgroup
    // idle instead, 8191 rows of 32 + 8 heads of 128 took 109 us against 70)
    const int64_t per = lanes * a.group;
    const int64_t low = per & -per;                     // its power of two
    a.tpw = low < NTHR ? (int)(NTHR / low) : 1;
    const int64_t gy = a.tpw * per / NTHR;
    int64_t gx = (a.T + a.tpw - 1) / a.tpw;
    int64_t most = int64_t(1) << 20;
    if (kind == NORM_BWD) most = kParts / gy > 1 ? kParts / gy : 1;
    if (gx > most) gx = most;
    return dim3((unsigned)gx, (unsigned)gy);
}

}  // namespace

size_t norm_rope_parts(bool bf16, NormRopeArgs a) {
    const dim3 g = shape(bf16, NORM_BWD, a);
    return (size_t)g.x * g.y;
}

hipError_t launch_norm_rope(bool bf16, NormKind kind, NormRopeArgs& a, hipStream_t s) {
    const dim3 grid = shape(bf16, kind, a);
    if (bf16) {
        if (a.pv == 8) return go<true, 8>(kind, a, grid, s);
        if (a.pv == 4) return go<true, 4>(kind, a, grid, s);
        if (a.pv == 2) return go<true, 2>(kind, a, grid, s);
        return go<true, 1>(kind, a, grid, s);
    }
    if (a.pv == 4) return go<false, 4>(kind, a, grid, s);
    if (a.pv == 2) return go<false, 2>(kind, a, grid, s);
    return go<false, 1>(kind, a, grid, s);
}

hipError_t launch_norm_gain(const NormRopeArgs& a, size_t parts, hipStream_t s) {
    norm_gain_kernel<<<(2 * a.hd + COLS - 1) / COLS, 1024, 0, s>>>(a.part, (int)parts, a.hd, a.dgq, a.dgk);
    return hipGetLastError();
}

}  // namespace cola
