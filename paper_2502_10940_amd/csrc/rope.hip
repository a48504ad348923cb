// rope.hip -- rotary positions of q and k rows, forward and backward, and the
// rotated rows' way into a paged cache (cola_rope_fwd, cola_rope_bwd,
// cola_cache_append).
//
// A pair (x, y) of a head at position p turns by the angle p f:
//   x' = x c - y s,  y' = y c + x s,   c = m cos(p f), s = m sin(p f);
// the backward is the transpose, the same with -s.  HBM bound: each element is
// read once and written once, 3 operations between.  32768 rows of 32 + 32 heads of
// 64 (537 MB): 101 us, 5.3 TB/s; 8191 rows of 32 + 8 heads of 128, interleaved (168
// MB): 30.4 us, 5.5 TB/s; 6001 rows of 32 + 8 into the cache (148 MB): 26.6 us, 5.5 TB/s; a
// large copy reaches 5.1 to 5.4.  Small calls cost a launch: 256 rows 5.1 us.
//
// A thread owns one unit of a head and walks over heads of its row with it: with the
// half layout PV pairs in two vectors of PV elements, u PV .. and rot/2 + u PV ..;
// interleaved PV/2 pairs in one.  Units past the rotated part copy.  Neighbouring
// threads own neighbouring vectors, so each load and store of a wave covers whole
// runs.  The first heads' loads are issued before the cosines and sines are formed,
// which every head of the row shares.  The angle is taken in turns, pos * (f / 2 pi)
// in 64 bits, and only its fraction goes to 32 bits: positions of 2^31 lose nothing.
// Vectors are loaded and stored at the elements' own alignment (gfx950 takes any
// address), so odd pitches need no other path (17143 rows with a pitch of 5157: 80 us,
// 4.4 TB/s, where aligned rows of as many bytes reach 5.6).
#include <type_traits>

#include "serve.hpp"
#include "device_math.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;

// PV elements, loaded and stored at the alignment of one of them.
template <bool BF16, int PV>
struct Vec {
    typedef typename std::conditional<BF16, uint16_t, float>::type E;
    typedef typename std::conditional<BF16 && PV == 1, uint16_t, uint32_t>::type W;
    static constexpr int N = BF16 && PV > 1 ? PV / 2 : PV;
    typedef W Raw __attribute__((ext_vector_type(N)));
    typedef Raw Loose __attribute__((aligned(sizeof(E))));
    // The address space is said: a destination picked among buffers loses it.
    typedef __attribute__((address_space(1))) E* G;
    Raw r;
    __device__ __forceinline__ void load(const E* p) { r = *reinterpret_cast<const Loose*>(p); }
    template <bool PAST>
    __device__ __forceinline__ void store(G p) const {
        if constexpr (PAST) __builtin_nontemporal_store(r, (__attribute__((address_space(1))) Loose*)p);
        else *(__attribute__((address_space(1))) Loose*)p = r;
    }
    // the first element alone
    __device__ __forceinline__ void load_first(const E* p) {
        if constexpr (sizeof(W) == sizeof(E)) r[0] = reinterpret_cast<const W*>(p)[0];
        else r[0] = p[0];
    }
    __device__ __forceinline__ void store_first(G p) const {
        if constexpr (sizeof(W) == sizeof(E)) ((__attribute__((address_space(1))) W*)p)[0] = r[0];
        else p[0] = (E)r[0];
    }
    __device__ __forceinline__ void get(float (&f)[PV]) const {
#pragma unroll
        for (int i = 0; i < PV; ++i) {
            if constexpr (!BF16) f[i] = __uint_as_float(r[i]);
            else if constexpr (PV == 1) f[i] = bf16_to_f32(r[0]);
            else f[i] = i & 1 ? __uint_as_float(r[i / 2] & 0xffff0000u) : bf16_to_f32(r[i / 2] & 0xffffu);
        }
    }
    __device__ __forceinline__ void put(const float (&f)[PV]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (!BF16) r[i] = __float_as_uint(f[i]);
            else if constexpr (PV == 1) r[0] = (uint16_t)f32_to_bf16(f[0]);
            else r[i] = pack_bf16x2(f[2 * i], f[2 * i + 1]);
        }
    }
};

// Cosine and sine of x turns, |x| <= 1/2.  bf16: the hardware instructions,
// whose arguments are turns (absolute error below 2^-18, the result is rounded
// to 2^-9); fp32: the library function.
template <bool BF16>
__device__ __forceinline__ void turn(float x, float& c, float& s) {
    if constexpr (BF16) {
        c = __builtin_amdgcn_cosf(x);
        s = __builtin_amdgcn_sinf(x);
    } else {
        sincospif(2.0f * x, &s, &c);
    }
}

// Row t's place of head h: q, then k, then (with a cache) v.
template <class E, bool CACHE>
__device__ __forceinline__ const E* source(const RopeArgs& a, int64_t t, int h) {
    if (h < a.hq) return (const E*)a.q + t * a.ldq + (int64_t)h * a.hd;
    const int hk = h - a.hq;
    if (CACHE && hk >= a.hk) return (const E*)a.v + t * a.ldv + (int64_t)(hk - a.hk) * a.hd;
    return (const E*)a.k + t * a.ldk + (int64_t)hk * a.hd;
}

template <bool BF16, int PV, bool INTER, bool CACHE, bool PAST>
__global__ __launch_bounds__(NTHR) void rope_kernel(const RopeArgs a) {
    typedef Vec<BF16, PV> V;
    typedef typename V::E E;
    typedef typename V::G G;
    constexpr int NV = INTER ? 1 : 2;                   // vectors of a unit
    constexpr int NP = INTER ? PV / 2 : PV;             // its pairs
    constexpr int CH = 8 / NV;                          // heads whose loads a thread has in flight
    const int per = a.lanes * a.units;                  // threads of one row
    int tl = 0, rem = (int)(blockIdx.y * NTHR + threadIdx.x);
    if (per < NTHR) {
        tl = rem / per;
        rem -= tl * per;
    }
    if (tl >= a.tpw || rem >= per) return;
    const int hl = rem / a.units, u = rem - hl * a.units;

    const bool turning = u < a.turning;
    int at[2];                                          // the unit's vectors in a head
    if (INTER) {
        at[0] = PV * u;
        at[1] = a.hd;
    } else if (turning) {
        at[0] = PV * u;
        at[1] = at[0] + a.rot / 2;
    } else {
        at[0] = a.rot + PV * (u - a.turning);
        at[1] = at[0] + PV * (a.units - a.turning);
    }
    // A vector past the head's end is left out; one across it (an odd head, pairs
    // interleaved) has its first element alone.
    const bool two = at[1] < a.hd, whole = at[0] + PV <= a.hd;

    const int H = a.hq + a.hk + (CACHE ? a.hk : 0);
    for (int64_t t = (int64_t)blockIdx.x * a.tpw + tl; t < a.T; t += (int64_t)gridDim.x * a.tpw) {
        V x[CH][NV];
        auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int h = h0 + j * a.lanes;
                if (h >= H) continue;
                const E* src = source<E, CACHE>(a, t, h);
                if (PV == 1 || !INTER || whole) x[j][0].load(src + at[0]);
                else x[j][0].load_first(src + at[0]);
                if (NV == 2 && two) x[j][NV - 1].load(src + at[1]);
            }
        };
        load(hl);
        float c[NP], s[NP];
        if (turning) {
            const int64_t p = a.pos ? (int64_t)a.pos[t] : (a.seq_len > 0 ? t % a.seq_len : t);
#pragma unroll
            for (int e = 0; e < NP; ++e) {
                const double turns = (double)p * a.rev[NP * u + e];
                turn<BF16>((float)(turns - rint(turns)), c[e], s[e]);
                c[e] *= a.mscale;
                s[e] *= a.mscale * a.sign;
            }
        }
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
                if (h >= H) continue;
                if (turning && h < a.hq + a.hk) {
                    float p[PV];
                    x[j][0].get(p);
                    if constexpr (INTER) {
#pragma unroll
                        for (int e = 0; e < NP; ++e) {
                            const float p0 = p[2 * e];
                            p[2 * e] = p0 * c[e] - p[2 * e + 1] * s[e];
                            p[2 * e + 1] = p[2 * e + 1] * c[e] + p0 * s[e];
                        }
                    } else {
                        float q[PV];
                        x[j][NV - 1].get(q);
#pragma unroll
                        for (int e = 0; e < NP; ++e) {
                            const float p0 = p[e];
                            p[e] = p0 * c[e] - q[e] * s[e];
                            q[e] = q[e] * c[e] + p0 * s[e];
                        }
                        x[j][NV - 1].put(q);
                    }
                    x[j][0].put(p);
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
                if (PV == 1 || !INTER || whole) x[j][0].template store<PAST>(dst + at[0]);
                else x[j][0].store_first(dst + at[0]);
                if (NV == 2 && two) x[j][NV - 1].template store<PAST>(dst + at[1]);
            }
        }
    }
}

template <bool BF16, int PV, bool INTER, bool CACHE>
void start(bool past, const RopeArgs& a, dim3 grid, hipStream_t s) {
    if (past) rope_kernel<BF16, PV, INTER, CACHE, true><<<grid, NTHR, 0, s>>>(a);
    else rope_kernel<BF16, PV, INTER, CACHE, false><<<grid, NTHR, 0, s>>>(a);
}

template <bool BF16, int PV>
hipError_t go(bool cache, bool past, const RopeArgs& a, dim3 grid, hipStream_t s) {
    if (a.interleaved) {
        if constexpr (PV > 1) {
            if (cache) start<BF16, PV, true, true>(past, a, grid, s);
            else start<BF16, PV, true, false>(past, a, grid, s);
        }
    } else {
        if (cache) start<BF16, PV, false, true>(past, a, grid, s);
        else start<BF16, PV, false, false>(past, a, grid, s);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(bool bf16, bool cache, RopeArgs& a, hipStream_t s) {
    // The widest vector that divides the rotated part's vectors and the head;
    // interleaved pairs need two elements, and an odd head then ends in half of one.
    int pv = bf16 ? 8 : 4;
    const int turned = a.interleaved ? a.rot : a.rot / 2, least = a.interleaved ? 2 : 1;
    while (pv > least && (turned % pv != 0 || a.hd % pv != 0)) pv /= 2;
    a.turning = turned / pv;
    const int copied = (a.hd - a.rot + pv - 1) / pv;
    a.units = a.turning + (a.interleaved ? copied : (copied + 1) / 2);
    const int H = a.hq + (cache ? 2 : 1) * a.hk, CH = a.interleaved ? 8 : 4;
    // Large results go past the caches, where they would only drive out the rows that
    // are still read: 64 MB in 22 us against 30, 128 MB in 51 against 54, and a kernel
    // that reads them next takes as long either way.  Smaller ones stay for it (16 MB
    // and a reader 19.0 us against 20.9, 32 MB 25.4 against 27.1).
    // Rows that begin inside a line of 64 bytes stay as well, for the caches put its
    // halves together (140 MB of rows with a pitch of 4133: 62 us against 74).
    const int es = bf16 ? 2 : 4;
    const bool whole = ((a.ldqo * es | a.ldko * es | (int64_t)(uintptr_t)a.qo | (int64_t)(uintptr_t)a.ko) & 63) == 0;
    const bool past = whole && (double)a.T * H * a.hd * es > 48e6;
    // Threads of a row share its heads out: as many heads each as it has loads in
    // flight, down to one each where rows are few (2^18 threads fill the chip).
    int64_t lanes = (int64_t(1) << 18) / (a.T * a.units) + 1;
    if (lanes < (H + CH - 1) / CH) lanes = (H + CH - 1) / CH;
    if (lanes > H) lanes = H;
    a.lanes = (int)lanes;
    const int per = a.lanes * a.units;
    a.tpw = per < NTHR ? NTHR / per : 1;
    int64_t gx = (a.T + a.tpw - 1) / a.tpw;
    if (gx > (1 << 20)) gx = 1 << 20;
    const dim3 grid((unsigned)gx, (unsigned)(per < NTHR ? 1 : (per + NTHR - 1) / NTHR));
    if (bf16) {
        if (pv == 8) return go<true, 8>(cache, past, a, grid, s);
        if (pv == 4) return go<true, 4>(cache, past, a, grid, s);
        if (pv == 2) return go<true, 2>(cache, past, a, grid, s);
        return go<true, 1>(cache, past, a, grid, s);
    }
    if (pv == 4) return go<false, 4>(cache, past, a, grid, s);
    if (pv == 2) return go<false, 2>(cache, past, a, grid, s);
    return go<false, 1>(cache, past, a, grid, s);
}

}  // namespace cola
