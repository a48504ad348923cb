// rope.hip -- rotary positions of q and k rows, forward and backward, and the
// rotated rows' way into a paged cache (cola_rope_fwd, cola_rope_bwd,
// cola_cache_append).
//
// A pair (x, y) of a head at position p turns by the angle p f:
//   x' = x c - y s,  y' = y c + x s,   c = m cos(p f), s = m sin(p f);
// the backward is the transpose, the same with -s.  HBM bound: each element is
// read once and written once, 3 operations between.
//
// A thread owns one unit of a head, PV pairs in two vectors of PV elements: with
// the half layout elements u PV .. and rot/2 + u PV .., interleaved the 2 PV
// elements from 2 u PV on; units past the rotated part copy two vectors.  It
// forms the unit's cosines and sines once and walks over heads of its row with
// them.  The angle is taken in turns, pos * (f / 2 pi) in 64 bits, and only its
// fraction goes to 32 bits: positions of 2^31 lose nothing.  Vectors are loaded
// and stored at the elements' own alignment (gfx950 takes any address), so odd
// pitches need no other path.
#include <type_traits>

#include "serve.hpp"
#include "device_math.hpp"

namespace cola {
namespace {

constexpr int NTHR = 256;
constexpr int CH = 4;                 // heads whose loads a thread has in flight

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
    __device__ __forceinline__ void store(G p) const { *(__attribute__((address_space(1))) Loose*)p = r; }
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

template <bool BF16, int PV, bool INTER, bool CACHE>
__global__ __launch_bounds__(NTHR) void rope_kernel(const RopeArgs a) {
    typedef Vec<BF16, PV> V;
    typedef typename V::E E;
    const int per = a.lanes * a.units;                  // threads of one row
    int tl = 0, rem = (int)(blockIdx.y * NTHR + threadIdx.x);
    if (per < NTHR) {
        tl = rem / per;
        rem -= tl * per;
    }
    if (tl >= a.tpw || rem >= per) return;
    const int hl = rem / a.units, u = rem - hl * a.units;

    const bool turning = u < a.turning;
    const int half = a.rot / 2;
    int A, B;                                           // the unit's two vectors in a head
    if (!turning) {
        A = a.rot + 2 * PV * (u - a.turning);
        B = A + PV;
    } else if (INTER) {
        A = 2 * PV * u;
        B = A + PV;
    } else {
        A = PV * u;
        B = A + half;
    }
    const bool two = B < a.hd;

    const int H = a.hq + a.hk + (CACHE ? a.hk : 0);
    for (int64_t t = (int64_t)blockIdx.x * a.tpw + tl; t < a.T; t += (int64_t)gridDim.x * a.tpw) {
        float c[PV], s[PV];
        if (turning) {
            const int64_t p = a.pos ? (int64_t)a.pos[t] : (a.seq_len > 0 ? t % a.seq_len : t);
#pragma unroll
            for (int e = 0; e < PV; ++e) {
                const double turns = (double)p * a.rev[PV * u + e];
                turn<BF16>((float)(turns - rint(turns)), c[e], s[e]);
                c[e] *= a.mscale;
                s[e] *= a.mscale * a.sign;
            }
        }
        int64_t at = -1;                                // this row's place in the cache, less the head's part
        if constexpr (CACHE) {
            const int64_t slot = a.slots[t];
            if (slot >= 0 && slot < a.n_slots) {
                const int64_t page = slot >> a.lg_page, off = slot & ((int64_t(1) << a.lg_page) - 1);
                at = ((page * a.hk) << a.lg_page) + off;
            }
        }
        for (int h0 = hl; h0 < H; h0 += CH * a.lanes) {
            V x[CH], y[CH];
            typename V::G dst[CH];
            bool on[CH];
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int h = h0 + j * a.lanes;
                on[j] = h < H;
                if (!on[j]) continue;
                const E* src;
                if (h < a.hq) {
                    src = (const E*)a.q + t * a.ldq + (int64_t)h * a.hd;
                    dst[j] = (typename V::G)a.qo + t * a.ldqo + (int64_t)h * a.hd;
                } else {
                    const int hk = h - a.hq;
                    if constexpr (CACHE) {
                        const bool val = hk >= a.hk;
                        const int hh = val ? hk - a.hk : hk;
                        src = (val ? (const E*)a.v + t * a.ldv : (const E*)a.k + t * a.ldk) + (int64_t)hh * a.hd;
                        dst[j] = (typename V::G)(val ? a.V : a.K) + (at + ((int64_t)hh << a.lg_page)) * a.hd;
                        on[j] = at >= 0;
                    } else {
                        src = (const E*)a.k + t * a.ldk + (int64_t)hk * a.hd;
                        dst[j] = (typename V::G)a.ko + t * a.ldko + (int64_t)hk * a.hd;
                    }
                }
                if (on[j]) {
                    x[j].load(src + A);
                    if (two) y[j].load(src + B);
                }
            }
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                if (!on[j]) continue;
                if (turning && h0 + j * a.lanes < a.hq + a.hk) {
                    float p[PV], q[PV];
                    x[j].get(p);
                    y[j].get(q);
                    if constexpr (INTER && PV > 1) {
                        // pairs 0 .. PV/2 - 1 in the first vector, the others in the second
#pragma unroll
                        for (int e = 0; e < PV / 2; ++e) {
                            const float p0 = p[2 * e], q0 = q[2 * e];
                            p[2 * e] = p0 * c[e] - p[2 * e + 1] * s[e];
                            p[2 * e + 1] = p[2 * e + 1] * c[e] + p0 * s[e];
                            q[2 * e] = q0 * c[e + PV / 2] - q[2 * e + 1] * s[e + PV / 2];
                            q[2 * e + 1] = q[2 * e + 1] * c[e + PV / 2] + q0 * s[e + PV / 2];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < PV; ++e) {
                            const float p0 = p[e];
                            p[e] = p0 * c[e] - q[e] * s[e];
                            q[e] = q[e] * c[e] + p0 * s[e];
                        }
                    }
                    x[j].put(p);
                    y[j].put(q);
                }
                x[j].store(dst[j] + A);
                if (two) y[j].store(dst[j] + B);
            }
        }
    }
}

template <bool BF16, int PV>
hipError_t go(bool inter, bool cache, const RopeArgs& a, dim3 grid, hipStream_t s) {
    if (inter) {
        if (cache) rope_kernel<BF16, PV, true, true><<<grid, NTHR, 0, s>>>(a);
        else rope_kernel<BF16, PV, true, false><<<grid, NTHR, 0, s>>>(a);
    } else {
        if (cache) rope_kernel<BF16, PV, false, true><<<grid, NTHR, 0, s>>>(a);
        else rope_kernel<BF16, PV, false, false><<<grid, NTHR, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(bool bf16, bool cache, RopeArgs& a, hipStream_t s) {
    // the widest vector that divides the rotated half and the head
    const int top = bf16 ? 8 : 4;
    int pv = top;
    while (pv > 1 && ((a.rot / 2) % pv != 0 || a.hd % pv != 0)) pv /= 2;
    a.turning = a.rot / 2 / pv;
    a.units = a.turning + (a.hd - a.rot + 2 * pv - 1) / (2 * pv);
    const int H = a.hq + (cache ? 2 : 1) * a.hk;
    // Threads of a row share its heads out: about eight heads each where there
    // are rows enough to fill the chip, down to one each where there are few.
    int64_t lanes = (int64_t(1) << 18) / (a.T * a.units) + 1;
    if (lanes < (H + 7) / 8) lanes = (H + 7) / 8;
    if (lanes > H) lanes = H;
    a.lanes = (int)lanes;
    const int per = a.lanes * a.units;
    a.tpw = per < NTHR ? NTHR / per : 1;
    int64_t gx = (a.T + a.tpw - 1) / a.tpw;
    if (gx > (1 << 20)) gx = 1 << 20;
    const dim3 grid((unsigned)gx, (unsigned)(per < NTHR ? 1 : (per + NTHR - 1) / NTHR));
    if (bf16) {
        if (pv == 8) return go<true, 8>(a.interleaved, cache, a, grid, s);
        if (pv == 4) return go<true, 4>(a.interleaved, cache, a, grid, s);
        if (pv == 2) return go<true, 2>(a.interleaved, cache, a, grid, s);
        return go<true, 1>(a.interleaved, cache, a, grid, s);
    }
    if (pv == 4) return go<false, 4>(a.interleaved, cache, a, grid, s);
    if (pv == 2) return go<false, 2>(a.interleaved, cache, a, grid, s);
    return go<false, 1>(a.interleaved, cache, a, grid, s);
}

}  // namespace cola
