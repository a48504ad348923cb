// rows.hpp -- rows of heads in vectors of any alignment, and the cosines and sines
// of their rotation: what rope.hip and norm_rope.hip share.
#pragma once

#include <type_traits>

#include "device_math.hpp"

namespace cola {

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

}  // namespace cola
