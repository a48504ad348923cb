// row_tile.hpp -- pieces that the attention kernels share: the 32 x 32 x 16 matrix
// instruction with its lane layout, a row-major LDS tile of keys, values or
// queries with both of its operand reads, and the softmax's small helpers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cola {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4* lptr4_t;

constexpr int STG = 64;          // rows (keys or queries) staged in LDS per barrier pair: two 32-row sub-blocks

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// exp2 by the hardware instruction alone (no range reduction for denormal
// results): its arguments here are scores minus their running maximum or
// minus the log-sum-exp, so a result it flushes to zero is below 2^-126 and
// far below the bf16 resolution of the probabilities it feeds.
__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

// Row (key or query) of register v of a 32 x 32 accumulator, within its tile.
__device__ __forceinline__ int acc_row(int v, int hh) { return 8 * (v >> 2) + 4 * hh + (v & 3); }

// Max with lane l ^ 32 (the other half of a query's scores) by one
// v_permlane32_swap.
__device__ __forceinline__ float xor32_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// LDS tile of STG rows x HD, row-major, 16-byte chunks XOR-swizzled by the
// row (conflict-free fragment reads of both kinds below).
template <int HD>
struct RowTile {
    static constexpr int BYTES = STG * HD * 2;
    __device__ static __forceinline__ int off(int row, int chunk) { return row * (HD * 2) + ((chunk ^ (row & 7)) << 4); }
    // A-operand fragment of step s (HD elements 16 s ..) for rows r0 .. r0 + 31
    // (lane: row r0 + lane % 32)
    __device__ static __forceinline__ bf16x8 frag(const char* t, int r0, int s, int lane) {
        const int row = r0 + (lane & 31);
        return *reinterpret_cast<const bf16x8*>(t + off(row, 2 * s + (lane >> 5)));
    }
    // A-operand fragment of the transpose: 32 HD elements (tile nt) x 16 rows
    // (step s of the 32-row sub-block at r0), by two transposing reads.  Lane
    // (n = 32 nt + lane % 32, hh = lane / 32) receives rows
    // r0 + 16 s + 4 hh + 0..3 and r0 + 16 s + 8 + 4 hh + 0..3 at element n --
    // the order in which the transposed score tile leaves those rows in a
    // lane's accumulator registers 8 s .. 8 s + 7.  (In each 16-lane group,
    // lanes 4q .. 4q + 3 point at row q of a 4 x 16 block, four consecutive
    // elements each, and lane i receives element i of the block.)
    __device__ static __forceinline__ bf16x8 frag_tr(const char* t, int r0, int nt, int s, int lane) {
        const int g = lane >> 4, i = lane & 15;
        const int m = 32 * nt + 16 * (g & 1) + 4 * (i & 3);
        const int k = r0 + 16 * s + 4 * (g >> 1) + (i >> 2);
        const int byte = (m & 7) * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr4_t)(t + off(k, m >> 3) + byte));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lptr4_t)(t + off(k + 8, m >> 3) + byte));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    }
};

}  // namespace cola
