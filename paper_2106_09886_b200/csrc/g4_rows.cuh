// The few-row form of the 4-bit products (g4_rows.cu) and the exact split of an fp32 value.
#pragma once
#include <type_traits>
#include "g4_format.cuh"

// Rows of x in blocks of `rows_together` (at most 8, fp32 at most 4; expert by expert when offsets is given) times their matrix.
int qnn_g4_rows(const void *x, int type, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, void *y,
                int64_t ldy, int rows_together, cudaStream_t st);

// fp32 = part 0 + part 1 + part 2, each with at most 8 significant bits (a bf16 in the upper half of the returned word):
// cutting towards zero leaves 16, then 8 bits.  (Below 2^-110 the last bits fall under bf16's smallest step and are cut.)  An infinity is (one of its sign, 0, the infinity): where both operands are
// split, the largest part of one meets every part of the other, and lower parts of finite values may be 0, which an infinity
// there would turn into NaN.  So part 2 meets part 0 alone, which is not 0 unless the value is (or lies below 2^-133, the
// smallest bf16).  A NaN is part 0 alone.
__device__ __forceinline__ uint32_t split_part_bits(float v, int part) {
    const uint32_t bits = __float_as_uint(v);
    const bool finite = (bits & 0x7F800000u) != 0x7F800000u;
    const float p0 = __uint_as_float(bits & 0xFFFF0000u);
    if (part == 0) return finite ? __float_as_uint(p0) : (v != v ? 0x7FC00000u : (bits & 0x80000000u) | 0x3F800000u);
    const float r1 = finite ? __fadd_rn(v, -p0) : 0.0f;
    const float p1 = __uint_as_float(__float_as_uint(r1) & 0xFFFF0000u);
    if (part == 1) return __float_as_uint(p1);
    return finite || v != v ? __float_as_uint(__fadd_rn(r1, -p1)) : bits;
}
