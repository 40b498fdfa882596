// The few-row form of the 4-bit products (g4_rows.cu) and the exact split of an fp32 value.
#pragma once
#include <type_traits>
#include "g4_format.cuh"

// Rows of x in blocks of `rows_together` (expert by expert when offsets is given) times their matrix.
int qnn_g4_rows(const void *x, int type, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, void *y,
                int64_t ldy, int rows_together, cudaStream_t st);

// fp32 = part 0 + part 1 + part 2, each with at most 8 significant bits (a bf16 in the upper half of the returned word):
// cutting towards zero leaves 16, then 8 bits.  An infinity or NaN is part 0 alone.
__device__ __forceinline__ uint32_t split_part_bits(float v, int part) {
    const bool finite = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
    const float p0 = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
    if (part == 0) return finite ? __float_as_uint(p0) : (v != v ? 0x7FC00000u : __float_as_uint(v));
    const float r1 = finite ? __fadd_rn(v, -p0) : 0.0f;
    const float p1 = __uint_as_float(__float_as_uint(r1) & 0xFFFF0000u);
    return part == 1 ? __float_as_uint(p1) : __float_as_uint(__fadd_rn(r1, -p1));
}
