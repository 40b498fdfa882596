// Real operands rewritten for the tensor cores (g4_stage.cu).
#pragma once
#include "g4_rows.cuh"

static inline int64_t g4_padded_width(int width) { return ((int64_t)width + 7) / 8 * 8; }
static inline int g4_type_parts(int type) { return type == QNN_F32 ? 3 : 1; }
// Can the tensor cores read the rows where they lie?
static inline bool g4_rows_in_place(const void *p, int type, int64_t ld) {
    return type != QNN_F32 && qnn_aligned(p, 16) && ld % 8 == 0;
}
// Bytes of the rewritten rows, a multiple of 256.
static inline size_t g4_staged_bytes(int type, int64_t rows, int width) {
    const size_t b = (size_t)g4_type_parts(type) * (size_t)rows * (size_t)g4_padded_width(width) * 2u;
    return (b + 255) / 256 * 256;
}
// dst [parts][rows][padded width].
int qnn_stage_rows(const void *src, int type, int64_t ld, int rows, int width, void *dst, cudaStream_t st);
// Two operands with the same rows in one launch.
int qnn_stage_rows_two(const void *src_a, int64_t ld_a, int width_a, void *dst_a, const void *src_b, int64_t ld_b, int width_b, void *dst_b,
                       int type, int rows, cudaStream_t st);
