// Host interface between the entry points of the grouped products and the translation units that hold their kernels.
#pragma once
#include "g4_format.cuh"

struct G4TensorArgs {
    G4Weights w;
    const int32_t *offsets;
    int experts, rows;
    void *out;
    int64_t ldo;
    void *sums;                           // fp32 [plan.parts][rows][features] when the plan has more than one part
};

// Tile and split of a grouped product.  tokens: width of a tile (32 and 64: one block and 128 features; 128 and 256: a pair of
// blocks and 256).  The time of a block is estimated as rounds x (steps x cycles a step + a fixed part); cycles are what the
// kernels take on a B200 when every SM is busy, and a split pays for the second kernel that adds the parts.  Sized for 148
// SMs, so that workspace queries and calls agree.
struct G4Plan {
    int tokens, parts, steps_each;
};
G4Plan g4_tensor_plan(bool data, bool fp32, int64_t rows, int experts, int features, int steps);
static inline size_t g4_sums_bytes(const G4Plan &plan, int64_t rows, int features) {
    return plan.parts > 1 ? ((size_t)plan.parts * (size_t)rows * (size_t)features * sizeof(float) + 255) / 256 * 256 : 0;
}
// Rows as the tensor cores read them: bf16 / fp16, fp32 as three bf16 parts [3][rows][ldx]; ldx a multiple of 8.
int qnn_g4_tensor_fwd(const void *x, int type, int64_t ldx, const G4TensorArgs &a, cudaStream_t st);
int qnn_g4_tensor_data(const void *dy, int type, int64_t lddy, const G4TensorArgs &a, cudaStream_t st);
int qnn_expert_wgrad(const void *x, int64_t ldx, const void *dy, int64_t lddy, int type, const int32_t *offsets, int experts, int rows,
                     int n, int k, float *gw, float *parts, cudaStream_t st);
void qnn_expert_wgrad_plan(int64_t rows, int experts, int n, int k, int *tile, int *parts);
size_t qnn_expert_wgrad_parts_bytes(int64_t rows, int experts, int n, int k);      // of `parts` (0: it may be NULL)
