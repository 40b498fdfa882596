// Host interface between the entry points of the grouped products and the translation units that hold their kernels.
#pragma once
#include "g4_format.cuh"

struct G4TensorArgs {
    G4Weights w;
    const int32_t *offsets;
    int experts, rows;
    void *out;
    int64_t ldo;
};
// Rows as the tensor cores read them: bf16 / fp16, fp32 as three bf16 parts [3][rows][ldx]; ldx a multiple of 8.
int qnn_g4_tensor_fwd(const void *x, int type, int64_t ldx, const G4TensorArgs &a, cudaStream_t st);
int qnn_g4_tensor_data(const void *dy, int type, int64_t lddy, const G4TensorArgs &a, cudaStream_t st);
int qnn_expert_wgrad(const void *x, int64_t ldx, const void *dy, int64_t lddy, int type, const int32_t *offsets, int experts, int rows,
                     int n, int k, float *gw, float *parts, cudaStream_t st);
size_t qnn_expert_wgrad_parts_bytes(int64_t rows, int experts, int n, int k);      // of `parts` (0: it may be NULL)
