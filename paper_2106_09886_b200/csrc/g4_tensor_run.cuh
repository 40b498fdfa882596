// Choice of the tile for a grouped product.
#pragma once
#include "g4_tensor.cuh"
#include "g4_tensor_api.cuh"

namespace {

template <int MODE, class T>
int g4_tensor_pick(const void *x, int64_t ldx, const G4TensorArgs &a, cudaStream_t st) {
    G4TensorParams p = {};
    p.w = a.w; p.offsets = a.offsets; p.experts = a.experts; p.rows = a.rows; p.out = a.out; p.ldo = a.ldo;
    p.features = MODE == G4_FWD ? a.w.n : a.w.k;
    p.steps = MODE == G4_FWD ? a.w.tiles_k : a.w.tiles_n;
    p.out_vec = sizeof(T) == 2 && qnn_aligned(a.out, 16) && a.ldo % 8 == 0;
    p.wait_limit = WAIT_LIMIT;
    if (!(p.err = qnn_tc_error_word())) return QNN_E_CUDA;
    const int sms = sm_count();
    if (sms <= 0) return QNN_E_CUDA;
    const int width = MODE == G4_FWD ? a.w.k : a.w.n;
    const G4Plan plan = g4_tensor_plan(MODE == G4_DATA, sizeof(T) == 4, a.rows, a.experts, p.features, p.steps);
    p.steps_each = plan.steps_each;
    p.parts = plan.parts;
    p.sums = static_cast<float *>(a.sums);
    if (plan.tokens == 32) return g4_tensor_launch<1, 32, MODE, T>(x, ldx, width, p, sms, st);
    if constexpr (G4Type<T>::PARTS == 1) {
        if (plan.tokens == 128) return g4_tensor_launch<2, 128, MODE, T>(x, ldx, width, p, sms, st);
        if (plan.tokens == 256) return g4_tensor_launch<2, 256, MODE, T>(x, ldx, width, p, sms, st);
    }
    return g4_tensor_launch<1, 64, MODE, T>(x, ldx, width, p, sms, st);
}

template <int MODE>
int g4_tensor_run(const void *x, int type, int64_t ldx, const G4TensorArgs &a, cudaStream_t st) {
    if (type == QNN_F32) return g4_tensor_pick<MODE, float>(x, ldx, a, st);
    if (type == QNN_BF16) return g4_tensor_pick<MODE, __nv_bfloat16>(x, ldx, a, st);
    return g4_tensor_pick<MODE, __half>(x, ldx, a, st);
}

}  // namespace
