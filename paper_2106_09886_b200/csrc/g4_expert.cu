// Products with group-scaled 4-bit weights: entry points, argument checks and the choice between the few-row and the
// tensor-memory kernels.
#include "g4_stage.cuh"
#include "g4_tensor_api.cuh"

namespace {

int check_weights(int experts, const uint32_t *codes, const uint8_t *scales, const float *alpha, int n, int k, int group) {
    if (!codes || !scales || !alpha || !g4_dims_ok(experts, n, k) || !g4_group_ok(group)) return QNN_E_ARG;
    if (!qnn_aligned(codes, 16) || !qnn_aligned(scales, 16) || !qnn_aligned(alpha, 4)) return QNN_E_ALIGN;
    return QNN_OK;
}

int check_rows(const void *p, int type, int64_t rows, int64_t ld, int width) {
    if (!g4_type_ok(type) || rows < 0 || ld < width) return QNN_E_ARG;
    if (rows > 0 && !p) return QNN_E_ARG;
    if (rows >= G4_MAX_ROWS) return QNN_E_RANGE;
    return qnn_aligned(p, g4_type_bytes(type)) ? QNN_OK : QNN_E_ALIGN;
}

int check_workspace(const void *ws, size_t have, size_t need) {
    if (need == 0) return QNN_OK;
    if (!ws || have < need) return QNN_E_ARG;
    return qnn_aligned(ws, 256) ? QNN_OK : QNN_E_ALIGN;
}

}  // namespace

extern "C" int qnn_g4_matvec(const void *x, int type, int64_t rows, int64_t ldx, const uint32_t *codes, const uint8_t *scales,
                             const float *alpha, int n, int k, int group, void *y, int64_t ldy, void *stream) {
    int rc = check_weights(1, codes, scales, alpha, n, k, group);
    if (rc == QNN_OK) rc = check_rows(x, type, rows, ldx, k);
    if (rc == QNN_OK) rc = check_rows(y, type, rows, ldy, n);
    if (rc != QNN_OK || rows == 0) return rc;
    const G4Weights w{codes, scales, alpha, n, k, group, g4_tiles(n), g4_tiles(k)};
    return qnn_g4_rows(x, type, ldx, (int)rows, nullptr, 1, w, y, ldy, rows < 32 ? (int)rows : 32, static_cast<cudaStream_t>(stream));
}

// Few rows for each expert: the form that reads the codes once for a handful of rows and splits the contraction.
static bool g4_few_rows(int64_t rows, int experts) { return rows <= 8 * (int64_t)experts; }

extern "C" size_t qnn_g4_expert_gemm_workspace(const void *x, int type, int64_t rows, int64_t ldx, int experts, int n, int k) {
    if (!g4_type_ok(type) || !g4_dims_ok(experts, n, k) || rows <= 0 || rows >= G4_MAX_ROWS) return 0;
    return g4_few_rows(rows, experts) || g4_rows_in_place(x, type, ldx) ? 0 : g4_staged_bytes(type, rows, k);
}

extern "C" int qnn_g4_expert_gemm(const void *x, int type, int64_t rows, int64_t ldx, const int32_t *offsets, int experts,
                                  const uint32_t *codes, const uint8_t *scales, const float *alpha, int n, int k, int group,
                                  void *y, int64_t ldy, void *workspace, size_t workspace_bytes, void *stream) {
    int rc = check_weights(experts, codes, scales, alpha, n, k, group);
    if (rc == QNN_OK && !offsets) rc = QNN_E_ARG;
    if (rc == QNN_OK && !qnn_aligned(offsets, 4)) rc = QNN_E_ALIGN;
    if (rc == QNN_OK) rc = check_rows(x, type, rows, ldx, k);
    if (rc == QNN_OK) rc = check_rows(y, type, rows, ldy, n);
    if (rc == QNN_OK) rc = check_workspace(workspace, workspace_bytes, qnn_g4_expert_gemm_workspace(x, type, rows, ldx, experts, n, k));
    if (rc != QNN_OK || rows == 0) return rc;
    const G4Weights w{codes, scales, alpha, n, k, group, g4_tiles(n), g4_tiles(k)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (g4_few_rows(rows, experts)) return qnn_g4_rows(x, type, ldx, (int)rows, offsets, experts, w, y, ldy, 8, st);
    const G4TensorArgs a{w, offsets, experts, (int)rows, y, ldy};
    if (g4_rows_in_place(x, type, ldx)) return qnn_g4_tensor_fwd(x, type, ldx, a, st);
    rc = qnn_stage_rows(x, type, ldx, (int)rows, k, workspace, st);
    return rc != QNN_OK ? rc : qnn_g4_tensor_fwd(workspace, type, g4_padded_width(k), a, st);
}

extern "C" size_t qnn_g4_expert_backward_data_workspace(const void *dy, int type, int64_t rows, int64_t lddy, int experts, int n,
                                                        int k) {
    if (!g4_type_ok(type) || !g4_dims_ok(experts, n, k) || rows <= 0 || rows >= G4_MAX_ROWS) return 0;
    return g4_rows_in_place(dy, type, lddy) ? 0 : g4_staged_bytes(type, rows, n);
}

extern "C" int qnn_g4_expert_backward_data(const void *dy, int type, int64_t rows, int64_t lddy, const int32_t *offsets,
                                           int experts, const uint32_t *codes, const uint8_t *scales, const float *alpha, int n,
                                           int k, int group, void *dx, int64_t lddx, void *workspace, size_t workspace_bytes,
                                           void *stream) {
    int rc = check_weights(experts, codes, scales, alpha, n, k, group);
    if (rc == QNN_OK && !offsets) rc = QNN_E_ARG;
    if (rc == QNN_OK && !qnn_aligned(offsets, 4)) rc = QNN_E_ALIGN;
    if (rc == QNN_OK) rc = check_rows(dy, type, rows, lddy, n);
    if (rc == QNN_OK) rc = check_rows(dx, type, rows, lddx, k);
    if (rc == QNN_OK)
        rc = check_workspace(workspace, workspace_bytes, qnn_g4_expert_backward_data_workspace(dy, type, rows, lddy, experts, n, k));
    if (rc != QNN_OK || rows == 0) return rc;
    const G4Weights w{codes, scales, alpha, n, k, group, g4_tiles(n), g4_tiles(k)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const G4TensorArgs a{w, offsets, experts, (int)rows, dx, lddx};
    if (g4_rows_in_place(dy, type, lddy)) return qnn_g4_tensor_data(dy, type, lddy, a, st);
    rc = qnn_stage_rows(dy, type, lddy, (int)rows, n, workspace, st);
    return rc != QNN_OK ? rc : qnn_g4_tensor_data(workspace, type, g4_padded_width(n), a, st);
}

extern "C" size_t qnn_expert_backward_weights_workspace(const void *dy, const void *x, int type, int64_t rows, int64_t lddy,
                                                        int64_t ldx, int experts, int n, int k) {
    if (!g4_type_ok(type) || !g4_dims_ok(experts, n, k) || rows <= 0 || rows >= G4_MAX_ROWS) return 0;
    return qnn_expert_wgrad_parts_bytes(rows, experts, n, k) + (g4_rows_in_place(dy, type, lddy) ? 0 : g4_staged_bytes(type, rows, n)) +
           (g4_rows_in_place(x, type, ldx) ? 0 : g4_staged_bytes(type, rows, k));
}

extern "C" int qnn_expert_backward_weights(const void *dy, const void *x, int type, int64_t rows, int64_t lddy, int64_t ldx,
                                           const int32_t *offsets, int experts, int n, int k, float *gw, void *workspace,
                                           size_t workspace_bytes, void *stream) {
    if (!offsets || !gw || !g4_dims_ok(experts, n, k)) return QNN_E_ARG;
    if (!qnn_aligned(offsets, 4) || !qnn_aligned(gw, 4)) return QNN_E_ALIGN;
    int rc = check_rows(dy, type, rows, lddy, n);
    if (rc == QNN_OK) rc = check_rows(x, type, rows, ldx, k);
    if (rc == QNN_OK)
        rc = check_workspace(workspace, workspace_bytes,
                             qnn_expert_backward_weights_workspace(dy, x, type, rows, lddy, ldx, experts, n, k));
    if (rc != QNN_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0)
        return cudaMemsetAsync(gw, 0, (size_t)experts * n * k * sizeof(float), st) == cudaSuccess ? QNN_OK : QNN_E_CUDA;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    float *parts = reinterpret_cast<float *>(ws);
    ws += qnn_expert_wgrad_parts_bytes(rows, experts, n, k);
    if (!g4_rows_in_place(dy, type, lddy)) {
        if ((rc = qnn_stage_rows(dy, type, lddy, (int)rows, n, ws, st)) != QNN_OK) return rc;
        dy = ws;
        lddy = g4_padded_width(n);
        ws += g4_staged_bytes(type, rows, n);
    }
    if (!g4_rows_in_place(x, type, ldx)) {
        if ((rc = qnn_stage_rows(x, type, ldx, (int)rows, k, ws, st)) != QNN_OK) return rc;
        x = ws;
        ldx = g4_padded_width(k);
    }
    return qnn_expert_wgrad(x, ldx, dy, lddy, type, offsets, experts, (int)rows, n, k, gw, parts, st);
}
