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

// Few rows for each expert: the form that needs no full tile (g4_rows.cu).
bool few_rows(int type, int64_t rows, int experts) { return rows <= (type == QNN_F32 ? 2 : 4) * (int64_t)experts; }
// And for one matrix.  Drawn at one size: 16 x 16384 x 8192 in fp16 takes 35 us there and 22.5 us in 32-row tiles of the tensor-memory
// form.  (A small matrix has few such tiles: 16 x 1024 x 1024 makes eight.)
bool few_rows_one(int type, int64_t rows) { return rows <= (type == QNN_F32 ? 4 : 8); }

size_t product_workspace(bool data, const void *x, int type, int64_t rows, int64_t ldx, int experts, int width, int features) {
    const G4Plan plan = g4_tensor_plan(data, type == QNN_F32, rows, experts, features, g4_tiles(width));
    return (g4_rows_in_place(x, type, ldx) ? 0 : g4_staged_bytes(type, rows, width)) + g4_sums_bytes(plan, rows, features);
}

int product(bool data, const void *x, int type, int64_t rows, int64_t ldx, const int32_t *offsets, int experts, const G4Weights &w, void *out,
            int64_t ldo, void *workspace, cudaStream_t st) {
    const int width = data ? w.n : w.k;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    G4TensorArgs a{w, offsets, experts, (int)rows, out, ldo, nullptr};
    if (!g4_rows_in_place(x, type, ldx)) {
        const int rc = qnn_stage_rows(x, type, ldx, (int)rows, width, ws, st);
        if (rc != QNN_OK) return rc;
        x = ws;
        ldx = g4_padded_width(width);
        ws += g4_staged_bytes(type, rows, width);
    }
    a.sums = ws;
    return data ? qnn_g4_tensor_data(x, type, ldx, a, st) : qnn_g4_tensor_fwd(x, type, ldx, a, st);
}

}  // namespace

G4Plan g4_tensor_plan(bool data, bool fp32, int64_t rows, int experts, int features, int steps) {
    struct Tile {
        int tokens, blocks, cycles_fwd, cycles_data;
    };
    static const Tile narrow[] = {{32, 1, 560, 760}, {64, 1, 620, 980}, {128, 2, 820, 1020}, {256, 2, 1050, 1280}};
    static const Tile split3[] = {{32, 1, 900, 1100}, {64, 1, 1500, 1700}};
    G4Plan best = {64, 1, steps};
    int64_t least = INT64_MAX;
    for (int i = 0; i < (fp32 ? 2 : 4); ++i) {
        const Tile &t = fp32 ? split3[i] : narrow[i];
        // blocks of rows: experts with rows get half to one and a half times the mean
        const int64_t active = rows < experts ? rows : experts;
        int64_t slots = 0;
        if (experts == 1) slots = (rows + t.tokens - 1) / t.tokens;
        else
            for (int u = 0; u < 8; ++u) {
                const int64_t r = rows * (9 + 2 * u) / (16 * active);
                slots += active * (((r > 0 ? r : 1) + t.tokens - 1) / t.tokens);
            }
        if (experts > 1) slots = (slots + 7) / 8;
        const int64_t tiles = slots * ((g4_tiles(features) + t.blocks - 1) / t.blocks), units = 148 / t.blocks;
        for (int parts = 1; parts <= 8; ++parts) {
            const int each = (steps + parts - 1) / parts;
            if (parts > 1 && (each < 2 || (steps + each - 1) / each != parts)) continue;
            const int64_t rounds = (tiles * parts + units - 1) / units;
            const int64_t cost = rounds * ((int64_t)each * (data ? t.cycles_data : t.cycles_fwd) + 3000) +
                                 (parts > 1 ? 4000 + (int64_t)parts * rows * features / 400 : 0);
            if (cost < least) { least = cost; best = {t.tokens, parts, each}; }
        }
    }
    return best;
}

extern "C" size_t qnn_g4_matvec_workspace(const void *x, int type, int64_t rows, int64_t ldx, int n, int k) {
    if (!g4_type_ok(type) || !g4_dims_ok(1, n, k) || rows <= 0 || rows >= G4_MAX_ROWS || few_rows_one(type, rows)) return 0;
    return product_workspace(false, x, type, rows, ldx, 1, k, n);
}

extern "C" int qnn_g4_matvec(const void *x, int type, int64_t rows, int64_t ldx, const uint32_t *codes, const uint8_t *scales,
                             const float *alpha, int n, int k, int group, void *y, int64_t ldy, void *workspace,
                             size_t workspace_bytes, void *stream) {
    int rc = check_weights(1, codes, scales, alpha, n, k, group);
    if (rc == QNN_OK) rc = check_rows(x, type, rows, ldx, k);
    if (rc == QNN_OK) rc = check_rows(y, type, rows, ldy, n);
    if (rc == QNN_OK) rc = check_workspace(workspace, workspace_bytes, qnn_g4_matvec_workspace(x, type, rows, ldx, n, k));
    if (rc != QNN_OK || rows == 0) return rc;
    const G4Weights w{codes, scales, alpha, n, k, group, g4_tiles(n), g4_tiles(k)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (few_rows_one(type, rows)) return qnn_g4_rows(x, type, ldx, (int)rows, nullptr, 1, w, y, ldy, (int)rows, st);
    return product(false, x, type, rows, ldx, nullptr, 1, w, y, ldy, workspace, st);
}

extern "C" size_t qnn_g4_expert_gemm_workspace(const void *x, int type, int64_t rows, int64_t ldx, int experts, int n, int k) {
    if (!g4_type_ok(type) || !g4_dims_ok(experts, n, k) || rows <= 0 || rows >= G4_MAX_ROWS || few_rows(type, rows, experts)) return 0;
    return product_workspace(false, x, type, rows, ldx, experts, k, n);
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
    if (few_rows(type, rows, experts))
        return qnn_g4_rows(x, type, ldx, (int)rows, offsets, experts, w, y, ldy, type == QNN_F32 ? 2 : 8, st);
    return product(false, x, type, rows, ldx, offsets, experts, w, y, ldy, workspace, st);
}

extern "C" size_t qnn_g4_expert_backward_data_workspace(const void *dy, int type, int64_t rows, int64_t lddy, int experts, int n,
                                                        int k) {
    if (!g4_type_ok(type) || !g4_dims_ok(experts, n, k) || rows <= 0 || rows >= G4_MAX_ROWS) return 0;
    return product_workspace(true, dy, type, rows, lddy, experts, n, k);
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
    return product(true, dy, type, rows, lddy, offsets, experts, w, dx, lddx, workspace, static_cast<cudaStream_t>(stream));
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
    const bool stage_dy = !g4_rows_in_place(dy, type, lddy), stage_x = !g4_rows_in_place(x, type, ldx);
    void *to_dy = ws, *to_x = ws + (stage_dy ? g4_staged_bytes(type, rows, n) : 0);
    if (stage_dy && stage_x) rc = qnn_stage_rows_two(dy, lddy, n, to_dy, x, ldx, k, to_x, type, (int)rows, st);
    else if (stage_dy) rc = qnn_stage_rows(dy, type, lddy, (int)rows, n, to_dy, st);
    else if (stage_x) rc = qnn_stage_rows(x, type, ldx, (int)rows, k, to_x, st);
    if (rc != QNN_OK) return rc;
    if (stage_dy) { dy = to_dy; lddy = g4_padded_width(n); }
    if (stage_x) { x = to_x; ldx = g4_padded_width(k); }
    return qnn_expert_wgrad(x, ldx, dy, lddy, type, offsets, experts, (int)rows, n, k, gw, parts, st);
}

extern "C" int qnn_g4_plan(int product, int one, int type, int64_t rows, int experts, int n, int k, int *tile, int *parts) {
    if (product < 0 || product > 2 || !tile || !parts || !g4_type_ok(type) || !g4_dims_ok(experts, n, k) || rows <= 0 ||
        (one && (product != 0 || experts != 1)))
        return QNN_E_ARG;
    if (rows >= G4_MAX_ROWS) return QNN_E_RANGE;
    if (product == 2) {
        qnn_expert_wgrad_plan(rows, experts, n, k, tile, parts);
        return QNN_OK;
    }
    const bool data = product == 1;
    const G4Plan plan = g4_tensor_plan(data, type == QNN_F32, rows, experts, data ? k : n, g4_tiles(data ? n : k));
    const bool few = !data && (one ? few_rows_one(type, rows) : few_rows(type, rows, experts));
    *tile = few ? 0 : plan.tokens;
    *parts = few ? 1 : plan.parts;
    return QNN_OK;
}
