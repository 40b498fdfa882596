// Products with group-scaled 4-bit weights, grouped by expert: entry points and kernels.
#include "g4_stage.cuh"
#include "g4_tensor_api.cuh"

namespace {

__device__ __forceinline__ float g4_weight(const G4Weights &w, int e, int j, int i) {
    const int64_t tile = ((int64_t)e * w.tiles_n + j / G4_TILE) * w.tiles_k + i / G4_TILE;
    const int r = j % G4_TILE, c = i % G4_TILE;
    const uint32_t word = __ldg(w.codes + tile * G4_TILE_WORDS + ((c / 8 % 4) * G4_TILE + r) * 4 + c / 32);
    const int t = (word >> ((c % 8 / 2) * 4 + (c % 2) * 16)) & 15;
    const float s = g4_scale_f32(__ldg(w.scales + (tile * (G4_TILE / w.group) + c / w.group) * G4_TILE + r));
    return s * (float)(2 * t - 15);
}

// One 64 x 64 tile of the result, 4 x 4 elements a thread, 16 steps of the contraction at a time.
// OP 0: y[r][j], contraction over i.  OP 1: dx[r][i], over j.  OP 2: gw[e][j][i], over e's rows.
template <int OP, class T>
__global__ void __launch_bounds__(256) simple_kernel(const T *a, int64_t lda, const T *b, int64_t ldb, int rows,
                                                    const int32_t *offsets, int experts, G4Weights w, void *out, int64_t ldo) {
    __shared__ float sa[16][65], sb[16][65];
    int e, first, last, m_count, c0 = blockIdx.x * 64, m0;
    const int n_cols = OP == 0 ? w.n : w.k;
    if (OP == 2) {
        e = blockIdx.z;
        expert_rows(offsets, e, rows, first, last);
        m0 = blockIdx.y * 64;
        m_count = w.n;
    } else {
        const ExpertSlot s = expert_slot(offsets, experts, rows, 64, blockIdx.y);
        if (s.expert < 0) return;
        e = s.expert; first = s.first; last = s.last; m0 = s.first; m_count = s.last;
    }
    const int len = OP == 0 ? w.k : (OP == 1 ? w.n : max(0, last - first));
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int p0 = 0; p0 < len; p0 += 16) {
        for (int v = threadIdx.x; v < 64 * 16; v += 256) {
            const int p = OP == 2 ? v / 64 : v % 16, m = OP == 2 ? v % 64 : v / 16;
            const int pp = p0 + p, mm = m0 + m, cc = c0 + m;
            float av = 0.0f, bv = 0.0f;
            if (pp < len && mm < m_count) av = real_load(OP == 2 ? a + (int64_t)(first + pp) * lda + mm : a + (int64_t)mm * lda + pp);
            if (pp < len && cc < n_cols)
                bv = OP == 0 ? g4_weight(w, e, cc, pp) : OP == 1 ? g4_weight(w, e, pp, cc) : real_load(b + (int64_t)(first + pp) * ldb + cc);
            sa[p][m] = av;
            sb[p][m] = bv;
        }
        __syncthreads();
        for (int p = 0; p < 16; ++p)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j) acc[i][j] = __fmaf_rn(sa[p][ty * 4 + i], sb[p][tx * 4 + j], acc[i][j]);
        __syncthreads();
    }
    const float alpha = OP == 2 ? 1.0f : __ldg(w.alpha + e);
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int m = m0 + ty * 4 + i, c = c0 + tx * 4 + j;
            if (m >= m_count || c >= n_cols) continue;
            if (OP == 2) static_cast<float *>(out)[((int64_t)e * w.n + m) * ldo + c] = acc[i][j];
            else real_store(static_cast<T *>(out) + (int64_t)m * ldo + c, acc[i][j] * alpha);
        }
}

template <int OP, class T>
int simple(const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, const int32_t *offsets, int experts,
           const G4Weights &w, void *out, int64_t ldo, cudaStream_t st) {
    const int n_cols = OP == 0 ? w.n : w.k;
    dim3 grid((n_cols + 63) / 64, 1, 1);
    if (OP == 2) {
        grid.y = (w.n + 63) / 64;
        grid.z = experts;
    } else {
        const int64_t slots = expert_slots_most(rows, experts, 64);
        if (slots > 65535) return QNN_E_RANGE;
        grid.y = (unsigned)slots;
    }
    simple_kernel<OP, T><<<grid, 256, 0, st>>>(static_cast<const T *>(a), lda, static_cast<const T *>(b), ldb, (int)rows, offsets,
                                               experts, w, out, ldo);
    return qnn_launch_status();
}

template <int OP>
int by_type(int type, const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows, const int32_t *offsets, int experts,
            const G4Weights &w, void *out, int64_t ldo, cudaStream_t st) {
    if (type == QNN_F32) return simple<OP, float>(a, lda, b, ldb, rows, offsets, experts, w, out, ldo, st);
    if (type == QNN_BF16) return simple<OP, __nv_bfloat16>(a, lda, b, ldb, rows, offsets, experts, w, out, ldo, st);
    return simple<OP, __half>(a, lda, b, ldb, rows, offsets, experts, w, out, ldo, st);
}

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

extern "C" size_t qnn_expert_backward_weights_workspace(const void *, const void *, int, int64_t, int64_t, int64_t, int, int, int) {
    return 0;
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
    if ((n + 63) / 64 > 65535) return QNN_E_RANGE;
    const G4Weights w{nullptr, nullptr, nullptr, n, k, 128, g4_tiles(n), g4_tiles(k)};
    return by_type<2>(type, dy, lddy, x, ldx, rows, offsets, experts, w, gw, k, static_cast<cudaStream_t>(stream));
}
