// Products of rows in 8 bits: argument checks, the choice of kernel, tile and split.
#include "i8_gemm.cuh"

namespace {

constexpr int I8_MAX_K = 131071;                         // 128 * 128 * k stays below 2^31
constexpr int64_t I8_MAX_ROWS = (1ll << 31) / 256;

struct I8Operands {
    const int8_t *x, *w;
    int64_t ldx, ldw;
    int k;
};

// tile: tokens; ranks 0: a pair of blocks and 256 features, else the blocks of a cluster that share the contraction of 128 features.
struct I8Plan {
    int tile, ranks;
};

I8Plan i8_plan(int64_t rows, int n, int k) {
    const int64_t steps = (k + I8_STEP - 1) / I8_STEP;
    const int64_t pairs = ((n + 255) / 256) * ((rows + 255) / 256);
    if (pairs >= 74) return {256, 0};
    const int tile = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128, at_once = tile <= 64 ? 296 : 148;
    const int64_t tiles = (int64_t)((n + 127) / 128) * ((rows + tile - 1) / tile);
    int ranks = 1;
    int64_t best = INT64_MAX;
    for (int r = 1; r <= 8 && r <= steps; r *= 2) {
        const int64_t rounds = (tiles * r + at_once - 1) / at_once, cost = rounds * ((steps + r - 1) / r + 8) + (r > 1 ? 4 : 0);
        if (cost < best) { best = cost; ranks = r; }
    }
    return {tile, ranks};
}

template <auto KERNEL, class... A>
int i8_launch(dim3 grid, int threads, int smem, int cluster, cudaStream_t st, A... args) {
    if (!allow_shared_memory<KERNEL>(smem)) return QNN_E_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    LaunchAttrs attrs(cluster);
    cfg.attrs = attrs.a;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, KERNEL, args...) == cudaSuccess) return QNN_OK;
    cudaGetLastError();
    return QNN_E_CUDA;
}

template <int TN, class T> int run_split(const I8Operands &o, const I8Params &p, int ranks, cudaStream_t st) {
    using L = I8Split<TN>;
    CUtensorMap w, x;
    if (!make_map_i8(&w, o.w, p.n, o.k, o.ldw, 128) || !make_map_i8(&x, o.x, p.rows, o.k, o.ldx, TN)) return QNN_E_CUDA;
    const int64_t ttiles = ((int64_t)p.rows + TN - 1) / TN;
    if (ttiles > 65535) return QNN_E_RANGE;
    int log_ranks = 0;
    while (1 << log_ranks < ranks) ++log_ranks;
    return i8_launch<i8_split_kernel<TN, T>>(dim3((p.n + 127) / 128 << log_ranks, (unsigned)ttiles), L::THREADS, L::TOTAL, ranks, st, w, x, p, log_ranks);
}
template <int TN, class T> int run_pair(const I8Operands &o, I8Params p, cudaStream_t st) {
    using L = I8Pair<TN, T>;
    CUtensorMap w, x;
    if (!make_map_i8(&w, o.w, p.n, o.k, o.ldw, 128) || !make_map_i8(&x, o.x, p.rows, o.k, o.ldx, L::XROWS)) return QNN_E_CUDA;
    p.ftiles = (p.n + 255) / 256;
    p.ttiles = (p.rows + TN - 1) / TN;
    p.band = 8;
    const int64_t items = (int64_t)p.ftiles * p.ttiles;
    if (items > 0x3FFFFFFF || (int64_t)p.band * p.ftiles > 0x3FFFFFFF) return QNN_E_RANGE;
    const int sms = sm_count(), most = sms / 2;
    if (most < 1) return QNN_E_CUDA;
    return i8_launch<i8_pair_kernel<TN, T>>(dim3((unsigned)(items < most ? items : most) * 2), L::THREADS, L::TOTAL, 2, st, w, x, p);
}
template <class T> int run(const I8Operands &o, const I8Params &p, cudaStream_t st) {
    const I8Plan plan = i8_plan(p.rows, p.n, o.k);
    if (plan.ranks == 0) return run_pair<256, T>(o, p, st);
    switch (plan.tile) {
        case 16: return run_split<16, T>(o, p, plan.ranks, st);
        case 32: return run_split<32, T>(o, p, plan.ranks, st);
        case 64: return run_split<64, T>(o, p, plan.ranks, st);
        default: return run_split<128, T>(o, p, plan.ranks, st);
    }
}

int check_operand(const int8_t *codes, const float *scales, int64_t ld, int k) {
    if (!codes || !scales || ld < k) return QNN_E_ARG;
    return qnn_aligned(codes, 16) && ld % 16 == 0 && qnn_aligned(scales, 4) ? QNN_OK : QNN_E_ALIGN;
}

}  // namespace

extern "C" int qnn_i8_gemm(const int8_t *x, const float *x_scales, int64_t rows, int64_t ldx, const int8_t *w, const float *w_scales, int n,
                           int k, int64_t ldw, const float *bias, int type, void *y, int64_t ldy, void *stream) {
    if (!g4_type_ok(type) || rows < 0 || n < 1 || k < 1) return QNN_E_ARG;
    if (k > I8_MAX_K || n > G4_MAX_DIM || rows >= I8_MAX_ROWS) return QNN_E_RANGE;
    int rc = check_operand(w, w_scales, ldw, k);
    if (rc == QNN_OK && bias && !qnn_aligned(bias, 4)) rc = QNN_E_ALIGN;
    if (rc != QNN_OK || rows == 0) return rc;
    if ((rc = check_operand(x, x_scales, ldx, k)) != QNN_OK) return rc;
    if (!y || ldy < n) return QNN_E_ARG;
    if (!qnn_aligned(y, g4_type_bytes(type))) return QNN_E_ALIGN;
    I8Params p{};
    p.x_scales = x_scales; p.w_scales = w_scales; p.bias = bias;
    p.out = y; p.ldo = ldy;
    p.rows = (int)rows; p.n = n; p.steps = (k + I8_STEP - 1) / I8_STEP;
    p.out_vec = qnn_aligned(y, 16) && ldy * g4_type_bytes(type) % 16 == 0;
    if (!(p.err = qnn_tc_error_word())) return QNN_E_CUDA;
    p.wait_limit = WAIT_LIMIT;
    const I8Operands o{x, w, ldx, ldw, k};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (type == QNN_F32) return run<float>(o, p, st);
    if (type == QNN_BF16) return run<__nv_bfloat16>(o, p, st);
    return run<__half>(o, p, st);
}

extern "C" int qnn_i8_plan(int64_t rows, int n, int k, int *tile, int *ranks) {
    if (rows < 1 || n < 1 || k < 1 || !tile || !ranks) return QNN_E_ARG;
    if (k > I8_MAX_K || n > G4_MAX_DIM || rows >= I8_MAX_ROWS) return QNN_E_RANGE;
    const I8Plan plan = i8_plan(rows, n, k);
    *tile = plan.tile;
    *ranks = plan.ranks;
    return QNN_OK;
}
