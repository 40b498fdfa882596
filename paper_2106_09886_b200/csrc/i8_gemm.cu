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

// The form that ends first by an estimate in nanoseconds: what a launch costs, and for each round of blocks a step of 128 elements
// and a fixed part (first copies, results).  Fitted to 323 sizes (1 to 8192 rows, n 200 to 16384, k 192 to 16384; times in a
// replayed graph), where the choice is 1.9 % off the best form on average and 22 % at most.  Two sides of it: 301 x 4096 x 4096
// takes 13.6 us in one block's tiles of 128 tokens and 10.4 in a pair's; 64 x 4096 x 4096 7.2 us in 32-token tiles with four ranks
// and 9.9 by pairs.  Blocks of tiles up to 64 tokens go two to an SM, and share it when more than 148 run (step + 31 %, fixed part
// x 4.5); clusters of four and eight do not fill every group of SMs.  Sized for 148 SMs.
I8Plan i8_plan(int64_t rows, int n, int k) {
    struct Form {
        int tile, launch, step, fixed;
    };
    static const Form split[] = {{16, 1330, 200, 368}, {32, 2260, 209, 375}, {64, 3170, 260, 499}, {128, 0, 222, 5390}};
    static const Form pair[] = {{128, 2950, 181, 1340}, {256, 2970, 318, 2280}};
    static const int join[] = {0, 740, 470, 0}, places[] = {148, 148, 136, 112};
    const double steps = (double)((k + I8_STEP - 1) / I8_STEP), wide = (double)((n + 255) / 256), narrow = (double)((n + 127) / 128);
    I8Plan best = {256, 0};
    double least = 1e300;
    for (const Form &f : split) {
        if (f.tile > 16 && f.tile >= 2 * rows) break;                              // half of such a tile would be empty
        if (rows > (int64_t)f.tile * 65535) continue;                              // (tiles of tokens are a grid's second dimension)
        const double tiles = narrow * (double)((rows + f.tile - 1) / f.tile);
        const int together = f.tile <= 64 ? 2 : 1;
        for (int l = 0; l < 4 && (1 << l) <= steps; ++l) {
            const double blocks = tiles * (1 << l), rounds = ceil(blocks / (places[l] * together)), each = ceil(steps / (1 << l));
            const double shared = together == 1 || blocks <= 148.0 ? 0.0 : blocks < 296.0 ? blocks / 148.0 - 1.0 : 1.0;
            const double cost = f.launch + rounds * (each * f.step * (1.0 + 0.31 * shared) + f.fixed * (1.0 + 3.5 * shared)) + join[l];
            if (cost < least) { least = cost; best = {f.tile, 1 << l}; }
        }
    }
    if (rows > 32)
        for (const Form &f : pair) {
            const double rounds = ceil(wide * (double)((rows + f.tile - 1) / f.tile) / 74.0), cost = f.launch + rounds * (steps * f.step + f.fixed);
            if (cost < least) { least = cost; best = {f.tile, 0}; }
        }
    return best;
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
    if (plan.ranks == 0) return plan.tile == 128 ? run_pair<128, T>(o, p, st) : run_pair<256, T>(o, p, st);
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
