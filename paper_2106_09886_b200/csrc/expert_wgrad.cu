// Weight gradients of products grouped by expert: gw[e][j][i] = sum over e's rows of dy[r][j] * x[r][i], fp32.
//
// Both operands are read with the contraction (rows) outermost, exactly as they lie in memory: boxes of 64 columns x 64
// rows, MN-major for the tensor cores.  The lanes of an accumulator are columns i of x and its columns are features j, so
// that a warp stores 32 neighbouring elements of a row of gw.  An expert's last block of rows reaches into the next
// expert's: one warp clears those rows in shared memory before the instructions see them (a zero in one operand alone
// would not do, as the other may hold NaN or infinity).
// fp32: both operands are three bf16 parts, below 1, 2^-7 and 2^-15 of the leading bit; the six products of parts whose bound is
// 2^-15 or more are summed, the three others together are below 2^-21 of the product.
//
// The tensor cores cut a sum towards zero at every addition, so a sum stays in tensor memory for 16 instructions (256 rows;
// fp32: one block of rows and its six products, smallest first) and the result warps add those to nearest in registers.
// Bound: writing gw (4 bytes an element) up to some 600 rows an expert, the matrix instructions beyond.  With few tiles
// the rows are split over the blocks too; the parts are added in a fixed order by a second kernel.
// Measured in a replayed graph, and as calls back to back: 4096 rows, eight experts 2048 x 4096, bf16: 90 and 101 us (268 MB of
// gw at 3.0 and 2.7 TB/s); 8192 rows, one expert 4096 x 4096: 207 and 244 us, 1.33 and 1.13 PFLOP/s.
#include "g4_stage.cuh"
#include "g4_tensor.cuh"

namespace {

struct WgradParams {
    const int32_t *offsets;
    int experts, rows, n, k;
    float *gw;
    int64_t part_stride;                  // elements between the results of two parts of the rows
    int itiles, jtiles;                   // tiles of 128 * CG columns of x, of TN features
    int parts;                            // parts of an expert's rows
    unsigned int *err;
    unsigned int wait_limit;
};

constexpr int W_THREADS = 384;            // warps: 0 TMA, 1 matrix instructions, 2 tail rows (and owner of the tensor memory),
                                          // 3 idle, 4-11 results: a warp has a quarter of the lanes and half of the columns

template <int CG, int TN>
struct WShape {
    static constexpr int ROWS = 64;                             // rows of a stage
    static constexpr int BLOCK = ROWS * 128;                    // 64 columns of them
    static constexpr int B_COLS = TN / CG;                      // features this block stages
    static constexpr int A_BYTES = 2 * BLOCK;
    static constexpr int STAGE = A_BYTES + B_COLS / 64 * BLOCK;
    static constexpr int STAGES = 216 * 1024 / STAGE > 8 ? 8 : 216 * 1024 / STAGE;
    static constexpr int BAR_OFF = STAGES * STAGE;
    static constexpr int TOTAL = BAR_OFF + (3 * STAGES + 5) * 8 + 16 + 1024;
    static_assert(B_COLS % 64 == 0 && 2 * TN <= 512 && TOTAL <= 227 * 1024 && TOTAL > 114 * 1024, "tile");   // (one block an SM)
};

// One tile of one expert: rows [first, last) of its part, first column of x, first feature.
struct WTile {
    int expert, part, first, last, i0, j0;
};
__device__ __noinline__ WTile wgrad_tile_of(const int32_t *offsets, int rows, int itiles, int jtiles, int parts, int i_step, int j_step, int t) {
    WTile w;
    w.i0 = t % itiles * i_step; t /= itiles;
    w.j0 = t % jtiles * j_step; t /= jtiles;
    w.part = t % parts;
    w.expert = t / parts;
    expert_rows(offsets, w.expert, rows, w.first, w.last);
    if (parts > 1) {                      // whole blocks of rows, as evenly as they go (at most 148 parts: no overflow)
        const int blocks = max(0, w.last - w.first + 63) / 64;
        const int lo = blocks * w.part / parts, hi = blocks * (w.part + 1) / parts, base = w.first;
        w.last = min(w.last, base + hi * 64);
        w.first = base + lo * 64;
    }
    return w;
}
template <int CG, int TN> __device__ __forceinline__ WTile wgrad_tile(const WgradParams &p, int t) {
    return wgrad_tile_of(p.offsets, p.rows, p.itiles, p.jtiles, p.parts, 128 * CG, TN, t);
}

// Products of parts, smallest first: (x part, dy part).
__device__ __forceinline__ int pair_x(int q) { return (0x201010 >> (4 * (5 - q))) & 15; }
__device__ __forceinline__ int pair_dy(int q) { return (0x021100 >> (4 * (5 - q))) & 15; }

template <int CG, int TN, class T>
__global__ void __launch_bounds__(W_THREADS, 1) expert_wgrad_kernel(const __grid_constant__ CUtensorMap map_x,
                                                                   const __grid_constant__ CUtensorMap map_dy, const WgradParams p) {
    using L = WShape<CG, TN>;
    constexpr int PAIRS = G4Type<T>::PARTS == 1 ? 1 : 6;
    constexpr int CHUNK = PAIRS == 1 ? 4 : PAIRS;                // stages that are added up in tensor memory
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t *landed = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF);     // each block: its copies of a stage
    uint64_t *ready = landed + L::STAGES;                                   // leader: both blocks' stages are fit to be read
    uint64_t *empty = ready + L::STAGES;                                    // each block
    uint64_t *acc_full = empty + L::STAGES;                                 // each block
    uint64_t *acc_empty = acc_full + 2;                                     // leader
    uint64_t *finish = acc_empty + 2;                                       // every instruction has completed
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(finish + 1);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int rank = (int)pair_rank<CG>();
    const int first_work = blockIdx.x / CG, work_stride = gridDim.x / CG;
    const int work = p.experts * p.parts * p.itiles * p.jtiles;

    if (threadIdx.x == 0) {
#pragma unroll 1
        for (int s = 0; s < L::STAGES; ++s) { mbar_init(&landed[s], 1); mbar_init(&ready[s], CG); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 8 * CG); }
        mbar_init(finish, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) pair_tmem_alloc<CG>(tmem_slot, 2 * TN);
    tc_fence_before();
    __syncthreads();
    pair_sync<CG>();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    start_next();
    wait_for_previous();
    auto warp_wait = [&](uint64_t *bar, uint32_t parity, unsigned id) {
        return __all_sync(0xffffffffu, short_wait(bar, parity, abort_flag, id, p.err, p.wait_limit));
    };
    auto stop = [&]() { return __any_sync(0xffffffffu, *abort_flag != 0); };

    if (warp == 0) {
        Ring g;
        long long it = 0;
#pragma unroll 1
        for (int t = first_work; t < work && !stop(); t += work_stride) {
            const WTile w = wgrad_tile<CG, TN>(p, t);
            const int first = w.first, last = w.last, i0 = w.i0 + rank * 128, j0 = w.j0 + rank * L::B_COLS;
            bool ok = true;
#pragma unroll 1
            for (int r = first; ok && r < last; r += L::ROWS)
#pragma unroll 1
                for (int q = 0; q < PAIRS; ++q) {
                    if (!(ok = warp_wait(&empty[g.s], g.ph ^ 1u, 0))) break;
                    if (elect_one()) {
                        mbar_expect_tx(&landed[g.s], L::STAGE);
                        uint8_t *dst = smem + g.s * L::STAGE;
                        const int rx = (PAIRS == 1 ? 0 : pair_x(q) * p.rows) + r, rd = (PAIRS == 1 ? 0 : pair_dy(q) * p.rows) + r;
#pragma unroll
                        for (int b = 0; b < 2; ++b) tma_load_2d(dst + b * L::BLOCK, &map_x, &landed[g.s], i0 + b * 64, rx);
#pragma unroll
                        for (int b = 0; b < L::B_COLS / 64; ++b)
                            tma_load_2d(dst + L::A_BYTES + b * L::BLOCK, &map_dy, &landed[g.s], j0 + b * 64, rd);
                    }
                    __syncwarp();
                    g.next(L::STAGES);
                    ++it;
                }
            if (!ok) break;
        }
        if (*abort_flag && lane == 0) drain_copies_in_flight(landed, it, L::STAGES, p.wait_limit);
    } else if (warp == 2) {               // stages whose rows all belong to the expert pass through
        Ring g;
#pragma unroll 1
        for (int t = first_work; t < work && !stop(); t += work_stride) {
            const WTile w = wgrad_tile<CG, TN>(p, t);
            const int first = w.first, last = w.last;
            bool ok = true;
#pragma unroll 1
            for (int r = first; ok && r < last; r += L::ROWS)
#pragma unroll 1
                for (int q = 0; q < PAIRS; ++q) {
                    if (!(ok = warp_wait(&landed[g.s], g.ph, 1))) break;
                    const int valid = last - r;
                    if (valid < L::ROWS) {
                        const uint32_t stage = smem_u32(smem) + g.s * L::STAGE;
#pragma unroll 1
                        for (int b = 0; b < L::STAGE / L::BLOCK; ++b)
#pragma unroll 1
                            for (int v = valid * 8 + lane; v < L::ROWS * 8; v += 32)
                                sts_128(stage + b * L::BLOCK + v * 16, 0u, 0u, 0u, 0u);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    if (lane == 0) arrive_leader<CG>(&ready[g.s]);
                    g.next(L::STAGES);
                }
            if (!ok) break;
        }
    } else if (warp == 1) {
        if (rank == 0) {
            Ring acc;
            constexpr uint32_t idesc = idesc_f16(G4Type<T>::FMT, 128 * CG, TN, true, true);
            const uint64_t a_desc = smem_desc_mn_sw128(smem_u32(smem), L::BLOCK);
            const uint64_t b_desc = smem_desc_mn_sw128(smem_u32(smem) + L::A_BYTES, L::BLOCK);
            int t = first_work, left = 0, chunk = 0;             // stages left of the tile, stages in this sum
            auto next_tile = [&]() {                             // tiles without rows have no stages
#pragma unroll 1
                for (; left == 0 && t < work; t += work_stride) {
                    const WTile w = wgrad_tile<CG, TN>(p, t);
                    left = (max(0, w.last - w.first) + L::ROWS - 1) / L::ROWS * PAIRS;
                }
                return left > 0;
            };
            bool ok = !stop() && next_tile();
#pragma unroll 1
            for (uint32_t ph = 0; ok; ph ^= 1u) {
#pragma unroll
                for (int g = 0; g < L::STAGES; ++g) {
                    if (chunk == 0 && !(ok = warp_wait(&acc_empty[acc.s], acc.ph ^ 1u, 3))) break;
                    if (!(ok = warp_wait(&ready[g], ph, 1))) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + (uint32_t)(acc.s * TN);
                    const bool done = chunk == CHUNK - 1 || left == 1;
                    if (elect_one()) {
#pragma unroll
                        for (int j = 0; j < L::ROWS / 16; ++j)
                            mma_f16_ss<CG>(d, a_desc + ((g * L::STAGE) >> 4) + 128 * j, b_desc + ((g * L::STAGE) >> 4) + 128 * j, idesc,
                                           j != 0 || chunk != 0 ? 1u : 0u);
                        pair_commit<CG>(&empty[g]);
                        if (done) pair_commit<CG>(&acc_full[acc.s]);
                    }
                    __syncwarp();
                    chunk = done ? 0 : chunk + 1;
                    if (done) acc.next(2);
                    if (--left == 0 && !(ok = next_tile())) break;
                }
            }
            // no instruction may still write tensor memory when it is given back: one more commit, waited for
            if (elect_one()) pair_commit<CG>(finish);
            __syncwarp();
#pragma unroll 1
            for (uint32_t w = 0; w < p.wait_limit && !mbar_try_wait(finish, 0u); ++w) {}
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        constexpr int COLS = TN / 2;                             // of this warp
        const uint32_t from = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * COLS);
        Ring acc;
#pragma unroll 1
        for (int t = first_work; t < work && !stop(); t += work_stride) {
            const WTile w = wgrad_tile<CG, TN>(p, t);
            const int i = w.i0 + rank * 128 + quarter * 32 + lane, j0 = w.j0 + half * COLS;
            float *dst = p.gw + w.part * p.part_stride + ((int64_t)w.expert * p.n + j0) * p.k + i;
            const int have = i < p.k ? min(COLS, p.n - j0) : 0;
            const int stages = (max(0, w.last - w.first) + L::ROWS - 1) / L::ROWS * PAIRS;
            float sum[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) sum[c] = 0.0f;
            bool ok = true;
#pragma unroll 1
            for (int s = 0; s < stages; s += CHUNK) {
                if (!(ok = warp_wait(&acc_full[acc.s], acc.ph, 2))) break;
                tc_fence_after();
#pragma unroll
                for (int c0 = 0; c0 < COLS; c0 += 16) {
                    uint32_t v[16];
                    tmem_load_lane_16(from + (uint32_t)(acc.s * TN + c0), v);
#pragma unroll
                    for (int c = 0; c < 16; ++c) sum[c0 + c] = __fadd_rn(sum[c0 + c], __uint_as_float(v[c]));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_leader<CG>(&acc_empty[acc.s]);
                acc.next(2);
            }
            if (!ok) break;
#pragma unroll
            for (int c = 0; c < COLS; ++c, dst += p.k)
                if (c < have) __stcs(dst, sum[c]);
        }
    }
    tc_fence_before();
    __syncthreads();
    pair_sync<CG>();
    if (warp == 2) {
        tc_fence_after();
        pair_tmem_dealloc<CG>(tmem_base, 2 * TN);
    }
}

template <int CG, int TN, class T>
int wgrad_launch(const void *x, int64_t ldx, const void *dy, int64_t lddy, WgradParams p, int sms, cudaStream_t st) {
    using L = WShape<CG, TN>;
    auto kernel = expert_wgrad_kernel<CG, TN, T>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::TOTAL) != cudaSuccess) return QNN_E_CUDA;
    constexpr bool fp16 = std::is_same<T, __half>::value;
    CUtensorMap map_x, map_dy;
    const int64_t rows = (int64_t)p.rows * G4Type<T>::PARTS;
    if (!make_map_16(&map_x, fp16, x, rows, p.k, ldx, L::ROWS) || !make_map_16(&map_dy, fp16, dy, rows, p.n, lddy, L::ROWS)) return QNN_E_CUDA;
    p.itiles = (p.k + 128 * CG - 1) / (128 * CG);
    p.jtiles = (p.n + TN - 1) / TN;
    const int64_t work = (int64_t)p.experts * p.parts * p.itiles * p.jtiles;
    if (work > 0x3FFFFFFFll) return QNN_E_RANGE;
    const int most = sms / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((work < most ? work : most) * CG));
    cfg.blockDim = dim3(W_THREADS);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    LaunchAttrs attrs(CG);
    cfg.attrs = attrs.a;
    cfg.numAttrs = CG > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, map_x, map_dy, p) != cudaSuccess) {
        cudaGetLastError();
        return QNN_E_CUDA;
    }
    return QNN_OK;
}

// gw = sum of the parts, in order.
__global__ void __launch_bounds__(256) wgrad_sum_kernel(const float *part, int parts, int64_t total, float *gw) {
    start_next();
    wait_for_previous();
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < total; v += (int64_t)gridDim.x * 256) {
        float s = part[v];
        for (int q = 1; q < parts; ++q) s = __fadd_rn(s, part[q * total + v]);
        gw[v] = s;
    }
}

// The tile: pairs of blocks on 256 x 256, or single blocks on 128 x 128 where those need fewer rounds of the GPU (a round of
// wide tiles takes about a quarter longer; sized for 148 SMs, so that workspace queries and calls agree).  Parts of the
// rows: as many as fill the GPU once, each of at least 256 rows on average.
struct WPlan {
    bool wide;
    int parts;
};
WPlan wgrad_plan(int64_t rows, int experts, int n, int k) {
    const int64_t wide = (int64_t)experts * ((k + 255) / 256) * ((n + 255) / 256);
    const int64_t narrow = (int64_t)experts * ((k + 127) / 128) * ((n + 127) / 128);
    WPlan w;
    w.wide = (wide + 73) / 74 * 5 <= (narrow + 147) / 148 * 4;
    const int64_t units = w.wide ? 74 : 148, tiles = w.wide ? wide : narrow, each = rows / experts;
    int64_t parts = units / tiles;
    if (parts > each / 256) parts = each / 256;
    w.parts = parts < 1 ? 1 : (int)parts;
    return w;
}

template <class T>
int wgrad(const void *x, int64_t ldx, const void *dy, int64_t lddy, const WgradParams &p, bool wide, cudaStream_t st) {
    const int sms = sm_count();
    if (sms <= 0) return QNN_E_CUDA;
    return wide ? wgrad_launch<2, 256, T>(x, ldx, dy, lddy, p, sms, st) : wgrad_launch<1, 128, T>(x, ldx, dy, lddy, p, sms, st);
}

}  // namespace

void qnn_expert_wgrad_plan(int64_t rows, int experts, int n, int k, int *tile, int *parts) {
    const WPlan plan = wgrad_plan(rows, experts, n, k);
    *tile = plan.wide ? 256 : 128;
    *parts = plan.parts;
}

size_t qnn_expert_wgrad_parts_bytes(int64_t rows, int experts, int n, int k) {
    const WPlan plan = wgrad_plan(rows, experts, n, k);
    return plan.parts > 1 ? ((size_t)plan.parts * experts * n * k * sizeof(float) + 255) / 256 * 256 : 0;
}

int qnn_expert_wgrad(const void *x, int64_t ldx, const void *dy, int64_t lddy, int type, const int32_t *offsets, int experts, int rows,
                     int n, int k, float *gw, float *parts, cudaStream_t st) {
    const WPlan plan = wgrad_plan(rows, experts, n, k);
    WgradParams p = {};
    p.offsets = offsets; p.experts = experts; p.rows = rows; p.n = n; p.k = k;
    p.parts = plan.parts;
    p.gw = plan.parts > 1 ? parts : gw;
    p.part_stride = (int64_t)experts * n * k;
    p.wait_limit = WAIT_LIMIT;
    if (!(p.err = qnn_tc_error_word())) return QNN_E_CUDA;
    int rc;
    if (type == QNN_F32) rc = wgrad<float>(x, ldx, dy, lddy, p, plan.wide, st);
    else if (type == QNN_BF16) rc = wgrad<__nv_bfloat16>(x, ldx, dy, lddy, p, plan.wide, st);
    else rc = wgrad<__half>(x, ldx, dy, lddy, p, plan.wide, st);
    if (rc != QNN_OK || plan.parts == 1) return rc;
    const int64_t blocks = (p.part_stride + 255) / 256;
    return launch_early(wgrad_sum_kernel, (unsigned)(blocks < 148 * 8 ? blocks : 148 * 8), 256, st, parts, plan.parts, p.part_stride, gw);
}
