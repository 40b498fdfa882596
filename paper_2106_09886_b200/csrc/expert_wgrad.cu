// Weight gradients of products grouped by expert: gw[e][j][i] = sum over e's rows of dy[r][j] * x[r][i], fp32.
//
// Both operands are read with the contraction (rows) outermost, exactly as they lie in memory: boxes of 64 columns x 64
// rows, MN-major for the tensor cores.  The lanes of an accumulator are columns i of x and its columns are features j, so
// that a warp stores 32 neighbouring elements of a row of gw.  An expert's last block of rows reaches into the next
// expert's: one warp clears those rows in shared memory before the instructions see them (a zero in one operand alone
// would not do, as the other may hold NaN or infinity).
// fp32: both operands are three bf16 parts; the six products of parts down to 2^-16 of the largest are summed.
#include "g4_stage.cuh"
#include "g4_tensor.cuh"

namespace {

struct WgradParams {
    const int32_t *offsets;
    int experts, rows, n, k;
    float *gw;
    int itiles, jtiles;                   // tiles of 128 * CG columns of x, of TN features
    unsigned int *err;
    unsigned int wait_limit;
};

constexpr int W_THREADS = 256;            // warps: 0 TMA, 1 matrix instructions, 2 tail rows (and owner of the tensor memory),
                                          // 3 idle, 4-7 results

template <int CG, int TN>
struct WShape {
    static constexpr int ROWS = 64;                             // rows of a stage
    static constexpr int BLOCK = ROWS * 128;                    // 64 columns of them
    static constexpr int B_COLS = TN / CG;                      // features this block stages
    static constexpr int A_BYTES = 2 * BLOCK;
    static constexpr int STAGE = A_BYTES + B_COLS / 64 * BLOCK;
    static constexpr int STAGES = 200 * 1024 / STAGE > 8 ? 8 : 200 * 1024 / STAGE;
    static constexpr int BAR_OFF = STAGES * STAGE;
    static constexpr int TOTAL = BAR_OFF + (3 * STAGES + 4) * 8 + 16 + 1024;
    static constexpr int ACC_BUFS = 512 / TN >= 2 ? 2 : 1;
    static_assert(B_COLS % 64 == 0, "features in blocks of 64");
};

// Products of parts, largest first: (x part, dy part).
__device__ __forceinline__ int pair_x(int q) { return (0x010120 >> (4 * (5 - q))) & 15; }
__device__ __forceinline__ int pair_dy(int q) { return (0x001102 >> (4 * (5 - q))) & 15; }

template <int CG, int TN, class T>
__global__ void __launch_bounds__(W_THREADS, 1) expert_wgrad_kernel(const __grid_constant__ CUtensorMap map_x,
                                                                   const __grid_constant__ CUtensorMap map_dy, const WgradParams p) {
    using L = WShape<CG, TN>;
    constexpr int PAIRS = G4Type<T>::PARTS == 1 ? 1 : 6;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t *landed = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF);     // each block: its copies of a stage
    uint64_t *ready = landed + L::STAGES;                                   // leader: both blocks' stages are fit to be read
    uint64_t *empty = ready + L::STAGES;                                    // each block
    uint64_t *acc_full = empty + L::STAGES;                                 // each block
    uint64_t *acc_empty = acc_full + 2;                                     // leader
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(acc_empty + 2);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int rank = (int)pair_rank<CG>();
    const int first_work = blockIdx.x / CG, work_stride = gridDim.x / CG;
    const int per_expert = p.itiles * p.jtiles, work = p.experts * per_expert;

    if (threadIdx.x == 0) {
        for (int s = 0; s < L::STAGES; ++s) { mbar_init(&landed[s], 1); mbar_init(&ready[s], CG); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 4 * CG); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) pair_tmem_alloc<CG>(tmem_slot, L::ACC_BUFS * TN);
    tc_fence_before();
    __syncthreads();
    pair_sync<CG>();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    auto warp_wait = [&](uint64_t *bar, uint32_t parity, unsigned id) {
        return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, id, p.err, p.wait_limit));
    };
    auto stop = [&]() { return __any_sync(0xffffffffu, *abort_flag != 0); };
    int committed = 0;

    if (warp == 0) {
        Ring g;
        long long it = 0;
        for (int t = first_work; t < work && !stop(); t += work_stride) {
            const int e = t / per_expert, in = t - e * per_expert;
            int first, last;
            expert_rows(p.offsets, e, p.rows, first, last);
            const int i0 = ((in % p.itiles) * CG + rank) * 128, j0 = (in / p.itiles) * TN + rank * L::B_COLS;
            bool ok = true;
            for (int r = first; ok && r < last; r += L::ROWS)
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
        for (int t = first_work; t < work && !stop(); t += work_stride) {
            const int e = t / per_expert;
            int first, last;
            expert_rows(p.offsets, e, p.rows, first, last);
            bool ok = true;
            for (int r = first; ok && r < last; r += L::ROWS)
                for (int q = 0; q < PAIRS; ++q) {
                    if (!(ok = warp_wait(&landed[g.s], g.ph, 1))) break;
                    const int valid = last - r;
                    if (valid < L::ROWS) {
                        const uint32_t stage = smem_u32(smem) + g.s * L::STAGE;
                        for (int b = 0; b < L::STAGE / L::BLOCK; ++b)
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
            Ring g;
            constexpr uint32_t idesc = idesc_f16(G4Type<T>::FMT, 128 * CG, TN, true, true);
            int local = 0;
            for (int t = first_work; t < work && !stop(); t += work_stride) {
                int first, last;
                expert_rows(p.offsets, t / per_expert, p.rows, first, last);
                if (first >= last) continue;                     // nothing to add up: the result warps write zeros
                const int buf = local % L::ACC_BUFS;
                if (!warp_wait(&acc_empty[buf], ((uint32_t)(local / L::ACC_BUFS) & 1u) ^ 1u, 3)) break;
                tc_fence_after();
                const uint32_t d = tmem_base + (uint32_t)(buf * TN);
                bool ok = true;
                for (int r = first; ok && r < last; r += L::ROWS)
                    for (int q = 0; q < PAIRS; ++q) {
                        if (!(ok = warp_wait(&ready[g.s], g.ph, 1))) break;
                        tc_fence_after();
                        const uint32_t at = smem_u32(smem + g.s * L::STAGE);
                        const uint64_t a = smem_desc_mn_sw128(at, L::BLOCK), b = smem_desc_mn_sw128(at + L::A_BYTES, L::BLOCK);
                        if (elect_one()) {
#pragma unroll
                            for (int j = 0; j < L::ROWS / 16; ++j)
                                mma_f16_ss<CG>(d, a + 128 * j, b + 128 * j, idesc, ((r - first) | q | j) != 0 ? 1u : 0u);
                            pair_commit<CG>(&empty[g.s]);
                        }
                        __syncwarp();
                        g.next(L::STAGES);
                    }
                if (elect_one()) pair_commit<CG>(&acc_full[buf]);            // also after a wait that gave up: see the end
                __syncwarp();
                committed = ++local;
            }
        }
    } else if (warp >= 4) {
        const int w = warp & 3;
        int local = 0;
        for (int t = first_work; t < work && !stop(); t += work_stride) {
            const int e = t / per_expert, in = t - e * per_expert;
            int first, last;
            expert_rows(p.offsets, e, p.rows, first, last);
            const int i = ((in % p.itiles) * CG + rank) * 128 + w * 32 + lane, j0 = (in / p.itiles) * TN;
            float *dst = p.gw + ((int64_t)e * p.n + j0) * p.k + i;
            const int have = min(TN, p.n - j0);
            if (first >= last) {
                if (i < p.k)
                    for (int j = 0; j < have; ++j) dst[(int64_t)j * p.k] = 0.0f;
                continue;
            }
            const int buf = local % L::ACC_BUFS;
            if (!warp_wait(&acc_full[buf], (uint32_t)(local / L::ACC_BUFS) & 1u, 2)) break;
            tc_fence_after();
#pragma unroll 1
            for (int c0 = 0; c0 < have; c0 += 32) {
                uint32_t v[32];
                tmem_load_32(tmem_base + ((uint32_t)(w * 32) << 16) + (uint32_t)(buf * TN + c0), v);
                if (i < p.k) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (c0 + j < have) __stcs(dst + (int64_t)(c0 + j) * p.k, __uint_as_float(v[j]));
                }
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader<CG>(&acc_empty[buf]);
            ++local;
        }
    }
    __syncwarp();
    if (warp == 1 && rank == 0 && lane == 0 && committed > 0) {
        const int final_acc = committed - 1;
        for (uint32_t w = 0; w < p.wait_limit && !mbar_try_wait(&acc_full[final_acc % L::ACC_BUFS], (uint32_t)(final_acc / L::ACC_BUFS) & 1u); ++w) {}
    }
    tc_fence_before();
    __syncthreads();
    pair_sync<CG>();
    if (warp == 2) {
        tc_fence_after();
        pair_tmem_dealloc<CG>(tmem_base, L::ACC_BUFS * TN);
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
    const int64_t work = (int64_t)p.experts * p.itiles * p.jtiles;
    if (work > 0x3FFFFFFFll) return QNN_E_RANGE;
    const int most = sms / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((work < most ? work : most) * CG));
    cfg.blockDim = dim3(W_THREADS);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = CG;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG > 1 ? 1 : 0;
    if (cudaLaunchKernelEx(&cfg, kernel, map_x, map_dy, p) != cudaSuccess) {
        cudaGetLastError();
        return QNN_E_CUDA;
    }
    return QNN_OK;
}

template <class T>
int wgrad(const void *x, int64_t ldx, const void *dy, int64_t lddy, const WgradParams &p, cudaStream_t st) {
    const int sms = sm_count();
    if (sms <= 0) return QNN_E_CUDA;
    return wgrad_launch<1, 128, T>(x, ldx, dy, lddy, p, sms, st);
}

}  // namespace

int qnn_expert_wgrad(const void *x, int64_t ldx, const void *dy, int64_t lddy, int type, const int32_t *offsets, int experts, int rows,
                     int n, int k, float *gw, cudaStream_t st) {
    WgradParams p = {};
    p.offsets = offsets; p.experts = experts; p.rows = rows; p.n = n; p.k = k; p.gw = gw;
    p.wait_limit = WAIT_LIMIT;
    if (!(p.err = qnn_tc_error_word())) return QNN_E_CUDA;
    if (type == QNN_F32) return wgrad<float>(x, ldx, dy, lddy, p, st);
    if (type == QNN_BF16) return wgrad<__nv_bfloat16>(x, ldx, dy, lddy, p, st);
    return wgrad<__half>(x, ldx, dy, lddy, p, st);
}
