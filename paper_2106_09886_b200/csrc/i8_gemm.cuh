// Products of rows in 8 bits on the fifth-generation tensor cores: int32 sums in tensor memory (exact), scales in the epilogue.
// Lanes of an accumulator are output features (rows of the weights), its columns tokens, so that one token costs 16 columns and not
// 128 lanes.  A stage of the ring is 128 elements of the contraction: 128 features and a block's share of the tokens, both by TMA
// with the 128-byte swizzle, four instructions of 32 elements.
//
//   i8_split_kernel<TN, T>   128 features x TN tokens by one block, the contraction split over a cluster of up to eight blocks, whose
//                            int32 sums are added through distributed shared memory (in any order: they are whole numbers).  For few
//                            tokens; bound: reading the weights (1 x 8192 x 8192 13.0 us, 5.2 TB/s; 16 x 16384 x 8192 23.6, 5.7 TB/s).
//   i8_pair_kernel<TN, T>    256 features x TN tokens by a pair of blocks (cta_group::2, half the tokens staged by each), persistent,
//                            two accumulators so that results leave under the next sum.  For many; bound: the tensor pipe (8192^3 328
//                            us in short bursts, 3.35 POP/s, and 375 back to back under the power cap).
#pragma once
#include "pair_ptx.cuh"
#include "real_rows.cuh"

namespace {

constexpr int I8_STEP = 128;                             // elements, and bytes of a row, of a stage

struct I8Params {
    const float *x_scales, *w_scales, *bias;             // bias NULL: none
    void *out;
    int64_t ldo;
    int rows, n, steps;
    bool out_vec;                                        // the result's rows start and advance by whole 16 bytes
    int ftiles, ttiles, band;                            // (pairs) tiles of features and of tokens; tiles of tokens of a band
    unsigned int *err;
    unsigned int wait_limit;
};

// Instruction descriptor of kind::i8: int32 sums at bit 4, signed 8-bit operands at bits 7 and 10, N/8 at bit 17, M/16 at bit 24.
__host__ __device__ constexpr uint32_t idesc_i8(int m, int n) {
    return (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
// D (+)= A * B^T, 32 elements of the contraction.
template <int CG> __device__ __forceinline__ void mma_i8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// The result of a sum: the token's scale first, then the feature's, then the bias, each rounded once.
__device__ __forceinline__ float i8_result(int sum, float x_scale, float w_scale, float bias) {
    return __fadd_rn(__fmul_rn(__fmul_rn((float)sum, x_scale), w_scale), bias);
}

// ------------------------------------------------------------------------------------------------ few tokens

template <int TN> struct I8Split {
    static constexpr int A_STAGE = 128 * I8_STEP, STAGE = A_STAGE + TN * I8_STEP;
    static constexpr int STAGES = TN <= 16 ? 6 : TN <= 32 ? 5 : TN <= 64 ? 4 : 6;
    static constexpr int BLOCKS = TN <= 64 ? 2 : 1;      // that fit an SM
    static constexpr int SCALE_OFF = STAGES * STAGE, BAR_OFF = SCALE_OFF + TN * 4;
    static constexpr int TOTAL = BAR_OFF + (2 * STAGES + 1) * 8 + 16 + 1024;
    static constexpr int COLS = TN < 32 ? 32 : TN;       // tensor-memory columns
    static constexpr int THREADS = 192;                  // warps 0-3 results, 4 copies, 5 instructions
    static_assert(TN * 128 * 4 <= SCALE_OFF, "the block's sums fit the ring");
};

// Tokens rank, rank + RANKS, ... of a tile: the ranks' sums, read through distributed shared memory with 16 loads under way (each takes
// a round trip), and the result.
template <int RANKS, class T>
__device__ __forceinline__ void i8_add_ranks(uint32_t mine, int rank, int have, T *out, int64_t ldo, const float *x_scales, float w_scale, float bias) {
    constexpr int TOKENS = 16 / RANKS;
    uint32_t there[RANKS];
#pragma unroll
    for (int q = 0; q < RANKS; ++q) asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there[q]) : "r"(mine), "r"(q));
#pragma unroll 1
    for (int c0 = rank; c0 < have; c0 += RANKS * TOKENS) {
        int v[TOKENS][RANKS];
        float s[TOKENS];
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const int c = c0 + i * RANKS;
            if (c < have) {
                s[i] = x_scales[c];
#pragma unroll
                for (int q = 0; q < RANKS; ++q) asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v[i][q]) : "r"(there[q] + c * 512) : "memory");
            }
        }
#pragma unroll
        for (int i = 0; i < TOKENS; ++i) {
            const int c = c0 + i * RANKS;
            if (c < have) {
                int sum = v[i][0];
#pragma unroll
                for (int q = 1; q < RANKS; ++q) sum += v[i][q];
                out[(int64_t)c * ldo] = from_f32<T>(i8_result(sum, s[i], w_scale, bias));
            }
        }
    }
}

template <int TN, class T>
__global__ void __launch_bounds__(I8Split<TN>::THREADS, I8Split<TN>::BLOCKS)
i8_split_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const I8Params p, int log_ranks) {
    using L = I8Split<TN>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_at = smem_u32(smem);
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF), *empty = full + L::STAGES, *done = empty + L::STAGES;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(done + 1);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int ranks = 1 << log_ranks, rank = blockIdx.x & (ranks - 1), f0 = (blockIdx.x >> log_ranks) * 128, t0 = blockIdx.y * TN;
    const int lo = (int)((int64_t)p.steps * rank >> log_ranks), hi = (int)((int64_t)p.steps * (rank + 1) >> log_ranks);      // ranks <= steps

    if (threadIdx.x == 0) {
        for (int s = 0; s < L::STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        mbar_init(done, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 5) tmem_alloc(tmem_slot, L::COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    start_next();
    wait_for_previous();

    if (warp == 4) {
        if (elect_one()) {
            Ring g;
            int it = 0;
#pragma unroll 1
            for (int k = lo; k < hi; ++k, ++it) {
                if (!short_wait(&empty[g.s], g.ph ^ 1u, abort_flag, 0, p.err, p.wait_limit)) break;
                mbar_expect_tx(&full[g.s], L::STAGE);
                tma_load_2d(smem + g.s * L::STAGE, &map_w, &full[g.s], k * I8_STEP, f0);
                tma_load_2d(smem + g.s * L::STAGE + L::A_STAGE, &map_x, &full[g.s], k * I8_STEP, t0);
                g.next(L::STAGES);
            }
            if (*abort_flag) drain_copies_in_flight(full, it, L::STAGES, p.wait_limit);
        }
        __syncwarp();
    } else if (warp == 5) {
        if (elect_one()) {
            constexpr uint32_t idesc = idesc_i8(128, TN);
            Ring g;
#pragma unroll 1
            for (int k = lo; k < hi; ++k) {
                if (!short_wait(&full[g.s], g.ph, abort_flag, 1, p.err, p.wait_limit)) break;
                tc_fence_after();
                const uint64_t a = smem_desc_k_sw128(smem_at + g.s * L::STAGE), b = smem_desc_k_sw128(smem_at + g.s * L::STAGE + L::A_STAGE);
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_i8<1>(tmem_base, a + 2 * j, b + 2 * j, idesc, k > lo || j > 0 ? 1u : 0u);
                tc_commit(&empty[g.s]);
                g.next(L::STAGES);
            }
            tc_commit(done);
        }
        __syncwarp();
    }
    const int have = min(TN, p.rows - t0), f = f0 + warp * 32 + lane;
    float *x_scales = reinterpret_cast<float *>(smem + L::SCALE_OFF);
    float w_scale = 0.0f, bias = 0.0f;
    if (warp < 4) {
        for (int c = threadIdx.x; c < have; c += 128) x_scales[c] = p.x_scales[t0 + c];
        if (f < p.n) {
            w_scale = p.w_scales[f];
            if (p.bias) bias = p.bias[f];
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
    }
    // every instruction has completed: the sums are there, and the ring is free
    const bool ok = __all_sync(0xffffffffu, short_wait(done, 0u, abort_flag, 2, p.err, p.wait_limit));
    tc_fence_after();
    const uint32_t at = tmem_base + ((uint32_t)((warp & 3) * 32) << 16);
    T *out = static_cast<T *>(p.out) + (int64_t)t0 * p.ldo + f;
    if (log_ranks == 0) {
        if (warp < 4 && ok)
#pragma unroll 1
            for (int c0 = 0; c0 < have; c0 += 16) {
                uint32_t v[16];
                tmem_load_lane_16(at + c0, v);
                if (f < p.n) {
                    if (have - c0 >= 16) {
#pragma unroll
                        for (int i = 0; i < 16; ++i, out += p.ldo) *out = from_f32<T>(i8_result((int)v[i], x_scales[c0 + i], w_scale, bias));
                    } else {
#pragma unroll
                        for (int i = 0; i < 16; ++i, out += p.ldo)
                            if (c0 + i < have) *out = from_f32<T>(i8_result((int)v[i], x_scales[c0 + i], w_scale, bias));
                    }
                }
                __syncwarp();
            }
    } else {
        const uint32_t mine = smem_at + (warp * 32 + lane) * 4;                  // sums as [token][feature]
        if (warp < 4 && ok)
#pragma unroll 1
            for (int c0 = 0; c0 < have; c0 += 16) {
                uint32_t v[16];
                tmem_load_lane_16(at + c0, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) asm volatile("st.shared.b32 [%0], %1;" ::"r"(mine + (c0 + i) * 512), "r"(v[i]) : "memory");
            }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (warp < 4 && f < p.n) {
            if (log_ranks == 1) i8_add_ranks<2>(mine, rank, have, out, p.ldo, x_scales, w_scale, bias);
            else if (log_ranks == 2) i8_add_ranks<4>(mine, rank, have, out, p.ldo, x_scales, w_scale, bias);
            else i8_add_ranks<8>(mine, rank, have, out, p.ldo, x_scales, w_scale, bias);
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");    // nobody leaves while its sums are read
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 5) {
        tc_fence_after();
        tmem_dealloc(tmem_base, L::COLS);
    }
}

// ------------------------------------------------------------------------------------------------ many tokens

template <int TN, class T> struct I8Pair {
    static constexpr int XROWS = TN / 2;                                         // tokens that a block stages
    static constexpr int A_STAGE = 128 * I8_STEP, STAGE = A_STAGE + XROWS * I8_STEP;
    static constexpr int OUT_WARP = sizeof(T) == 2 ? 32 * 80 : 0;                // transposing buffer of a result warp
    static constexpr int FIXED = 8 * (OUT_WARP + TN * 4) + 2048;
    static constexpr int STAGES = (227 * 1024 - FIXED) / STAGE < 8 ? (227 * 1024 - FIXED) / STAGE : 8;
    static constexpr int OUT_OFF = STAGES * STAGE, SCALE_OFF = OUT_OFF + 8 * OUT_WARP, BAR_OFF = SCALE_OFF + 8 * TN * 4;
    static constexpr int TOTAL = BAR_OFF + (2 * STAGES + 5) * 8 + 16 + 1024;
    // warps: 0 copies, 1 instructions, 2 owner of the tensor memory, 3 idle, 4-11 results (two for each quarter of the lanes, whose
    // latencies cover one another, and scales that are loaded an item ahead: 4096 x 5000 x 700 takes 19.7 us, 28.6 with one and without)
    static constexpr int THREADS = 384;
    static_assert(TOTAL <= 227 * 1024, "shared memory");
};

struct I8Item {
    int f, t;
};
// Items go through bands of tokens, so that the pairs that run together share rows of both operands in L2.
__device__ __forceinline__ I8Item i8_item(int item, const I8Params &p) {
    const int per_band = p.band * p.ftiles, b = item / per_band, in = item - b * per_band;
    const int high = min(p.band, p.ttiles - b * p.band), f = in / high;
    return {f, b * p.band + in - f * high};
}

// 32 tokens x 32 features of an accumulator -> rows of a 2-byte result, transposed on the way through shared memory (80 bytes a
// token: free of bank conflicts), so that a token's features leave as 16-byte stores.
template <class T>
__device__ __forceinline__ void i8_store_quarter(uint32_t taddr, uint32_t buf, const float *scales, T *row0, int64_t ldo, int tokens, int f,
                                                 int n, const float (&w_scale)[4], const float (&bias)[4], bool vec) {
    const int lane = threadIdx.x & 31;
    const uint32_t at = buf + ((lane >> 4) * 8 + (lane & 7)) * 80 + ((lane >> 3) & 1) * 16;
    float2 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = *reinterpret_cast<const float2 *>(scales + 8 * i + 2 * (lane & 3));
    uint32_t r[2][16];
    tmem_load_16x32(taddr, r[0]);
    tmem_load_16x32(taddr + (16u << 16), r[1]);
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)              // register pair i: features 16h + 8 (i % 2) + lane / 4, tokens 8 (i / 2) + 2 (lane % 4) + {0, 1}
            v[i] = pack_pair<T>(i8_result((int)r[h][2 * i], s[i >> 1].x, w_scale[2 * h + (i & 1)], bias[2 * h + (i & 1)]),
                                i8_result((int)r[h][2 * i + 1], s[i >> 1].y, w_scale[2 * h + (i & 1)], bias[2 * h + (i & 1)]));
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                         ::"r"(at + i * 16 * 80 + h * 32), "r"(v[4 * i]), "r"(v[4 * i + 1]), "r"(v[4 * i + 2]), "r"(v[4 * i + 3]) : "memory");
    }
    __syncwarp();
    if (vec && f + 32 <= n) {
        const int c0 = f + (lane >> 3) * 8;
        uint4 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = lds_128(buf + (i * 8 + (lane & 7)) * 80 + (lane >> 3) * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int token = i * 8 + (lane & 7);
            if (token < tokens) *reinterpret_cast<uint4 *>(row0 + (int64_t)token * ldo + c0) = v[i];
        }
    } else if (f + lane < n) {                   // a token's 32 features by the warp, element by element (pairs of them at even
        uint16_t *dst = reinterpret_cast<uint16_t *>(row0) + f + lane;      // addresses, half a warp a token, took a third longer)
        const uint32_t src = buf + lane * 2;
#pragma unroll 1
        for (int t0 = 0; t0 < min(tokens, 32); t0 += 8) {
            uint16_t v[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v[t]) : "r"(src + (t0 + t) * 80) : "memory");
            if (tokens - t0 >= 8) {
#pragma unroll
                for (int t = 0; t < 8; ++t, dst += ldo) *dst = v[t];
            } else {
#pragma unroll
                for (int t = 0; t < 8; ++t, dst += ldo)
                    if (t0 + t < tokens) *dst = v[t];
            }
        }
    }
    __syncwarp();
}

template <int TN, class T>
__global__ void __launch_bounds__(I8Pair<TN, T>::THREADS, 1)
i8_pair_kernel(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_x, const I8Params p) {
    using L = I8Pair<TN, T>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_at = smem_u32(smem);
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF);            // leader: both blocks' copies have landed
    uint64_t *empty = full + L::STAGES;                                          // each block: the instructions have read a stage
    uint64_t *acc_full = empty + L::STAGES;                                      // each block
    uint64_t *acc_empty = acc_full + 2;                                          // leader: both blocks have read an accumulator out
    uint64_t *finish = acc_empty + 2;                                            // every instruction has completed
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(finish + 1);
    volatile uint32_t *abort_flag = tmem_slot + 1;
    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int rank = (int)pair_rank<2>(), first = blockIdx.x / 2, stride = gridDim.x / 2, items = p.ftiles * p.ttiles;

    if (threadIdx.x == 0) {
        for (int s = 0; s < L::STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 16); }
        mbar_init(finish, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) pair_tmem_alloc<2>(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    pair_sync<2>();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    start_next();
    wait_for_previous();
    auto stop = [&]() { return *abort_flag != 0; };

    if (warp == 0) {
        if (elect_one()) {
            Ring g;
            long long it = 0;
            bool ok = true;
#pragma unroll 1
            for (int t = first; ok && t < items && !stop(); t += stride) {
                const I8Item work = i8_item(t, p);
                const int f = (work.f * 2 + rank) * 128, x = work.t * TN + rank * L::XROWS;
#pragma unroll 1
                for (int k = 0; k < p.steps; ++k, ++it) {
                    if (!(ok = short_wait(&empty[g.s], g.ph ^ 1u, abort_flag, 0, p.err, p.wait_limit))) break;
                    if (rank == 0) mbar_expect_tx(&full[g.s], 2 * L::STAGE);
                    pair_load_2d<2>(smem + g.s * L::STAGE, &map_w, &full[g.s], k * I8_STEP, f);
                    pair_load_2d<2>(smem + g.s * L::STAGE + L::A_STAGE, &map_x, &full[g.s], k * I8_STEP, x);
                    g.next(L::STAGES);
                }
            }
            // after an abort the copies in flight may still land (the other block's may never be issued)
            if (stop() && it > 0)
#pragma unroll 1
                for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (rank == 0) {
            if (elect_one()) {
                constexpr uint32_t idesc = idesc_i8(256, TN);
                const uint64_t a0 = smem_desc_k_sw128(smem_at), b0 = smem_desc_k_sw128(smem_at + L::A_STAGE);
                Ring g, acc;
                bool ok = true;
#pragma unroll 1
                for (int t = first; ok && t < items && !stop(); t += stride) {
                    if (!(ok = short_wait(&acc_empty[acc.s], acc.ph ^ 1u, abort_flag, 3, p.err, p.wait_limit))) break;
                    tc_fence_after();
                    const uint32_t d = tmem_base + (uint32_t)(acc.s * TN);
#pragma unroll 1
                    for (int k = 0; k < p.steps; ++k) {
                        if (!(ok = short_wait(&full[g.s], g.ph, abort_flag, 1, p.err, p.wait_limit))) break;
                        tc_fence_after();
                        const uint32_t at = (uint32_t)(g.s * L::STAGE) >> 4;
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma_i8<2>(d, a0 + at + 2 * j, b0 + at + 2 * j, idesc, k > 0 || j > 0 ? 1u : 0u);
                        pair_commit<2>(&empty[g.s]);
                        g.next(L::STAGES);
                    }
                    if (ok) pair_commit<2>(&acc_full[acc.s]);
                    acc.next(2);
                }
                // no instruction may still write tensor memory when it is given back: one more commit, waited for
                pair_commit<2>(finish);
#pragma unroll 1
                for (uint32_t w = 0; w < p.wait_limit && !mbar_try_wait(finish, 0u); ++w) {}
            }
            __syncwarp();
        }
    } else if (warp >= 4) {
        const int q = warp & 3, w = warp - 4;                    // quarter of the lanes; warps w and w + 4 share it
        const uint32_t lanes = (uint32_t)(q * 32) << 16;
        float *scales = reinterpret_cast<float *>(smem + L::SCALE_OFF) + w * TN;
        Ring acc;
        // scales of an item's tokens and features, loaded while the item before it is stored
        constexpr int FEATURES = sizeof(T) == 2 ? 4 : 1;
        float token_scale[TN / 32], next_scale[FEATURES], next_bias[FEATURES];
        auto load_scales = [&](int t) {
            const I8Item work = i8_item(t, p);
            const int f = (work.f * 2 + rank) * 128 + q * 32, t0 = work.t * TN;
#pragma unroll
            for (int c = 0; c < TN / 32; ++c) token_scale[c] = t0 + c * 32 + lane < p.rows ? p.x_scales[t0 + c * 32 + lane] : 0.0f;
#pragma unroll
            for (int i = 0; i < FEATURES; ++i) {
                const int at = sizeof(T) == 2 ? f + 8 * i + (lane >> 2) : f + lane;
                next_scale[i] = at < p.n ? p.w_scales[at] : 0.0f;
                next_bias[i] = p.bias && at < p.n ? p.bias[at] : 0.0f;
            }
        };
        if (first < items) load_scales(first);
#pragma unroll 1
        for (int t = first; t < items && !__any_sync(0xffffffffu, stop()); t += stride) {
            const I8Item work = i8_item(t, p);
            const int f = (work.f * 2 + rank) * 128 + q * 32, t0 = work.t * TN, have = min(TN, p.rows - t0);
            T *dst = static_cast<T *>(p.out) + (int64_t)t0 * p.ldo;
            float w_scale[4], bias[4];
#pragma unroll
            for (int c = 0; c < TN / 32; ++c) scales[c * 32 + lane] = token_scale[c];
#pragma unroll
            for (int i = 0; i < FEATURES; ++i) { w_scale[i] = next_scale[i]; bias[i] = next_bias[i]; }
            __syncwarp();
            if (t + stride < items) load_scales(t + stride);
            if (!__all_sync(0xffffffffu, short_wait(&acc_full[acc.s], acc.ph, abort_flag, 2, p.err, p.wait_limit))) break;
            tc_fence_after();
            const uint32_t from = tmem_base + lanes + (uint32_t)(acc.s * TN);
#pragma unroll 1
            for (int c0 = (w >> 2) * 32; c0 < have; c0 += 64) {
                if constexpr (sizeof(T) == 2) {
                    i8_store_quarter<T>(from + c0, smem_at + L::OUT_OFF + w * L::OUT_WARP, scales + c0, dst + (int64_t)c0 * p.ldo, p.ldo, have - c0, f,
                                        p.n, w_scale, bias, p.out_vec);
                } else {
                    uint32_t v[32];
                    tmem_load_32(from + c0, v);
                    if (f + lane < p.n) {
                        T *to = dst + (int64_t)c0 * p.ldo + f + lane;
                        if (have - c0 >= 32) {
#pragma unroll
                            for (int i = 0; i < 32; ++i, to += p.ldo) *to = i8_result((int)v[i], scales[c0 + i], w_scale[0], bias[0]);
                        } else {
#pragma unroll
                            for (int i = 0; i < 32; ++i, to += p.ldo)
                                if (c0 + i < have) *to = i8_result((int)v[i], scales[c0 + i], w_scale[0], bias[0]);
                        }
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader<2>(&acc_empty[acc.s]);
            acc.next(2);
        }
    }
    tc_fence_before();
    __syncthreads();
    pair_sync<2>();
    if (warp == 2) {
        tc_fence_after();
        pair_tmem_dealloc<2>(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------ host side

// Tensor map of rows of codes: boxes of 128 elements x box_rows rows, 128-byte swizzle, zeros outside.
inline bool make_map_i8(CUtensorMap *map, const int8_t *base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld};
    cuuint32_t box[2] = {I8_STEP, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace
