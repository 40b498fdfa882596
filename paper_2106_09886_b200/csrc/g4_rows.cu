// Few rows times group-scaled 4-bit weights: y[r][j] = alpha_e * sum_i x[r][i] * scale_e[j][i/G] * q_e[j][i].
//
// Bound: reading the codes once (n*k/2 bytes).  At HBM speed a B200 streams 13e12 weights a second, 2.8 lane
// instructions each, which one fused multiply-add per weight and row does not fit; so the products run as warp-level
// m16n8k16 matrix instructions with 16 features as the rows and up to 8 x-columns per instruction, and a weight costs
// only its unpacking: per pair a shift, a logic operation that leaves the 4-bit code as a small multiple of the type's
// smallest step, and one fused multiply-add that makes the odd integer 2t - 15 (times a power of two) exactly.
// Group scales multiply the fp32 sums of a group, not the weights.  (The tensor memory path needs 128 features and a
// pipeline per thread block; with a few rows its fixed cost is the larger part.)
//
// A block takes a stored row of tiles (128 features): one warp streams its tiles of 8 KB through a ring in shared memory by
// bulk copies, which keeps some 50 KB a block in flight at no cost in registers; eight warps multiply, 16 features each, all
// with the same columns of x.  Aligned 16-bit rows of x travel with the codes; others are converted into shared memory,
// once for the block, some tiles at a time.  The contraction is split over a cluster of up to eight blocks, whose sums are
// added in a fixed order through distributed shared memory.
// fp32 rows are split exactly into three bf16 parts (8 + 8 + 8 bits) that occupy three of the instruction's columns.
// Measured in a replayed graph: 1 x 8192 x 8192 13.6 to 14.1 us (2.5 TB/s of codes and scales), 1 x 4096 x 4096 6.1, 1 x 1024 x 1024
// 3.1; issue-bound (164 instructions per warp and tile in all) with some 3 us of start and joining around it.
#include "g4_rows.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int WARPS = 8;                                  // that multiply; one more copies
constexpr int STRIP = 16;                                 // features of one matrix instruction
constexpr int THREADS = (WARPS + 1) * 32;
constexpr int UNIT = 128 * 16;                            // a quarter of a tile's codes: 16 bytes of each row
constexpr int UNIT_PITCH = UNIT + 32;                     // (the four lanes of a quad read the same row of the four units)
constexpr int SCALES_AT = 4 * UNIT_PITCH;
constexpr int C_TILE = SCALES_AT + 512;                   // codes and up to four rows of scales
constexpr int U = 2;                                      // tiles of a stage: one wait, and their reads overlap
constexpr int C_STAGE = U * C_TILE;
constexpr int C_STAGES = 3;
constexpr int X_PITCH = 320;                              // bytes of a column's 128 elements: 16-byte reads without bank conflicts

template <class T> struct RowType;
template <> struct RowType<__nv_bfloat16> { static constexpr int PARTS = 1; };
template <> struct RowType<__half> { static constexpr int PARTS = 1; };
template <> struct RowType<float> { static constexpr int PARTS = 3; };

// Pair p of a code word as numbers of the operand's type, exact:
//   bf16  the bare nibble is the subnormal t * 2^-133; times 2^127 minus 15 * 2^-7 it is q / 128;
//   fp16  the nibble under the exponent of 1024 is 1024 + 16t; an eighth of it minus 143 is q.
// The group's scale takes that factor out, and for the types with fp32's range leaves 2^-13, for the last multiplication to undo.
template <class T> struct CodeScale { static constexpr float GROUP = 128.0f / 8192.0f, UNDO = 8192.0f; };
template <> struct CodeScale<__half> { static constexpr float GROUP = 1.0f, UNDO = 1.0f; };
template <class T>
__device__ __forceinline__ uint32_t code_pair(uint32_t word, int p) {
    uint32_t r;
    if constexpr (std::is_same<T, __half>::value) {
        const uint32_t s = p == 0 ? word << 4 : word >> (4 * p - 4);
        uint32_t u;
        asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(u) : "r"(s));
        const __half2 v = __hfma2(*reinterpret_cast<const __half2 *>(&u), __half2half2(__ushort_as_half(0x3000)),
                                  __half2half2(__ushort_as_half(0xD878)));
        r = *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const uint32_t u = (word >> (4 * p)) & 0x000F000Fu;
        const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u), __bfloat162bfloat162(__ushort_as_bfloat16(0x7F00)),
                                         __bfloat162bfloat162(__ushort_as_bfloat16(0xBDF0)));
        r = *reinterpret_cast<const uint32_t *>(&v);
    }
    return r;
}

// Volatile, as is every load of its operands: what a stage's release has to come after may not be moved behind it.
template <class T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Elements [i0, i0 + 128 * tiles) of `have` rows of x as columns in shared memory: tile t, column c at (t * cols + c) *
// X_PITCH; zeros from element k on.  fp32 rows become PARTS columns each.  Element by element (consecutive threads,
// consecutive elements), many loads in flight.
template <class T>
__device__ __noinline__ void stage_columns(const T *x, int64_t ldx, int have, int i0, int tiles, int k, int cols, uint32_t xs) {
    constexpr int PARTS = RowType<T>::PARTS, BATCH = 16;
    // warps of a row: all eight for one row, one when there are many
    const int log_warps = have == 1 ? 3 : have == 2 ? 2 : have <= 4 ? 1 : 0;
    const int lanes = 32 << log_warps, lane0 = threadIdx.x & (lanes - 1);
#pragma unroll 1
    for (int r = threadIdx.x >> (5 + log_warps); r < have; r += WARPS >> log_warps) {
        const T *src = x + (int64_t)r * ldx + i0;
#pragma unroll 1
        for (int o0 = lane0; o0 < tiles * 128; o0 += BATCH * lanes) {
            uint32_t v[BATCH];
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int o = o0 + j * lanes;
                v[j] = 0u;
                if (o < tiles * 128 && i0 + o < k) {
                    if constexpr (PARTS == 1) v[j] = reinterpret_cast<const unsigned short *>(src)[o];
                    else v[j] = __float_as_uint(src[o]);
                }
            }
#pragma unroll
            for (int j = 0; j < BATCH; ++j) {
                const int o = o0 + j * lanes;
                if (o >= tiles * 128) break;
                const uint32_t at = xs + ((o >> 7) * cols + r * PARTS) * X_PITCH + (o & 127) * 2;
                if constexpr (PARTS == 1) {
                    asm volatile("st.shared.u16 [%0], %1;" ::"r"(at), "h"((unsigned short)v[j]) : "memory");
                } else {
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(at + p * X_PITCH), "h"((unsigned short)(split_part_bits(__uint_as_float(v[j]), p) >> 16)) : "memory");
                }
            }
        }
    }
}
__device__ __forceinline__ void multiplying_warps_sync() { asm volatile("bar.sync 1, %0;" ::"n"(WARPS * 32) : "memory"); }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Block (row of stored tiles, rank in the cluster) x block of rows of one expert.  The cluster's ranks share the contraction.
// STREAM: the rows of x start and advance by whole 16 bytes and travel with the codes.
template <class T, int NT, bool STREAM> struct RowsShape {
    static constexpr int X_TILE = NT * 8 * X_PITCH;
    static constexpr int STAGE = C_STAGE + (STREAM ? U * X_TILE : 0);
    static constexpr int X_TILES = 16 / NT / U * U;                     // tiles of converted x held at a time
    static constexpr int X_OFF = C_STAGES * STAGE;
    static constexpr int BAR_OFF = X_OFF + (STREAM ? 0 : X_TILES * X_TILE);
    static constexpr int TOTAL = BAR_OFF + 2 * C_STAGES * 8 + 16;
    static constexpr int BLOCKS = STREAM && NT == 1 ? 3 : 2;            // that fit an SM
};
template <class T, int NT, int GROUP, bool STREAM>
__global__ void __launch_bounds__(THREADS, RowsShape<T, NT, STREAM>::BLOCKS) g4_rows_kernel(const T *x, int64_t ldx, int rows, const int32_t *offsets,
                                                         int experts, G4Weights w, T *y, int64_t ldy, int log_ranks,
                                                         unsigned int *err, unsigned int wait_limit) {
    constexpr int PARTS = RowType<T>::PARTS, COLS = NT * 8, CAP = COLS / PARTS, GROUPS = G4_TILE / GROUP;
    using L = RowsShape<T, NT, STREAM>;
    extern __shared__ __align__(128) uint8_t smem[];
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF);
    uint64_t *empty = full + C_STAGES;
    volatile uint32_t *abort_flag = reinterpret_cast<uint32_t *>(empty + C_STAGES);
    const uint32_t cs = smem_u32(smem), xs = cs + L::X_OFF;
    const int warp = warp_index(), lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const int ranks = 1 << log_ranks, rank = blockIdx.x & (ranks - 1), jt = blockIdx.x >> log_ranks;

    if (threadIdx.x == 0) {
        for (int s = 0; s < C_STAGES; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], WARPS); }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    wait_for_previous();
    const ExpertSlot slot = expert_slot(offsets, experts, rows, CAP, blockIdx.y);
    if (slot.expert < 0) return;                                        // (for every block of the cluster)
    const int first = (int)((int64_t)w.tiles_k * rank >> log_ranks), last = (int)((int64_t)w.tiles_k * (rank + 1) >> log_ranks);
    const int have = slot.last - slot.first;
    float acc[NT][4] = {};

    if (warp == WARPS) {
        Ring s;
        int64_t tile = ((int64_t)slot.expert * w.tiles_n + jt) * w.tiles_k + first;
        int it = 0;
#pragma unroll 1
        for (int t = first; t < last; t += U, tile += U, ++it) {
            if (!__all_sync(0xffffffffu, short_wait(&empty[s.s], s.ph ^ 1u, abort_flag, 0, err, wait_limit))) break;
            const int here = min(U, last - t);
            uint8_t *stage = smem + s.s * L::STAGE;
            const int end = min(w.k - t * G4_TILE, here * G4_TILE);         // elements of x in this stage
            if constexpr (STREAM) {
                if (end < here * G4_TILE && lane < have) {                  // the contraction ends inside: zeros behind it
                    const uint32_t row = cs + s.s * L::STAGE + C_STAGE + (here - 1) * L::X_TILE + lane * X_PITCH;
#pragma unroll 1
                    for (int o = end - (here - 1) * G4_TILE; o < G4_TILE; o += 8) sts_128(row + o * 2, 0u, 0u, 0u, 0u);
                }
                __syncwarp();
            }
            if (elect_one()) {
                mbar_expect_tx(&full[s.s], here * (G4_TILE_WORDS * 4 + GROUPS * G4_TILE) + (STREAM ? have * end * 2 : 0));
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (u >= here) break;
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        bulk_load(stage + u * C_TILE + q * UNIT_PITCH, w.codes + (tile + u) * G4_TILE_WORDS + q * (UNIT / 4), UNIT, &full[s.s]);
                    bulk_load(stage + u * C_TILE + SCALES_AT, w.scales + (tile + u) * (GROUPS * G4_TILE), GROUPS * G4_TILE, &full[s.s]);
                }
            }
            if constexpr (STREAM) {
                __syncwarp();
                if (lane < have)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (u >= here) break;
                        bulk_load(stage + C_STAGE + u * L::X_TILE + lane * X_PITCH, x + (int64_t)(slot.first + lane) * ldx + (t + u) * G4_TILE,
                                  min(G4_TILE, end - u * G4_TILE) * 2, &full[s.s]);
                    }
            }
            __syncwarp();
            s.next(C_STAGES);
        }
        if (*abort_flag && lane == 0) drain_copies_in_flight(full, it, C_STAGES, wait_limit);
        __syncwarp();
    } else {
        Ring s;
        bool ok = true;
#pragma unroll 1
        for (int t0 = first; t0 < last; t0 += STREAM ? last : L::X_TILES) {      // (a warp that gave up still comes to the barriers)
            const int here = STREAM ? last - first : min(L::X_TILES, last - t0);
            if constexpr (!STREAM) {
                if (t0 > first) multiplying_warps_sync();               // the columns are still being read
                stage_columns<T>(x + (int64_t)slot.first * ldx, ldx, have, t0 * G4_TILE, here, w.k, COLS, xs);
                multiplying_warps_sync();
            }
            const uint32_t at_row = cs + c * UNIT_PITCH + (warp * STRIP + g) * 16;
            const uint32_t at_col = (STREAM ? C_STAGE : L::X_OFF) + g * X_PITCH + c * 16;
#pragma unroll 1
            for (int t = 0; ok && t < here; t += U) {
                if (!(ok = __all_sync(0xffffffffu, short_wait(&full[s.s], s.ph, abort_flag, 1, err, wait_limit)))) break;
                uint4 lo[U], hi[U];                                         // unit c of features g and g + 8 of the strip
                uint8_t blo[U], bhi[U];                                     // their scales of group c
#pragma unroll
                for (int u = 0; u < U; ++u) {                               // (behind an odd end: what an earlier stage left, not used)
                    const uint32_t src = at_row + s.s * L::STAGE + u * C_TILE;
                    lo[u] = lds_128(src);
                    hi[u] = lds_128(src + 128);
                    const uint32_t sc = cs + s.s * L::STAGE + u * C_TILE + SCALES_AT + (GROUPS > 1 ? (c & (GROUPS - 1)) * G4_TILE : 0) + warp * STRIP + g;
                    blo[u] = lds_8(sc);
                    bhi[u] = lds_8(sc + 8);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (t + u >= here) break;
                    const float slo = __fmul_rn(g4_scale_f32(blo[u]), CodeScale<T>::GROUP), shi = __fmul_rn(g4_scale_f32(bhi[u]), CodeScale<T>::GROUP);
                    float sum[NT][2][4];                                    // two chains: an instruction takes long to answer
#pragma unroll
                    for (int ww = 0; ww < 4; ++ww) {
                        if ((ww * 32) % GROUP == 0) {
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int i = 0; i < 8; ++i) sum[n][i >> 2][i & 3] = 0.0f;
                        }
                        const uint32_t wl = ww == 0 ? lo[u].x : ww == 1 ? lo[u].y : ww == 2 ? lo[u].z : lo[u].w;
                        const uint32_t wh = ww == 0 ? hi[u].x : ww == 1 ? hi[u].y : ww == 2 ? hi[u].z : hi[u].w;
                        const uint32_t l0 = code_pair<T>(wl, 0), l1 = code_pair<T>(wl, 1), l2 = code_pair<T>(wl, 2), l3 = code_pair<T>(wl, 3);
                        const uint32_t h0 = code_pair<T>(wh, 0), h1 = code_pair<T>(wh, 1), h2 = code_pair<T>(wh, 2), h3 = code_pair<T>(wh, 3);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint4 b = lds_128(cs + at_col + (STREAM ? s.s * L::STAGE : t * L::X_TILE) + u * L::X_TILE + n * 8 * X_PITCH + ww * 64);
                            mma_16x8x16<T>(sum[n][0], l0, h0, l1, h1, b.x, b.y);
                            mma_16x8x16<T>(sum[n][1], l2, h2, l3, h3, b.z, b.w);
                        }
                        if ((ww * 32 + 32) % GROUP == 0) {
                            const int grp = ww * 32 / GROUP;                // quad lane `grp` holds that group's scales
                            const float s0 = GROUPS == 1 ? slo : __shfl_sync(0xffffffffu, slo, grp, 4);
                            const float s1 = GROUPS == 1 ? shi : __shfl_sync(0xffffffffu, shi, grp, 4);
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                acc[n][0] = __fmaf_rn(s0, __fadd_rn(sum[n][0][0], sum[n][1][0]), acc[n][0]);
                                acc[n][1] = __fmaf_rn(s0, __fadd_rn(sum[n][0][1], sum[n][1][1]), acc[n][1]);
                                acc[n][2] = __fmaf_rn(s1, __fadd_rn(sum[n][0][2], sum[n][1][2]), acc[n][2]);
                                acc[n][3] = __fmaf_rn(s1, __fadd_rn(sum[n][0][3], sum[n][1][3]), acc[n][3]);
                            }
                        }
                    }
                }
                // only now: an arrival does not wait for loads whose values nobody has used yet (the instructions that use them
                // are volatile, so they stay ahead of it)
                __syncwarp();
                if (lane == 0) arrive_local(&empty[s.s]);
                s.next(C_STAGES);
            }
        }
        multiplying_warps_sync();                                       // all tiles have been used: room for the sums
        float *sums = reinterpret_cast<float *>(smem);                  // [128 features][COLS + 1]
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float *at = sums + (warp * STRIP + g) * (COLS + 1) + n * 8 + 2 * c;
            at[0] = acc[n][0];
            at[1] = acc[n][1];
            at[8 * (COLS + 1)] = acc[n][2];
            at[8 * (COLS + 1) + 1] = acc[n][3];
        }
    }
    start_next();       // not earlier: blocks of the next kernel would settle unevenly between this one's (12.6 -> 14.9 us a call
                        // for 16 rows of 64 experts)
    if (log_ranks) cluster_sync();
    else __syncthreads();
    // each rank adds up its share of the features over all ranks, in their order
    const SumScale scale(w.alpha[slot.expert], CodeScale<T>::UNDO);
    const int log_feats = 7 - log_ranks;
#pragma unroll 1
    for (int v = threadIdx.x; v < have << log_feats; v += THREADS) {
        const int f = (rank << log_feats) + (v & ((1 << log_feats) - 1)), r = v >> log_feats, j = jt * G4_TILE + f;
        if (j >= w.n) continue;
        const uint32_t at = cs + (f * (COLS + 1) + r * PARTS) * 4;
        float one[8][PARTS], total = 0.0f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {                                   // all loads first: each takes a round trip
            if (q >= ranks) break;
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(q));
#pragma unroll
            for (int p = 0; p < PARTS; ++p) asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(one[q][p]) : "r"(there + p * 4) : "memory");
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            if (q >= ranks) break;
#pragma unroll
            for (int p = PARTS - 2; p >= 0; --p) one[q][PARTS - 1] = __fadd_rn(one[q][PARTS - 1], one[q][p]);     // smallest first
            total = __fadd_rn(total, one[q][PARTS - 1]);
        }
        real_store(y + (int64_t)(slot.first + r) * ldy + j, scale.of(total));
    }
    if (log_ranks) {                                                    // nobody leaves while its sums are read; they have
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // been, so nothing is waited for but that
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    }
}

template <class T, int NT, int GROUP, bool STREAM>
int launch(const T *x, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, T *y, int64_t ldy, cudaStream_t st) {
    constexpr int CAP = NT * 8 / RowType<T>::PARTS, SMEM = RowsShape<T, NT, STREAM>::TOTAL;
    auto kernel = g4_rows_kernel<T, NT, GROUP, STREAM>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM) != cudaSuccess) return QNN_E_CUDA;
    const int64_t slots = offsets ? expert_slots_most(rows, experts, CAP) : (rows + CAP - 1) / CAP;
    if (slots > 65535) return QNN_E_RANGE;
    // Ranks of a cluster: what ends first when a block costs three tiles' time besides its own, one
    // more for each doubling of the cluster (3 x 4097 x 1000 fp32: 5.6 us with four ranks, 7.6 with eight, 7.2 with one)
    int log_ranks = 0;
    int64_t best = INT64_MAX;
    for (int l = 0; l < 4 && (1 << l) <= w.tiles_k; ++l) {
        const int64_t blocks = slots * w.tiles_n << l, at_once = RowsShape<T, NT, STREAM>::BLOCKS * 148;
        const int64_t rounds = (blocks + at_once - 1) / at_once;
        const int64_t cost = rounds * ((w.tiles_k + (1 << l) - 1) / (1 << l) + 3 + l);
        if (cost < best) { best = cost; log_ranks = l; }
    }
    unsigned int *err = qnn_tc_error_word();
    if (!err) return QNN_E_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(w.tiles_n << log_ranks), (unsigned)slots);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = st;
    LaunchAttrs attrs((1u << log_ranks));
    cfg.attrs = attrs.a;
    cfg.numAttrs = (1u << log_ranks) > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, x, ldx, rows, offsets, experts, w, y, ldy, log_ranks, err, WAIT_LIMIT) != cudaSuccess) {
        cudaGetLastError();
        return QNN_E_CUDA;
    }
    return QNN_OK;
}

template <class T, int NT, bool STREAM>
int by_group(const T *x, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, T *y, int64_t ldy, cudaStream_t st) {
    if (w.group == 32) return launch<T, NT, 32, STREAM>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    if (w.group == 64) return launch<T, NT, 64, STREAM>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    return launch<T, NT, 128, STREAM>(x, ldx, rows, offsets, experts, w, y, ldy, st);
}
template <class T, int NT>
int by_rows(const T *x, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, T *y, int64_t ldy, cudaStream_t st) {
    if constexpr (sizeof(T) == 2)
        if (qnn_aligned(x, 16) && ldx % 8 == 0 && w.k % 8 == 0) return by_group<T, NT, true>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    return by_group<T, NT, false>(x, ldx, rows, offsets, experts, w, y, ldy, st);
}

// Columns per block: eight, one instruction's worth, which hold eight rows of 2-byte elements or two of fp32; sixteen for more
// fp32 rows together (the callers give at most 8 and 4).
template <class T>
int by_columns(const void *xv, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, void *yv, int64_t ldy,
               int rows_together, cudaStream_t st) {
    const T *x = static_cast<const T *>(xv);
    T *y = static_cast<T *>(yv);
    if constexpr (RowType<T>::PARTS > 1)
        if (rows_together * RowType<T>::PARTS > 8) return by_rows<T, 2>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    return by_rows<T, 1>(x, ldx, rows, offsets, experts, w, y, ldy, st);
}

}  // namespace

int qnn_g4_rows(const void *x, int type, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, void *y,
                int64_t ldy, int rows_together, cudaStream_t st) {
    if (type == QNN_F32) return by_columns<float>(x, ldx, rows, offsets, experts, w, y, ldy, rows_together, st);
    if (type == QNN_BF16) return by_columns<__nv_bfloat16>(x, ldx, rows, offsets, experts, w, y, ldy, rows_together, st);
    return by_columns<__half>(x, ldx, rows, offsets, experts, w, y, ldy, rows_together, st);
}
