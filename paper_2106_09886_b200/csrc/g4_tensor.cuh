// Products grouped by expert on the fifth-generation tensor cores: result = weights x rows, accumulated in tensor memory
// with the weight features as the 128 lanes of an accumulator and the rows (tokens) as its columns, so that a stored
// 128 x 128 tile of codes is unpacked once and multiplied with up to 256 tokens.  An expert's last tile multiplies all its
// columns too, whatever rows follow in memory; only the stores stop at the expert's last row.
//
//   G4_FWD   y[r][j]  = alpha sum_i W[j][i] x[r][i]:  lanes j, contraction over i.  A thread owns a lane and unpacks the
//            64 codes of its row straight into the A operand in tensor memory: no shared-memory round trip, one group
//            scale per thread.
//   G4_DATA  dx[r][i] = alpha sum_j W[j][i] dy[r][j]: lanes i, contraction over j.  The same stored tile is needed
//            transposed; it is unpacked row by row into shared memory and read as an MN-major operand, which transposes.
//
// W / alpha = scale * (2t - 15) has at most 8 significant bits: exact in bf16 and fp16, so the only roundings are the
// fp32 additions and the last one to the result's type.  fp32 rows come as three bf16 parts; A is unpacked once for them.
//
// CG = 2: a pair of thread blocks (cluster) works on 256 lanes x TN tokens with cta_group::2 instructions, each block
// holding its 128 lanes of weights and half of the tokens, which halves what is read per product.
//
// Bound, with times in a replayed graph and of calls from Python back to back: the tensor pipe for many tokens (16384 rows,
// eight experts 4096 x 4096, bf16: 390 and 454 us, 1.41 and 1.21 PFLOP/s, the latter under the power cap); unpacking for few
// (1024 rows, 32 experts 2048 x 4096, fp16: 45 and 54 us, some 600 cycles a stored tile); the tensor pipe for the data
// gradient too, where it is busy (86 % of the cycles in which an SM has a block), but 4096 rows on eight 4096 x 4096 experts
// make 20 tiles, a quarter of whose columns are padding, and 320 items for 74 pairs, 4.3 rounds that take 5 (123 and 142 us).
#pragma once
#include "tc_ptx.cuh"
#include "g4_rows.cuh"

namespace {

enum G4Mode { G4_FWD = 0, G4_DATA = 1 };

template <class T> struct G4Type;                       // operand type, parts of a row, instruction-descriptor format
template <> struct G4Type<float> { typedef __nv_bfloat16 Op; static constexpr int PARTS = 3; static constexpr uint32_t FMT = 1; };
template <> struct G4Type<__nv_bfloat16> { typedef __nv_bfloat16 Op; static constexpr int PARTS = 1; static constexpr uint32_t FMT = 1; };
template <> struct G4Type<__half> { typedef __half Op; static constexpr int PARTS = 1; static constexpr uint32_t FMT = 0; };

// ------------------------------------------------------------------------------------------------ pair-aware PTX

template <int CG> __device__ __forceinline__ uint32_t pair_rank() {
    uint32_t r = 0;
    if constexpr (CG == 2) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
template <int CG> __device__ __forceinline__ void pair_sync() {       // every thread of both blocks
    if constexpr (CG == 1) {
        __syncthreads();
    } else {
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}
// Address of the leading block's copy of a barrier (the two blocks lay out their shared memory alike).
template <int CG> __device__ __forceinline__ uint32_t leader_addr(const void *p) {
    uint32_t a = smem_u32(p);
    if constexpr (CG == 2) asm volatile("mapa.shared::cluster.u32 %0, %0, 0;" : "+r"(a));
    return a;
}
// (Without a cluster-scope release, which waits some 1400 cycles for unrelated stores: what the arrival hands over is ordered
// by tcgen05 fences for tensor memory and by the proxy fence for shared memory.)
template <int CG> __device__ __forceinline__ void arrive_leader(uint64_t *bar) {
    if constexpr (CG == 1)
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(leader_addr<2>(bar)) : "memory");
}
// 2-D box into this block's shared memory, its bytes counted on the leading block's barrier.
template <int CG>
__device__ __forceinline__ void pair_load_2d(void *dst, const CUtensorMap *map, uint64_t *bar, int x, int y) {
    if constexpr (CG == 1)
        tma_load_2d(dst, map, bar, x, y);
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
            ::"r"(smem_u32(dst)), "l"(map), "r"(leader_addr<2>(bar)), "r"(x), "r"(y) : "memory");
}
template <int CG> __device__ __forceinline__ void pair_tmem_alloc(uint32_t *slot, uint32_t ncols) {   // one whole warp per block
    if constexpr (CG == 1) {
        tmem_alloc(slot, ncols);
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(slot)), "r"(ncols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CG> __device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t ncols) {
    if constexpr (CG == 1) tmem_dealloc(taddr, ncols);
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
}
// Arrives on the barrier (of both blocks) when the instructions issued so far have completed.
template <int CG> __device__ __forceinline__ void pair_commit(uint64_t *bar) {
    if constexpr (CG == 1)
        tc_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// D (+)= A * B^T, 16 steps of the contraction; A in tensor memory (TS) or shared memory (SS), B in shared memory.
template <int CG>
__device__ __forceinline__ void mma_f16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_f16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// 16 columns of this thread's lane.
__device__ __forceinline__ void tmem_store_16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_load_lane_16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory descriptor of an MN-major tile with the 128-byte swizzle: blocks of 64 elements of the M (or N) dimension
// (128 bytes) x the contraction's rows; rows in groups of 8 (1024 bytes apart, the stride offset), the next 64 elements
// `block_bytes` further (the leading offset).  16 steps of the contraction are 2048 bytes.
__device__ __forceinline__ uint64_t smem_desc_mn_sw128(uint32_t saddr, uint32_t block_bytes) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)(block_bytes >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor of kind::f16 with fp32 accumulation: formats (0 fp16, 1 bf16) at bits 7 and 10, transposition of
// A and B (MN-major) at bits 15 and 16, N/8 at bit 17, M/16 at bit 24.
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t fmt, int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (fmt << 7) | (fmt << 10) | ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) |
           ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// Blocks of TN rows, counted expert by expert, visited in increasing order by a whole warp.
struct SlotCursor {
    const int32_t *offsets;
    int experts, rows, tile;
    int base = 0, before = 0, a = 0, b = 0, mine = 0, incl = 0;
    __device__ __forceinline__ SlotCursor(const int32_t *o, int e, int r, int t) : offsets(o), experts(e), rows(r), tile(t) { load(); }
    __device__ __forceinline__ void load() {
        const int lane = threadIdx.x & 31;
        a = b = 0;
        if (base + lane < experts) expert_rows(offsets, base + lane, rows, a, b);
        mine = b > a ? (b - a + tile - 1) / tile : 0;
        incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += o;
        }
    }
    __device__ __forceinline__ ExpertSlot seek(int slot) {
#pragma unroll 1
        while (base < experts) {
            const unsigned hit = __ballot_sync(0xffffffffu, slot < before + incl);
            if (hit) {
                const int src = __ffs(hit) - 1;
                const int first = __shfl_sync(0xffffffffu, a, src) + (slot - before - __shfl_sync(0xffffffffu, incl - mine, src)) * tile;
                return {base + src, first, min(__shfl_sync(0xffffffffu, b, src), first + tile)};
            }
            before += __shfl_sync(0xffffffffu, incl, 31);
            base += 32;
            if (base < experts) load();
        }
        return {-1, 0, 0};
    }
};

// Blocks of `tile` rows in all; by a whole warp.
__device__ __noinline__ int64_t count_slots(const int32_t *offsets, int experts, int rows, int tile) {
    int64_t total = 0;
    for (int e = threadIdx.x & 31; e < experts; e += 32) {
        int a, b;
        expert_rows(offsets, e, rows, a, b);
        total += b > a ? (b - a + tile - 1) / tile : 0;
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    return total;
}

// Work item t: a part of the contraction of a tile of features x a block of rows.
struct G4Item {
    int slot, f, part, lo, steps;
};
__device__ __noinline__ G4Item g4_item(int t, int parts, int ftiles, int steps, int steps_each) {
    const int tile = t / parts, part = t - tile * parts, slot = tile / ftiles;
    return {slot, tile - slot * ftiles, part, part * steps_each, min(steps_each, steps - part * steps_each)};
}
// Steps of the items first, first + stride, ...
__device__ __noinline__ int64_t g4_stages(int64_t items, int first, int stride, int parts, int steps, int steps_each) {
    int64_t total = 0;
    if (parts == 1) return items > first ? (items - first + stride - 1) / stride * steps : 0;
#pragma unroll 1
    for (int64_t t = first; t < items; t += stride) total += min(steps_each, steps - (int)(t % parts) * steps_each);
    return total;
}

struct G4TensorParams {
    G4Weights w;
    const int32_t *offsets;
    int experts, rows;
    void *out;
    int64_t ldo;
    int features;                         // width of the result
    int ftiles;                           // tiles of 128 * CG features
    int steps;                            // stored tiles along the contraction
    // Most items that offsets in order can make, below 2^30.  Offsets that decrease can name the same rows again and again and
    // make more items than 31 bits count; every role stops here.
    int items;
    // With few tiles the contraction is split: `parts` items of steps_each (the last one maybe fewer) steps per tile, whose
    // fp32 results go to sums [part][rows][features], to be added in order by g4_sum_parts_kernel.
    int parts, steps_each;
    float *sums;
    bool out_vec;                         // the result's rows start and advance by whole 16 bytes
    unsigned int *err;
    unsigned int wait_limit;
};

// Warps: 0 rows by TMA, 1 matrix instructions, 2 codes by bulk copies (and owner of the tensor memory), 3 idle, 4-7 results,
// from 8 on groups of four that unpack.
constexpr int G4_UNPACK_WARPS = 4;

// A stage is one stored tile of the contraction (128 steps): its unpacked weights (64 columns of tensor memory, or 32 KB
// of shared memory) and the rows' parts.  Both halves of a stage fill and empty on one pair of barriers.
template <int CG, int TN, int MODE, int PARTS>
struct G4Shape {
    static constexpr int XROWS = TN / CG;                       // tokens whose rows this block stages
    static constexpr int X_SUB = XROWS * 128;                   // 64 columns of them, 128-byte swizzle
    static constexpr int X_PART = 2 * X_SUB;
    static constexpr int A_STAGE = MODE == G4_DATA ? 128 * 128 * 2 : 0;
    static constexpr int STAGE = PARTS * X_PART + A_STAGE;
    static constexpr int C_STAGE = G4_TILE_WORDS * 4 + 512;     // codes and up to four rows of scales
    // deep where reading the codes is the bound; two where that makes room for a third stage
    static constexpr int C_STAGES = TN <= 64 && PARTS == 1 && MODE == G4_FWD ? 8 : (MODE == G4_DATA && TN > 128 ? 2 : 4);
    // Two accumulators, so that results are stored under the next sum, where tensor memory has room for them.
    static constexpr int ACC_BUFS = (MODE == G4_DATA ? 2 * TN <= 512 : 2 * TN <= 256) ? 2 : 1;
    static constexpr int ACC_COLS = ACC_BUFS * TN;
    // fp32: sums leave tensor memory after every stage (see PROMOTE in the kernel)
    static constexpr int OUT_WARP = PARTS == 1 ? 32 * 80 : 0;   // transposing buffer of a result warp: 32 tokens x 32 features
    static constexpr int FIXED = C_STAGES * C_STAGE + 4 * OUT_WARP + 2048;
    static constexpr int FIT_SMEM = (227 * 1024 - FIXED) / STAGE;
    static constexpr int FIT_TMEM = MODE == G4_DATA ? 8 : (512 - ACC_COLS) / 64;
    static constexpr int STAGES = FIT_SMEM < FIT_TMEM ? FIT_SMEM : FIT_TMEM;
    // Groups of unpacking warps, each with a stage of its own.  One tile takes a warp some 1100 cycles: two groups keep up
    // with the 1024 (or 512) cycles that wide tiles multiply for, narrow ones are bound by unpacking and take what fits.
    static constexpr int GROUPS = PARTS > 1 || TN > 64 || STAGES < 4 ? 2 : 4;
    static constexpr int THREADS = 256 + 128 * GROUPS;
    static constexpr bool ONE_THREAD = TN <= 64;
    static constexpr int C_OFF = STAGES * STAGE;
    static constexpr int OUT_OFF = C_OFF + C_STAGES * C_STAGE;
    static constexpr int BAR_OFF = OUT_OFF + 4 * OUT_WARP;
    static constexpr int USED = BAR_OFF + (2 * (STAGES + C_STAGES) + 5) * 8 + 16 + 1024;
    // At least half of an SM's shared memory, so that a block of the next kernel, started early, never waits for tensor memory
    // that this one holds.
    static constexpr int TOTAL = USED > 115 * 1024 ? USED : 115 * 1024;
    // A group waits for a phase by its parity, so it must know that the phase before has completed.  Copies of codes may land
    // out of order: a stage of codes has to come back to the group that waited for it last.  (Unpacked stages are freed in
    // order, and a group that is G stages on has seen one S + G back freed, which covers the phase before for G <= S.)
    static_assert(C_STAGES % GROUPS == 0 && GROUPS <= STAGES, "groups and rings");
    static_assert(STAGES >= 2 && TOTAL <= 227 * 1024, "shared memory");
};

// A group's scale as the unpacking needs it.  A masked nibble is an integer multiple of the smallest step of its format:
//   bf16  the bare nibble is the subnormal t * 2^-133, and one fused multiply-add by s * 2^119 makes s * (2t - 15) * 2^-15
//         (the power of two that keeps the factor finite; the results are multiplied by 2^15);
//   fp16  the nibble under the exponent of 1024 is 1024 + t or 1024 + 16t; less 1024, times 2s or s/8, minus 15s.
// Every step is exact: s has 4 significant bits, 15s and s * q have 8.
template <class Op> struct GroupScale;
template <> struct GroupScale<__nv_bfloat16> {
    static constexpr float UNDO = 32768.0f;
    __nv_bfloat162 mul, add;
    __device__ __forceinline__ explicit GroupScale(uint8_t b) {
        const float s = g4_scale_f32(b);
        mul = __float2bfloat162_rn(__fmul_rn(s, 6.646139978924579e+35f));          // 2^119
        add = __float2bfloat162_rn(__fmul_rn(s, -15.0f / 32768.0f));
    }
};
template <> struct GroupScale<__half> {
    static constexpr float UNDO = 1.0f;
    __half2 mul0, mul1, add;
    __device__ __forceinline__ explicit GroupScale(uint8_t b) {
        const __half2 s = __float2half2_rn(g4_scale_f32(b));
        mul0 = __hadd2(s, s);
        mul1 = __hmul2(s, __half2half2(__ushort_as_half(0x3000)));                  // 1/8
        add = __hmul2(s, __half2half2(__ushort_as_half(0xCB80)));                   // -15
    }
};

// Eight codes of a word -> four packed pairs of scale * q (times 1 / UNDO).
__device__ __forceinline__ void unpack_word(uint32_t word, const GroupScale<__nv_bfloat16> &s, uint32_t *out) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t u = (word >> (4 * p)) & 0x000F000Fu;
        const __nv_bfloat162 v = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u), s.mul, s.add);
        out[p] = *reinterpret_cast<const uint32_t *>(&v);
    }
}
__device__ __forceinline__ void unpack_word(uint32_t word, const GroupScale<__half> &s, uint32_t *out) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        uint32_t u;
        const uint32_t w = p < 2 ? word : word >> 8;
        if (p & 1) asm("lop3.b32 %0, %1, 0x00F000F0, 0x64006400, 0xEA;" : "=r"(u) : "r"(w));
        else asm("lop3.b32 %0, %1, 0x000F000F, 0x64006400, 0xEA;" : "=r"(u) : "r"(w));
        const __half2 d = __hadd2(*reinterpret_cast<const __half2 *>(&u), __half2half2(__ushort_as_half(0xE400)));    // -1024
        const __half2 v = __hfma2(d, (p & 1) ? s.mul1 : s.mul0, s.add);
        out[p] = *reinterpret_cast<const uint32_t *>(&v);
    }
}

// 16 lanes x 32 columns: register 4i + {0, 1} of lane l holds row l/4, columns 8i + 2(l%4) + {0, 1}; + {2, 3} row l/4 + 8.
__device__ __forceinline__ void tmem_load_16x32(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
}
template <class T> __device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&v);
    }
}

// 32 tokens x 32 features of an accumulator (lanes = features) -> rows of a 2-byte result.  The quarter is transposed on its
// way through shared memory (80 bytes a token: every store and load below is free of bank conflicts), so that a token's
// features leave as 16-byte stores.  `f` the first feature, `vec`: rows start and advance by whole 16 bytes.
template <class T>
__device__ __forceinline__ void store_quarter(uint32_t taddr, uint32_t buf, T *row0, int64_t ldo, int tokens, int f, int features,
                                              SumScale scale, bool vec) {
    const int lane = threadIdx.x & 31;
    const uint32_t at = buf + ((lane >> 4) * 8 + (lane & 7)) * 80 + ((lane >> 3) & 1) * 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t r[16];
        tmem_load_16x32(taddr + ((uint32_t)(16 * h) << 16), r);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
        uint32_t v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = pack_pair<T>(scale.of(__uint_as_float(r[2 * i])), scale.of(__uint_as_float(r[2 * i + 1])));
#pragma unroll
        for (int i = 0; i < 2; ++i)                       // tokens 16i .. 16i + 15, features 16h .. 16h + 15
            asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};"
                         ::"r"(at + i * 16 * 80 + h * 32), "r"(v[4 * i]), "r"(v[4 * i + 1]), "r"(v[4 * i + 2]), "r"(v[4 * i + 3]) : "memory");
    }
    __syncwarp();
    const int f0 = f + (lane >> 3) * 8;
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = lds_128(buf + (i * 8 + (lane & 7)) * 80 + (lane >> 3) * 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int token = i * 8 + (lane & 7);
        if (token < tokens) {
            T *dst = row0 + (int64_t)token * ldo + f0;
            if (vec && f0 + 8 <= features) {
                *reinterpret_cast<uint4 *>(dst) = v[i];
            } else {
                const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (f0 + j < features) reinterpret_cast<uint16_t *>(dst)[j] = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            }
        }
    }
    __syncwarp();
}

template <int CG, int TN, int MODE, class T>
__global__ void __launch_bounds__(G4Shape<CG, TN, MODE, G4Type<T>::PARTS>::THREADS, 1) g4_tensor_kernel(const __grid_constant__ CUtensorMap map_x, const G4TensorParams p) {
    using Op = typename G4Type<T>::Op;
    constexpr int PARTS = G4Type<T>::PARTS;
    using L = G4Shape<CG, TN, MODE, PARTS>;
    // The tensor cores cut a sum towards zero at every addition, which for a long contraction is a hundred times the
    // rounding of an fp32 result.  fp32 results therefore add up only one stage in tensor memory (smallest parts first) and
    // the result warps add the stages in registers, to nearest.
    constexpr bool PROMOTE = PARTS > 1;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_at = smem_u32(smem);
    uint64_t *full = reinterpret_cast<uint64_t *>(smem + L::BAR_OFF);       // leader: both blocks' rows and unpacked weights
    uint64_t *empty = full + L::STAGES;                                     // each block: the instructions have read a stage
    uint64_t *c_full = empty + L::STAGES;                                   // each block: its codes have landed
    uint64_t *c_empty = c_full + L::C_STAGES;
    uint64_t *acc_full = c_empty + L::C_STAGES;                             // each block
    uint64_t *acc_empty = acc_full + 2;                                     // leader: both blocks have read an accumulator out
    uint64_t *finish = acc_empty + 2;                                       // every instruction has completed
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(finish + 1);
    volatile uint32_t *abort_flag = tmem_slot + 1;

    const int warp = warp_index(), lane = threadIdx.x & 31;
    const int rank = (int)pair_rank<CG>();
    const int first_work = blockIdx.x / CG, work_stride = gridDim.x / CG;

    if (threadIdx.x == 0) {
#pragma unroll 1
        for (int s = 0; s < L::STAGES; ++s) { mbar_init(&full[s], G4_UNPACK_WARPS * CG + 1); mbar_init(&empty[s], 1); }
#pragma unroll 1
        for (int s = 0; s < L::C_STAGES; ++s) { mbar_init(&c_full[s], 1); mbar_init(&c_empty[s], G4_UNPACK_WARPS); }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], 4 * CG); }
        mbar_init(finish, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) pair_tmem_alloc<CG>(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    pair_sync<CG>();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    start_next();
    wait_for_previous();
    // waits of a whole warp: every lane polls (each needs the barrier's acquire), all go on or all give up
    auto warp_wait = [&](uint64_t *bar, uint32_t parity, unsigned id) {
        return __all_sync(0xffffffffu, short_wait(bar, parity, abort_flag, id, p.err, p.wait_limit));
    };
    auto item = [&](int t) { return g4_item(t, p.parts, p.ftiles, p.steps, p.steps_each); };
    auto stages_of_this_block = [&]() {
        const int64_t items = count_slots(p.offsets, p.experts, p.rows, TN) * p.ftiles * p.parts;
        return g4_stages(items < p.items ? items : p.items, first_work, work_stride, p.parts, p.steps, p.steps_each);
    };
    auto stop = [&]() { return __any_sync(0xffffffffu, *abort_flag != 0); };       // the same answer for a whole warp

    // The matrix instructions of `left` stages; agree() and alone() say how a wait's outcome is shared and who issues.
    auto issue_stages = [&](int64_t left, auto agree, auto alone) {
        Ring acc;
        constexpr uint32_t idesc = idesc_f16(G4Type<T>::FMT, 128 * CG, TN, MODE == G4_DATA, false);
        const uint64_t b_desc = smem_desc_k_sw128(smem_at);
        const uint64_t a_desc = smem_desc_mn_sw128(smem_at + PARTS * L::X_PART, 128 * 128);
        bool ok = true;
        uint32_t ph = 0;
        int kt = 0, t = first_work, steps = item(t).steps;
#pragma unroll 1
        for (; ok && left > 0; ph ^= 1u) {
#pragma unroll
            for (int g = 0; g < L::STAGES; ++g) {
                if (left-- <= 0) break;
                const bool fresh = PROMOTE || kt == 0, done = PROMOTE || kt == steps - 1;
                if (fresh && !(ok = agree(short_wait(&acc_empty[acc.s], acc.ph ^ 1u, abort_flag, 3, p.err, p.wait_limit)))) break;
                if (!(ok = agree(short_wait(&full[g], ph, abort_flag, 1, p.err, p.wait_limit)))) break;
                tc_fence_after();
                const uint32_t d = tmem_base + (uint32_t)(acc.s * TN);
                alone([&]() {
#pragma unroll
                    for (int part = PARTS - 1; part >= 0; --part) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const uint64_t bd = b_desc + ((g * L::STAGE + part * L::X_PART + (j >> 2) * L::X_SUB) >> 4) + 2 * (j & 3);
                            const uint32_t more = part != PARTS - 1 || j != 0 ? 1u : (fresh ? 0u : 1u);
                            if constexpr (MODE == G4_FWD) mma_f16_ts<CG>(d, tmem_base + L::ACC_COLS + g * 64 + 8 * j, bd, idesc, more);
                            else mma_f16_ss<CG>(d, a_desc + ((g * L::STAGE) >> 4) + 128 * j, bd, idesc, more);
                        }
                    }
                    pair_commit<CG>(&empty[g]);
                    if (done) pair_commit<CG>(&acc_full[acc.s]);
                });
                if (done) acc.next(L::ACC_BUFS);
                if (++kt == steps) {
                    kt = 0;
                    t += work_stride;
                    steps = item(t).steps;
                }
            }
        }
    };

    if (warp == 0) {                      // ------------------------------------------------ rows
        SlotCursor cur(p.offsets, p.experts, p.rows, TN);
        Ring g;
        long long it = 0;
#pragma unroll 1
        for (int t = first_work; t < p.items && !stop(); t += work_stride) {
            const G4Item work = item(t);
            const ExpertSlot slot = cur.seek(work.slot);
            if (slot.expert < 0) break;
            const int row = slot.first + rank * L::XROWS, lo = work.lo, hi = lo + work.steps;
            bool ok = true;
#pragma unroll 1
            for (int kt = lo; kt < hi; ++kt) {
                if (!(ok = warp_wait(&empty[g.s], g.ph ^ 1u, 0))) break;
                if (elect_one()) {
                    if (rank == 0) mbar_expect_tx(&full[g.s], CG * PARTS * L::X_PART);
                    uint8_t *dst = smem + g.s * L::STAGE;
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        pair_load_2d<CG>(dst + part * L::X_PART, &map_x, &full[g.s], kt * 128, part * p.rows + row);
                        pair_load_2d<CG>(dst + part * L::X_PART + L::X_SUB, &map_x, &full[g.s], kt * 128 + 64, part * p.rows + row);
                    }
                }
                __syncwarp();
                g.next(L::STAGES);
                ++it;
            }
            if (!ok) break;
        }
        // after an abort the copies in flight may still land (their barriers may never complete, with unpacking stopped)
        if (*abort_flag && it > 0)
#pragma unroll 1
            for (int i = 0; i < 1000; ++i) __nanosleep(1000);
    } else if (warp == 2) {               // ------------------------------------------------ codes and scales
        SlotCursor cur(p.offsets, p.experts, p.rows, TN);
        Ring c;
        long long it = 0;
        const int groups = G4_TILE / p.w.group;
        const int64_t stride = MODE == G4_FWD ? 1 : p.w.tiles_k;            // stored tiles between steps of the contraction
#pragma unroll 1
        for (int t = first_work; t < p.items && !stop(); t += work_stride) {
            const G4Item work = item(t);
            const ExpertSlot slot = cur.seek(work.slot);
            if (slot.expert < 0) break;
            // a block whose features lie past the end repeats the last tile; its results are not stored
            const int f = min(work.f * CG + rank, (MODE == G4_FWD ? p.w.tiles_n : p.w.tiles_k) - 1);
            int64_t tile = (int64_t)slot.expert * p.w.tiles_n * p.w.tiles_k + (MODE == G4_FWD ? (int64_t)f * p.w.tiles_k : f) + work.lo * stride;
            bool ok = true;
#pragma unroll 1
            for (int kt = 0; kt < work.steps; ++kt, tile += stride) {
                if (!(ok = warp_wait(&c_empty[c.s], c.ph ^ 1u, 0))) break;
                if (elect_one()) {
                    mbar_expect_tx(&c_full[c.s], G4_TILE_WORDS * 4 + groups * G4_TILE);
                    uint8_t *dst = smem + L::C_OFF + c.s * L::C_STAGE;
                    bulk_load(dst, p.w.codes + tile * G4_TILE_WORDS, G4_TILE_WORDS * 4, &c_full[c.s]);
                    bulk_load(dst + G4_TILE_WORDS * 4, p.w.scales + tile * (groups * G4_TILE), groups * G4_TILE, &c_full[c.s]);
                }
                __syncwarp();
                c.next(L::C_STAGES);
                ++it;
            }
            if (!ok) break;
        }
        if (*abort_flag && lane == 0) drain_copies_in_flight(c_full, it, L::C_STAGES, p.wait_limit);
    } else if (warp == 1) {               // ------------------------------------------------ matrix instructions
        if (rank == 0) {
            // It needs the number of stages, not whose tiles they are.  Wide tiles: the whole warp walks along and one lane
            // issues, which keeps the operands' addresses in uniform registers.  Narrow tiles: one thread does it all, which
            // makes the waits cheaper; there they take longer than the instructions.
            const int64_t total = stages_of_this_block();
            if constexpr (L::ONE_THREAD) {
                if (elect_one()) issue_stages(total, [](bool ok) { return ok; }, [](auto f) { f(); });
            } else {
                issue_stages(total, [](bool ok) { return (bool)__all_sync(0xffffffffu, ok); }, [](auto f) { if (elect_one()) f(); __syncwarp(); });
            }
            __syncwarp();
            // no instruction may still write tensor memory when it is given back: one more commit, waited for
            if (elect_one()) pair_commit<CG>(finish);
            __syncwarp();
#pragma unroll 1
            for (uint32_t w = 0; w < p.wait_limit && !mbar_try_wait(finish, 0u); ++w) {}
        }
    } else if (warp >= 8) {               // ------------------------------------------------ unpacking
        // The groups take stored tiles in turn, a thread unpacks a whole row of one: the waits and latencies of one group are
        // covered by the others' arithmetic.  Which tile it is does not matter here.
        const int q = warp & 3, group = (warp - 8) >> 2;
        const int r = q * 32 + lane;
        const int log_group = p.w.group == 32 ? 5 : p.w.group == 64 ? 6 : 7;
        Ring c, g;
        c.s = g.s = group;
#pragma unroll 1
        for (int64_t left = stages_of_this_block() - group; left > 0; left -= L::GROUPS, c.skip(L::GROUPS, L::C_STAGES), g.skip(L::GROUPS, L::STAGES)) {
            if (!warp_wait(&c_full[c.s], c.ph, 1)) break;
            const uint32_t src = smem_at + L::C_OFF + c.s * L::C_STAGE;
            uint4 u4[4];                                   // word w of unit u: columns 32w + 8u .. + 7 of row r
#pragma unroll
            for (int u = 0; u < 4; ++u) u4[u] = lds_128(src + u * 2048 + r * 16);
            uint8_t sb[4];
            sb[0] = lds_8(src + G4_TILE_WORDS * 4 + r);
#pragma unroll
            for (int w = 1; w < 4; ++w)
                sb[w] = log_group == 7 ? sb[0] : lds_8(src + G4_TILE_WORDS * 4 + ((32 * w) >> log_group) * G4_TILE + r);
            if (!warp_wait(&empty[g.s], g.ph ^ 1u, 0)) break;
            if constexpr (MODE == G4_FWD) {
                // lane r of the A operand, 16 tensor-memory columns (32 codes) at a time
                tc_fence_after();
                const uint32_t at = tmem_base + ((uint32_t)(q * 32) << 16) + L::ACC_COLS + g.s * 64;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t v[16];
                    const GroupScale<Op> s(sb[w]);
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        unpack_word(w == 0 ? u4[u].x : w == 1 ? u4[u].y : w == 2 ? u4[u].z : u4[u].w, s, v + 4 * u);
                    tmem_store_16(at + 16 * w, v);
                }
                tmem_store_wait();
                tc_fence_before();
            } else {
                // row r of the contraction: eight lanes a word, 16 bytes of the MN-major operand
                const uint32_t dst = smem_at + g.s * L::STAGE + PARTS * L::X_PART + r * 128;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const GroupScale<Op> s(sb[w]);
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        uint32_t v[4];
                        unpack_word(w == 0 ? u4[u].x : w == 1 ? u4[u].y : w == 2 ? u4[u].z : u4[u].w, s, v);
                        const int chunk = (w & 1) * 4 + u;
                        sts_128(dst + (w >> 1) * (128 * 128) + ((chunk ^ (r & 7)) << 4), v[0], v[1], v[2], v[3]);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            __syncwarp();
            if (lane == 0) {
                arrive_local(&c_empty[c.s]);              // only now: an arrival does not wait for loads nobody has used yet
                arrive_leader<CG>(&full[g.s]);
            }
        }
    } else if (warp >= 4) {               // ------------------------------------------------ results
        SlotCursor cur(p.offsets, p.experts, p.rows, TN);
        const int q = warp & 3;
        Ring acc;
#pragma unroll 1
        for (int t = first_work; t < p.items && !stop(); t += work_stride) {
            const G4Item work = item(t);
            const ExpertSlot slot = cur.seek(work.slot);
            if (slot.expert < 0) break;
            const int f = (work.f * CG + rank) * 128 + q * 32;
            const SumScale scale(p.w.alpha[slot.expert], GroupScale<Op>::UNDO);
            T *dst = static_cast<T *>(p.out) + (int64_t)slot.first * p.ldo;
            const int have = slot.last - slot.first;
            const uint32_t lanes = (uint32_t)(q * 32) << 16;
            float *sums = p.sums + ((int64_t)work.part * p.rows + slot.first) * p.features + f + lane;      // (only with parts)
            bool ok = true;
            if constexpr (PROMOTE) {
                float sum[TN];
#pragma unroll
                for (int i = 0; i < TN; ++i) sum[i] = 0.0f;
                #pragma unroll 1
                for (int kt = 0; kt < work.steps; ++kt) {
                    if (!(ok = warp_wait(&acc_full[acc.s], acc.ph, 2))) break;
                    tc_fence_after();
#pragma unroll
                    for (int c0 = 0; c0 < TN; c0 += 32) {
                        uint32_t v[32];
                        tmem_load_32(tmem_base + lanes + (uint32_t)(acc.s * TN + c0), v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[c0 + i] = __fadd_rn(sum[c0 + i], __uint_as_float(v[i]));
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_leader<CG>(&acc_empty[acc.s]);
                    acc.next(L::ACC_BUFS);
                }
                if (ok && f + lane < p.features)
#pragma unroll
                    for (int i = 0; i < TN; ++i)
                        if (i < have) {
                            const float v = scale.of(sum[i]);
                            if (p.parts == 1) real_store(dst + (int64_t)i * p.ldo + f + lane, v);
                            else sums[(int64_t)i * p.features] = v;
                        }
            } else {
                if ((ok = warp_wait(&acc_full[acc.s], acc.ph, 2))) {
                    tc_fence_after();
                    const uint32_t buf = smem_at + L::OUT_OFF + q * L::OUT_WARP;
                    if (p.parts > 1) {
#pragma unroll 1
                        for (int c0 = 0; c0 < have; c0 += 16) {
                            uint32_t v[16];
                            tmem_load_lane_16(tmem_base + lanes + (uint32_t)(acc.s * TN + c0), v);
                            if (f + lane < p.features) {
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    if (c0 + i < have) sums[(int64_t)(c0 + i) * p.features] = scale.of(__uint_as_float(v[i]));
                            }
                            __syncwarp();
                        }
                    } else {
#pragma unroll 1
                    for (int c0 = 0; c0 < have; c0 += 32)
                        store_quarter<T>(tmem_base + lanes + (uint32_t)(acc.s * TN + c0), buf, dst + (int64_t)c0 * p.ldo, p.ldo, have - c0, f,
                                         p.features, scale, p.out_vec);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) arrive_leader<CG>(&acc_empty[acc.s]);
                    acc.next(L::ACC_BUFS);
                }
            }
            if (!ok) break;
        }
    }
    tc_fence_before();
    __syncthreads();
    pair_sync<CG>();
    if (warp == 2) {
        tc_fence_after();
        pair_tmem_dealloc<CG>(tmem_base, 512);
    }
}

// ------------------------------------------------------------------------------------------------ host side

// Tensor map of a row-major matrix of 2-byte elements: boxes of 64 columns x box_rows rows, 128-byte swizzle, zeros outside.
inline bool make_map_16(CUtensorMap *map, bool fp16, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    EncodeTiledFn fn = encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * 2};
    cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(map, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(base), dims,
              strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// out[r][f] = sum over the parts, in order, of the rows that belong to an expert.
template <class T>
__global__ void __launch_bounds__(256) g4_sum_parts_kernel(const float *sums, int parts, int rows, int features,
                                                          const int32_t *offsets, int experts, T *out, int64_t ldo) {
    start_next();
    wait_for_previous();
    int first = 0, last = rows;
    if (offsets) {
        first = min(max(offsets[0], 0), rows);
        last = min(max(offsets[experts], 0), rows);
    }
    const int f = blockIdx.x * 256 + threadIdx.x;
    if (f >= features) return;
    for (int r = first + blockIdx.y; r < last; r += gridDim.y) {
        const float *src = sums + (int64_t)r * features + f;
        float v[8], total = 0.0f;
#pragma unroll
        for (int p = 0; p < 8; ++p) v[p] = p < parts ? __ldcs(src + (int64_t)p * rows * features) : 0.0f;
#pragma unroll
        for (int p = 0; p < 8; ++p) total = __fadd_rn(total, v[p]);
        real_store(out + (int64_t)r * ldo + f, total);
    }
}

// x: operand rows of G4Type<T>::Op, [PARTS * rows][ldx], 16-byte aligned rows, `width` columns.
template <int CG, int TN, int MODE, class T>
int g4_tensor_launch(const void *x, int64_t ldx, int width, G4TensorParams p, int sms, cudaStream_t st) {
    using L = G4Shape<CG, TN, MODE, G4Type<T>::PARTS>;
    auto kernel = g4_tensor_kernel<CG, TN, MODE, T>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::TOTAL) != cudaSuccess) return QNN_E_CUDA;
    CUtensorMap map;
    if (!make_map_16(&map, std::is_same<T, __half>::value, x, (int64_t)p.rows * G4Type<T>::PARTS, width, ldx, L::XROWS)) return QNN_E_CUDA;
    p.ftiles = (g4_tiles(p.features) + CG - 1) / CG;
    const int64_t work = expert_slots_most(p.rows, p.experts, TN) * p.ftiles * p.parts;
    if (work > 0x3FFFFFFFll) return QNN_E_RANGE;
    p.items = (int)work;
    const int most = sms / CG;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((work < most ? work : most) * CG));
    cfg.blockDim = dim3(L::THREADS);
    cfg.dynamicSmemBytes = L::TOTAL;
    cfg.stream = st;
    LaunchAttrs attrs(CG);
    cfg.attrs = attrs.a;
    cfg.numAttrs = CG > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, map, p) != cudaSuccess) {
        cudaGetLastError();
        return QNN_E_CUDA;
    }
    if (p.parts > 1) {
        const dim3 grid((unsigned)((p.features + 255) / 256), (unsigned)(p.rows < 1024 ? p.rows : 1024));
        return launch_early(g4_sum_parts_kernel<T>, grid, 256, st, p.sums, p.parts, p.rows, p.features, p.offsets, p.experts,
                            static_cast<T *>(p.out), p.ldo);
    }
    return QNN_OK;
}

}  // namespace
