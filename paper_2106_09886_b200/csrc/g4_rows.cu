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
// fp32 rows are split exactly into three bf16 parts (8 + 8 + 8 bits) that occupy three of the instruction's columns.
#include "g4_rows.cuh"

namespace {

constexpr int WARPS = 8;
constexpr int STRIP = 16;                                 // features of one matrix instruction

template <class T> struct RowType;
template <> struct RowType<__nv_bfloat16> { static constexpr int PARTS = 1; };
template <> struct RowType<__half> { static constexpr int PARTS = 1; };
template <> struct RowType<float> { static constexpr int PARTS = 3; };

// Pair p of a code word as numbers of the operand's type, exact:
//   bf16  the bare nibble is the subnormal t * 2^-133; times 2^127 minus 15 * 2^-7 it is q / 128;
//   fp16  the nibble under the exponent of 1024 is 1024 + 16t; an eighth of it minus 143 is q.
template <class T> struct CodeScale { static constexpr float UNDO = 128.0f; };
template <> struct CodeScale<__half> { static constexpr float UNDO = 1.0f; };
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

template <class T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight consecutive elements x[i .. i+7] of a row as four packed pairs: this lane's column of the B operand.  `part`
// selects the part of a split fp32 row.  VEC: rows start and advance by whole 16 bytes.  Elements from k on are zero.
template <class T, bool VEC>
__device__ __forceinline__ uint4 load_octet(const T *__restrict__ row, int i, int k, int part) {
    if (row == nullptr || i >= k) return make_uint4(0u, 0u, 0u, 0u);
    if constexpr (sizeof(T) == 2) {
        if (VEC && i + 8 <= k) return __ldg(reinterpret_cast<const uint4 *>(row + i));
        uint16_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = i + j < k ? __ldg(reinterpret_cast<const unsigned short *>(row) + i + j) : (uint16_t)0;
        return make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
    } else {
        float v[8];
        if (VEC && i + 8 <= k) {
            const float4 lo = __ldg(reinterpret_cast<const float4 *>(row + i)), hi = __ldg(reinterpret_cast<const float4 *>(row + i) + 1);
            v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = i + j < k ? __ldg(row + i + j) : 0.0f;
        }
        uint32_t b[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) b[j] = split_part_bits(v[j], part);
        return make_uint4(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632), __byte_perm(b[4], b[5], 0x7632), __byte_perm(b[6], b[7], 0x7632));
    }
}

// A thread block computes 16 * (8 / kparts) features for one block of rows (NT * 8 / PARTS of them); its warps are
// arranged as 8 / kparts feature strips x kparts parts of the contraction, whose sums are added in a fixed order.
template <class T, int NT, int GROUP, bool VEC>
__global__ void __launch_bounds__(WARPS * 32) g4_rows_kernel(const T *__restrict__ x, int64_t ldx, int rows,
                                                            const int32_t *__restrict__ offsets, int experts, G4Weights w,
                                                            T *__restrict__ y, int64_t ldy, int log_kparts) {
    constexpr int PARTS = RowType<T>::PARTS, CAP = NT * 8 / PARTS, GROUPS = G4_TILE / GROUP, U = 2;
    __shared__ float sums[WARPS][STRIP][NT * 8 + 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
    const ExpertSlot slot = expert_slot(offsets, experts, rows, CAP, blockIdx.y);
    if (slot.expert < 0) return;

    const int kparts = 1 << log_kparts, strips = WARPS >> log_kparts;
    const int part = warp & (kparts - 1), strip = warp >> log_kparts;
    const int j0 = (blockIdx.x * strips + strip) * STRIP;               // first feature of this warp
    float acc[NT][4] = {};
    if (j0 < w.n) {
        // column lane/4 of the B operand: row and part of x
        const T *xrow[NT];
        int xpart[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int col = t * 8 + g, r = slot.first + col / PARTS;
            xrow[t] = col / PARTS < CAP && r < slot.last ? x + (int64_t)r * ldx : nullptr;
            xpart[t] = col % PARTS;
        }
        const int64_t tile0 = ((int64_t)slot.expert * w.tiles_n + j0 / G4_TILE) * w.tiles_k;
        const int rr = j0 % G4_TILE + g;
        const uint4 *codes = reinterpret_cast<const uint4 *>(w.codes + tile0 * G4_TILE_WORDS) + c * G4_TILE + rr;
        const uint8_t *scales = w.scales + tile0 * (GROUPS * G4_TILE) + (GROUPS > 1 ? (c & (GROUPS - 1)) * G4_TILE : 0) + rr;
#pragma unroll 1
        for (int kt = part; kt < w.tiles_k; kt += U * kparts) {
            uint4 lo[U], hi[U];                                         // features g and g + 8: unit c of their 128 codes
            float slo[U], shi[U];                                       // their scales of group c
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = kt + u * kparts;
                if (at < w.tiles_k) {
                    lo[u] = __ldcs(codes + (int64_t)at * (G4_TILE_WORDS / 4));
                    hi[u] = __ldcs(codes + (int64_t)at * (G4_TILE_WORDS / 4) + 8);
                    slo[u] = __fmul_rn(g4_scale_f32(__ldg(scales + (int64_t)at * (GROUPS * G4_TILE))), CodeScale<T>::UNDO);
                    shi[u] = __fmul_rn(g4_scale_f32(__ldg(scales + (int64_t)at * (GROUPS * G4_TILE) + 8)), CodeScale<T>::UNDO);
                } else {
                    lo[u] = hi[u] = make_uint4(0u, 0u, 0u, 0u);
                    slo[u] = shi[u] = 0.0f;
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = kt + u * kparts;
                if (at >= w.tiles_k) break;
                float sum[NT][4];
#pragma unroll
                for (int ww = 0; ww < 4; ++ww) {
                    uint4 b[NT];
#pragma unroll
                    for (int t = 0; t < NT; ++t) b[t] = load_octet<T, VEC>(xrow[t], at * G4_TILE + ww * 32 + c * 8, w.k, xpart[t]);
                    if ((ww * 32) % GROUP == 0) {
#pragma unroll
                        for (int t = 0; t < NT; ++t) sum[t][0] = sum[t][1] = sum[t][2] = sum[t][3] = 0.0f;
                    }
                    const uint32_t wl = ww == 0 ? lo[u].x : ww == 1 ? lo[u].y : ww == 2 ? lo[u].z : lo[u].w;
                    const uint32_t wh = ww == 0 ? hi[u].x : ww == 1 ? hi[u].y : ww == 2 ? hi[u].z : hi[u].w;
                    const uint32_t l0 = code_pair<T>(wl, 0), l1 = code_pair<T>(wl, 1), l2 = code_pair<T>(wl, 2), l3 = code_pair<T>(wl, 3);
                    const uint32_t h0 = code_pair<T>(wh, 0), h1 = code_pair<T>(wh, 1), h2 = code_pair<T>(wh, 2), h3 = code_pair<T>(wh, 3);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        mma_16x8x16<T>(sum[t], l0, h0, l1, h1, b[t].x, b[t].y);
                        mma_16x8x16<T>(sum[t], l2, h2, l3, h3, b[t].z, b[t].w);
                    }
                    if ((ww * 32 + 32) % GROUP == 0) {
                        const int grp = ww * 32 / GROUP;                // quad lane `grp` holds that group's scales
                        const float s0 = GROUPS == 1 ? slo[u] : __shfl_sync(0xffffffffu, slo[u], grp, 4);
                        const float s1 = GROUPS == 1 ? shi[u] : __shfl_sync(0xffffffffu, shi[u], grp, 4);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            acc[t][0] = __fmaf_rn(s0, sum[t][0], acc[t][0]);
                            acc[t][1] = __fmaf_rn(s0, sum[t][1], acc[t][1]);
                            acc[t][2] = __fmaf_rn(s1, sum[t][2], acc[t][2]);
                            acc[t][3] = __fmaf_rn(s1, sum[t][3], acc[t][3]);
                        }
                    }
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        sums[warp][g][t * 8 + 2 * c] = acc[t][0];
        sums[warp][g][t * 8 + 2 * c + 1] = acc[t][1];
        sums[warp][g + 8][t * 8 + 2 * c] = acc[t][2];
        sums[warp][g + 8][t * 8 + 2 * c + 1] = acc[t][3];
    }
    __syncthreads();
    const float alpha = __ldg(w.alpha + slot.expert);
    const int feats = strips * STRIP, jbase = blockIdx.x * feats, have = slot.last - slot.first;
    for (int v = threadIdx.x; v < feats * have; v += WARPS * 32) {
        const int f = v % feats, r = v / feats, j = jbase + f;
        if (j >= w.n) continue;
        float total = 0.0f;
        for (int p = 0; p < kparts; ++p) {
            const float *s = sums[(f / STRIP) * kparts + p][f % STRIP] + r * PARTS;
            float one = s[PARTS - 1];                                   // smallest part first
#pragma unroll
            for (int q = PARTS - 2; q >= 0; --q) one = __fadd_rn(one, s[q]);
            total = __fadd_rn(total, one);
        }
        real_store(y + (int64_t)(slot.first + r) * ldy + j, __fmul_rn(total, alpha));
    }
}

template <class T, int NT, int GROUP>
int launch(const T *x, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, T *y, int64_t ldy, cudaStream_t st) {
    constexpr int CAP = NT * 8 / RowType<T>::PARTS;
    int log_kparts = 0;
    while (log_kparts < 3 && (2 << log_kparts) <= w.tiles_k) ++log_kparts;
    const int64_t slots = offsets ? expert_slots_most(rows, experts, CAP) : (rows + CAP - 1) / CAP;
    if (slots > 65535) return QNN_E_RANGE;
    const int feats = STRIP * (WARPS >> log_kparts);
    const dim3 grid((unsigned)((w.n + feats - 1) / feats), (unsigned)slots);
    const bool vec = qnn_aligned(x, 16) && (ldx * (int64_t)sizeof(T)) % 16 == 0;
    if (vec) g4_rows_kernel<T, NT, GROUP, true><<<grid, WARPS * 32, 0, st>>>(x, ldx, rows, offsets, experts, w, y, ldy, log_kparts);
    else g4_rows_kernel<T, NT, GROUP, false><<<grid, WARPS * 32, 0, st>>>(x, ldx, rows, offsets, experts, w, y, ldy, log_kparts);
    return qnn_launch_status();
}

template <class T, int NT>
int by_group(const T *x, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, T *y, int64_t ldy, cudaStream_t st) {
    if (w.group == 32) return launch<T, NT, 32>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    if (w.group == 64) return launch<T, NT, 64>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    return launch<T, NT, 128>(x, ldx, rows, offsets, experts, w, y, ldy, st);
}

// Columns per block: the fewest instructions' worth that hold the rows, at most 4 (32 columns).
template <class T>
int by_columns(const void *xv, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, void *yv, int64_t ldy,
               int rows_together, cudaStream_t st) {
    const T *x = static_cast<const T *>(xv);
    T *y = static_cast<T *>(yv);
    const int cols = rows_together * RowType<T>::PARTS;
    if (cols <= 8) return by_group<T, 1>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    if (cols <= 16) return by_group<T, 2>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    if (cols <= 24) return by_group<T, 3>(x, ldx, rows, offsets, experts, w, y, ldy, st);
    return by_group<T, 4>(x, ldx, rows, offsets, experts, w, y, ldy, st);
}

}  // namespace

int qnn_g4_rows(const void *x, int type, int64_t ldx, int rows, const int32_t *offsets, int experts, const G4Weights &w, void *y,
                int64_t ldy, int rows_together, cudaStream_t st) {
    if (type == QNN_F32) return by_columns<float>(x, ldx, rows, offsets, experts, w, y, ldy, rows_together, st);
    if (type == QNN_BF16) return by_columns<__nv_bfloat16>(x, ldx, rows, offsets, experts, w, y, ldy, rows_together, st);
    return by_columns<__half>(x, ldx, rows, offsets, experts, w, y, ldy, rows_together, st);
}
