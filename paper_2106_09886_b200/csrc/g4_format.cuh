// Group-scaled 4-bit weights: the storage of include/qnn.h, argument checks and the row ranges of the experts, shared
// by every translation unit that reads them.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include "qnn_internal.cuh"

constexpr int G4_TILE = 128;                       // rows and columns of a stored tile
constexpr int G4_TILE_WORDS = 128 * 128 / 8;       // its codes: 8 KB
constexpr float G4_SCALE_MAX = 448.0f;             // largest 1-4-3 float
constexpr int G4_MAX_DIM = 65535 * 16;
constexpr int G4_MAX_EXPERTS = 4096;               // blocks of rows stay countable in 31 bits whatever the offsets hold
constexpr int64_t G4_MAX_ROWS = (1ll << 31) / 256; // row tiles stay far inside 32-bit tile arithmetic

struct G4Weights {
    const uint32_t *codes;
    const uint8_t *scales;
    const float *alpha;
    int n, k, group;
    int tiles_n, tiles_k;
};

static inline bool g4_type_ok(int t) { return t == QNN_F32 || t == QNN_BF16 || t == QNN_F16; }
static inline int g4_type_bytes(int t) { return t == QNN_F32 ? 4 : 2; }
static inline bool g4_dims_ok(int experts, int n, int k) {
    return experts >= 1 && experts <= G4_MAX_EXPERTS && n >= 1 && n <= G4_MAX_DIM && k >= 1 && k <= G4_MAX_DIM;
}
static inline bool g4_group_ok(int g) { return g == 32 || g == 64 || g == 128; }
static inline int g4_tiles(int v) { return (v + G4_TILE - 1) / G4_TILE; }

// 1-4-3 float -> fp32 (exact).
__device__ __forceinline__ float g4_scale_f32(uint8_t b) {
    __nv_fp8_e4m3 v;
    v.__x = b;
    return (float)v;
}

// Rows [first, last) of expert e; empty where offsets decrease, clamped to the rows that exist.  offsets NULL = one matrix
// that owns every row.
__device__ __forceinline__ void expert_rows(const int32_t *offsets, int e, int rows, int &first, int &last) {
    if (!offsets) {
        first = 0;
        last = rows;
        return;
    }
    first = min(max(offsets[e], 0), rows);
    last = min(max(offsets[e + 1], 0), rows);
}

// The slot-th block of `tile` rows, blocks counted expert by expert: its expert and rows, or expert -1 past the last.
// Called by whole warps; every lane gets the answer.  offsets NULL = one matrix that owns every row.
struct ExpertSlot {
    int expert, first, last;
};
__device__ __forceinline__ ExpertSlot expert_slot(const int32_t *offsets, int experts, int rows, int tile, int slot) {
    if (!offsets) {
        const int first = slot * tile;
        if (first >= rows) return {-1, 0, 0};
        return {0, first, min(rows, first + tile)};
    }
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int base = 0; base < experts; base += 32) {
        int a = 0, b = 0;
        if (base + lane < experts) expert_rows(offsets, base + lane, rows, a, b);
        const int mine = b > a ? (b - a + tile - 1) / tile : 0;
        int incl = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += o;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, slot < before + incl);
        if (hit) {
            const int src = __ffs(hit) - 1;
            const int e_first = __shfl_sync(0xffffffffu, a, src), e_last = __shfl_sync(0xffffffffu, b, src);
            const int in = slot - before - __shfl_sync(0xffffffffu, incl - mine, src);
            const int first = e_first + in * tile;
            return {base + src, first, min(e_last, first + tile)};
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
    }
    return {-1, 0, 0};
}

// Most blocks of `tile` rows that `rows` rows of `experts` experts can make: an expert's last block may hold one row.
static inline int64_t expert_slots_most(int64_t rows, int experts, int tile) {
    const int64_t some = rows < experts ? rows : experts;
    return (rows + some * (tile - 1)) / tile;
}

// Sums are kept in units of alpha * undo, undo a power of two that keeps one product of a row's element and a weight below
// the element itself (|scale * q| <= 6720): a sum overflows only where the result, or one of its parts, is within a factor
// alpha * undo of doing so, or past it.  The two factors below give sum * undo * alpha with one rounding and without leaving
// fp32 on the way: undo goes with a small alpha first, and last behind a large one.
struct SumScale {
    float first, second;
    __device__ __forceinline__ SumScale(float alpha, float undo) : first(alpha < 1.0f ? alpha * undo : alpha), second(alpha < 1.0f ? 1.0f : undo) {}
    __device__ __forceinline__ float of(float sum) const { return sum * first * second; }
};

// Element loads and stores of the real operands.
__device__ __forceinline__ float real_load(const float *p) { return *p; }
__device__ __forceinline__ float real_load(const __nv_bfloat16 *p) { return __bfloat162float(*p); }
__device__ __forceinline__ float real_load(const __half *p) { return __half2float(*p); }
__device__ __forceinline__ void real_store(float *p, float v) { *p = v; }
__device__ __forceinline__ void real_store(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void real_store(__half *p, float v) { *p = __float2half_rn(v); }
