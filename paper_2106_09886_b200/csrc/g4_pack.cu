// Packing real weights into group-scaled 4-bit codes (include/qnn.h, qnn_g4_pack_weights).  Offline: two passes over the
// weights, the largest magnitude of a matrix first, then scales and codes of one stored tile per thread block.
#include "g4_format.cuh"

namespace {

// Largest magnitude of a matrix into alpha[e] (as float bits, which order like integers for values >= 0; NaNs ignored).
template <class T>
__global__ void __launch_bounds__(256) g4_amax_kernel(const T *__restrict__ w, int n, int k, int64_t ldw, float *alpha) {
    const int e = blockIdx.y;
    float m = 0.0f;
    for (int64_t j = blockIdx.x; j < n; j += gridDim.x) {
        const T *row = w + ((int64_t)e * n + j) * ldw;
        for (int i = threadIdx.x; i < k; i += 256) m = fmaxf(m, fabsf(real_load(row + i)));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if ((threadIdx.x & 31) == 0) atomicMax(reinterpret_cast<int *>(alpha + e), __float_as_int(m));   // order-free
}

__global__ void g4_alpha_kernel(float *alpha, int experts) {
    const int e = blockIdx.x * 256 + threadIdx.x;
    if (e < experts) alpha[e] = __fdiv_rn(alpha[e], 15.0f * G4_SCALE_MAX);
}

__device__ __forceinline__ uint32_t g4_code(float x, float step) {
    if (!(step > 0.0f)) return 0u;
    const float v = __fdiv_rn(x, step);                       // NaN and -inf take the low end, +inf the high one
    const float c = fminf(fmaxf(v, -16.0f), 16.0f);
    const float u = __fmaf_rn(c, 0.5f, 8.0f);                 // code boundaries (even values of v) are integers of u
    const float t = c > 0.0f ? floorf(u) : ceilf(u) - 1.0f;
    return (uint32_t)fminf(fmaxf(t, 0.0f), 15.0f);
}

// One stored tile: thread r owns row r.  Offline, so rows are read straight (each thread walks its own row).
template <class T>
__global__ void __launch_bounds__(128) g4_pack_kernel(const T *__restrict__ w, int n, int k, int64_t ldw, int group, int tiles_n,
                                                     int tiles_k, uint32_t *codes, uint8_t *scales,
                                                     const float *__restrict__ alpha) {
    const int64_t tile = blockIdx.x;
    const int tk = (int)(tile % tiles_k);
    const int64_t rest = tile / tiles_k;
    const int tn = (int)(rest % tiles_n), e = (int)(rest / tiles_n);
    const int r = threadIdx.x, row = tn * G4_TILE + r;
    const float a = alpha[e];
    const T *src = w + ((int64_t)e * n + row) * ldw + tk * G4_TILE;
    const int cols = row < n ? min(G4_TILE, k - tk * G4_TILE) : 0;
    uint32_t *dst = codes + tile * G4_TILE_WORDS;
    const int groups = G4_TILE / group;
    for (int g = 0; g < groups; ++g) {
        float m = 0.0f;
        for (int i = g * group; i < min(cols, (g + 1) * group); ++i) m = fmaxf(m, fabsf(real_load(src + i)));
        const float s = a > 0.0f ? fminf(__fdiv_rn(m, __fmul_rn(15.0f, a)), G4_SCALE_MAX) : 0.0f;
        const uint8_t sb = (uint8_t)__nv_cvt_float_to_fp8(s, __NV_SATFINITE, __NV_E4M3);
        scales[(tile * groups + g) * G4_TILE + r] = sb;
        const float step = __fmul_rn(a, g4_scale_f32(sb));
        for (int o = g * group / 8; o < (g + 1) * group / 8; ++o) {      // octet o: word o / 4 of unit o % 4
            uint32_t word = 0u;
            for (int j = 0; j < 8; ++j) {
                const int i = o * 8 + j;
                const uint32_t t = i < cols ? g4_code(real_load(src + i), step) : 0u;
                word |= t << (4 * (j >> 1) + 16 * (j & 1));
            }
            dst[((o & 3) * G4_TILE + r) * 4 + (o >> 2)] = word;
        }
    }
}

template <class T>
int pack(const void *w, int experts, int n, int k, int64_t ldw, int group, uint32_t *codes, uint8_t *scales, float *alpha,
         cudaStream_t st) {
    const T *src = static_cast<const T *>(w);
    if (cudaMemsetAsync(alpha, 0, sizeof(float) * (size_t)experts, st) != cudaSuccess) return QNN_E_CUDA;
    g4_amax_kernel<T><<<dim3(n < 296 ? n : 296, experts), 256, 0, st>>>(src, n, k, ldw, alpha);
    g4_alpha_kernel<<<(experts + 255) / 256, 256, 0, st>>>(alpha, experts);
    const int tn = g4_tiles(n), tk = g4_tiles(k);
    g4_pack_kernel<T><<<(unsigned)((int64_t)experts * tn * tk), 128, 0, st>>>(src, n, k, ldw, group, tn, tk, codes, scales, alpha);
    return qnn_launch_status();
}

}  // namespace

extern "C" size_t qnn_g4_codes_bytes(int experts, int n, int k) {
    if (!g4_dims_ok(experts, n, k)) return 0;
    return (size_t)experts * g4_tiles(n) * g4_tiles(k) * G4_TILE_WORDS * 4u;
}

extern "C" size_t qnn_g4_scales_bytes(int experts, int n, int k, int group) {
    if (!g4_dims_ok(experts, n, k) || !g4_group_ok(group)) return 0;
    return (size_t)experts * g4_tiles(n) * g4_tiles(k) * (G4_TILE / group) * G4_TILE;
}

extern "C" int qnn_g4_pack_weights(const void *w, int type, int experts, int n, int k, int64_t ldw, int group, uint32_t *codes,
                                   uint8_t *scales, float *alpha, void *stream) {
    if (!w || !codes || !scales || !alpha || !g4_type_ok(type) || !g4_dims_ok(experts, n, k) || !g4_group_ok(group) || ldw < k)
        return QNN_E_ARG;
    if (!qnn_aligned(w, g4_type_bytes(type)) || !qnn_aligned(codes, 16) || !qnn_aligned(scales, 16) || !qnn_aligned(alpha, 4))
        return QNN_E_ALIGN;
    if ((int64_t)experts * g4_tiles(n) * g4_tiles(k) > 0x7FFFFFFFll) return QNN_E_RANGE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (type == QNN_F32) return pack<float>(w, experts, n, k, ldw, group, codes, scales, alpha, st);
    if (type == QNN_BF16) return pack<__nv_bfloat16>(w, experts, n, k, ldw, group, codes, scales, alpha, st);
    return pack<__half>(w, experts, n, k, ldw, group, codes, scales, alpha, st);
}
