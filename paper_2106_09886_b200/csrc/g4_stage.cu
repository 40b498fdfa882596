// Real operands rewritten for the tensor cores: rows of 2-byte elements whose start and stride are multiples of 16 bytes.
// Streaming; bound: HBM (reads the rows once, writes 2 bytes per element and part).  Needed for fp32 rows, which become
// three bf16 parts, and for rows that are not aligned.
#include "g4_stage.cuh"

namespace {

// Eight columns a thread.
template <class T>
__global__ void __launch_bounds__(256) stage_rows_kernel(const T *__restrict__ src, int64_t ld, int rows, int width, int octets,
                                                        uint16_t *__restrict__ dst, bool vec) {
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    const int64_t total = (int64_t)rows * octets;
    for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < total; v += (int64_t)gridDim.x * 256) {
        const int r = (int)(v / octets), o = (int)(v - (int64_t)r * octets), i = o * 8;
        const T *s = src + (int64_t)r * ld + i;
        if constexpr (PARTS == 1) {
            uint16_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = i + j < width ? __ldg(reinterpret_cast<const unsigned short *>(s) + j) : (uint16_t)0;
            reinterpret_cast<uint4 *>(dst)[v] = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16,
                                                           e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
        } else {
            float f[8];
            if (vec && i + 8 <= width) {
                const float4 a = __ldg(reinterpret_cast<const float4 *>(s)), b = __ldg(reinterpret_cast<const float4 *>(s) + 1);
                f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = i + j < width ? __ldg(s + j) : 0.0f;
            }
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                uint32_t b[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] = split_part_bits(f[j], p);
                reinterpret_cast<uint4 *>(dst)[p * total + v] =
                    make_uint4(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632), __byte_perm(b[4], b[5], 0x7632),
                               __byte_perm(b[6], b[7], 0x7632));
            }
        }
    }
}

}  // namespace

int qnn_stage_rows(const void *src, int type, int64_t ld, int rows, int width, void *dst, cudaStream_t st) {
    const int octets = (width + 7) / 8;
    const int64_t blocks = ((int64_t)rows * octets + 255) / 256;
    const int grid = (int)(blocks < 148 * 8 ? blocks : 148 * 8);
    uint16_t *d = static_cast<uint16_t *>(dst);
    if (type == QNN_F32) {
        const bool vec = qnn_aligned(src, 16) && ld % 4 == 0;
        stage_rows_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float *>(src), ld, rows, width, octets, d, vec);
    } else {                                              // the two 2-byte types are copied as they are
        stage_rows_kernel<uint16_t><<<grid, 256, 0, st>>>(static_cast<const uint16_t *>(src), ld, rows, width, octets, d, false);
    }
    return qnn_launch_status();
}
