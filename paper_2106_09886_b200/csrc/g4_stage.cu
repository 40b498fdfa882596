// Real operands rewritten for the tensor cores: rows of 2-byte elements whose start and stride are multiples of 16 bytes.
// Streaming; bound: HBM (reads the rows once, writes 2 bytes per element and part).  Needed for fp32 rows, which become
// three bf16 parts, and for rows that are not aligned.
#include "g4_stage.cuh"
#include "tc_ptx.cuh"

namespace {

struct StageJob {
    const void *src;
    int64_t ld;
    int width, octets;
    uint4 *dst;                                        // [parts][rows][octets]
    bool vec;                                          // fp32 rows can be read 16 bytes at a time
};

// A thread rewrites eight columns of a row; z picks one of two operands with the same rows.
template <class T>
__global__ void __launch_bounds__(256) stage_rows_kernel(StageJob first, StageJob second, int rows) {
    start_next();
    wait_for_previous();
    const StageJob &job = blockIdx.z ? second : first;
    const int o = blockIdx.x * 32 + threadIdx.x, i = o * 8;
    if (o >= job.octets) return;
    const int64_t part = (int64_t)rows * job.octets;
    for (int r = blockIdx.y * 8 + threadIdx.y; r < rows; r += gridDim.y * 8) {
        const T *s = static_cast<const T *>(job.src) + (int64_t)r * job.ld + i;
        uint4 *dst = job.dst + (int64_t)r * job.octets + o;
        if constexpr (sizeof(T) == 2) {
            uint16_t e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = i + j < job.width ? reinterpret_cast<const unsigned short *>(s)[j] : (uint16_t)0;
            *dst = make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
        } else {
            float f[8];
            if (job.vec && i + 8 <= job.width) {
                const float4 a = reinterpret_cast<const float4 *>(s)[0], b = reinterpret_cast<const float4 *>(s)[1];
                f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = i + j < job.width ? s[j] : 0.0f;
            }
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                uint32_t b[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) b[j] = split_part_bits(f[j], p);
                dst[p * part] = make_uint4(__byte_perm(b[0], b[1], 0x7632), __byte_perm(b[2], b[3], 0x7632), __byte_perm(b[4], b[5], 0x7632),
                                           __byte_perm(b[6], b[7], 0x7632));
            }
        }
    }
}

StageJob job_of(const void *src, int64_t ld, int width, void *dst) {
    return {src, ld, width, (width + 7) / 8, static_cast<uint4 *>(dst), qnn_aligned(src, 16) && ld % 4 == 0};
}

int stage(const StageJob &a, const StageJob &b, int jobs, int type, int rows, cudaStream_t st) {
    const int octets = jobs > 1 && b.octets > a.octets ? b.octets : a.octets, ys = (rows + 7) / 8;
    const dim3 grid((octets + 31) / 32, ys < 32768 ? ys : 32768, jobs), block(32, 8);
    if (type == QNN_F32) return launch_early(stage_rows_kernel<float>, grid, block, st, a, b, rows);
    return launch_early(stage_rows_kernel<uint16_t>, grid, block, st, a, b, rows);      // the two 2-byte types are copied as they are
}

}  // namespace

int qnn_stage_rows(const void *src, int type, int64_t ld, int rows, int width, void *dst, cudaStream_t st) {
    const StageJob a = job_of(src, ld, width, dst);
    return stage(a, a, 1, type, rows, st);
}
int qnn_stage_rows_two(const void *src_a, int64_t ld_a, int width_a, void *dst_a, const void *src_b, int64_t ld_b, int width_b, void *dst_b,
                       int type, int rows, cudaStream_t st) {
    return stage(job_of(src_a, ld_a, width_a, dst_a), job_of(src_b, ld_b, width_b, dst_b), 2, type, rows, st);
}
