// Rows of real numbers: the residual's addition and the root-mean-square norm, with the result as real numbers, in 8 bits with a
// scale for each row, or both; rows into 8 bits without a norm, and back; the norm's backward products.
//
//   h = round(x + residual)     rstd = 1 / sqrt(mean(h^2) + eps)     y = (h * gain) * rstd
//   scale = max|y| / 127        code = rint(y / scale)
//
// Bound: HBM.  A row is read once and stays in registers.  The order (h * gain) * rstd makes max|y| = max|h * gain| * rstd exactly,
// rounding being monotone: the sum of squares and the largest magnitude come out of one pass and one reduction, and the codes follow
// from the registers by a few multiplications and fused multiply-adds each, without a branch (RowScale): a sum with 1.5 * 2^23 holds
// the nearest whole number in its low byte.
// 16384 x 4096 bf16 with a residual take 73 us (470 MB, some of the writes still in L2 at the end), the quantiser of as many 44, decoding 32.
// With a conversion, a clamp and a comparison for each code the norm took 125; with codes by two bounds of the product, and those that
// the bounds leave open by division out of line, 91; with the product alone, whose codes are not always the quotient's, 72.
#include "real_rows.cuh"
#include "tc_ptx.cuh"

namespace {

constexpr int NORM_MAX_WIDTH = 32768, CODES_MAX_WIDTH = 131072;

struct NormParams {
    const void *x, *residual, *gain;          // residual NULL: h is x.  gain NULL: no norm (y = x)
    int64_t ldx, ldr, ldh, ldy, ldc;
    int64_t rows;
    int width;
    float eps;
    void *h, *y;
    int8_t *codes;
    float *scales, *rstd;
};

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
// Of magnitudes: their bits are in the numbers' order, NaN's beyond infinity's.
__device__ __forceinline__ float warp_max(float v) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v))); }

// Over the threads of a row: blockDim.x of them, whole warps.  With two sums a thread, of packs blockDim.x apart, the warps' are added as if
// each pack had a thread of its own, so that a row's bits do not depend on which form its call takes: the warp's lower lanes end up
// with its first sum and the upper ones with its second, as warp_sum has them.
template <bool SUM, int SUMS> __device__ __forceinline__ void block_sum_and_max(float (&sums)[SUMS], float &most, float (*parts)[32]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    float sum = sums[0];
    if constexpr (SUM && SUMS == 2) {
        const float other = __shfl_xor_sync(0xffffffffu, lane < 16 ? sums[1] : sums[0], 16);
        sum = __fadd_rn(lane < 16 ? sums[0] : sums[1], other);
#pragma unroll
        for (int d = 8; d; d >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, d));
    } else if constexpr (SUM) {
        sum = warp_sum(sum);
    }
    most = warp_max(most);
    if (blockDim.x > 32) {
        if (SUMS == 2 ? (lane & 15) == 0 : lane == 0) parts[0][(lane >> 4) * warps + warp] = sum;
        if (lane == 0) parts[1][warp] = most;
        __syncthreads();
        if constexpr (SUM) sum = warp_sum(lane < SUMS * warps ? parts[0][lane] : 0.0f);
        most = warp_max(lane < warps ? parts[1][lane] : 0.0f);
    } else if constexpr (SUM && SUMS == 2) {
        sum = __fadd_rn(sum, __shfl_xor_sync(0xffffffffu, sum, 16));
    }
    sums[0] = sum;
}
__device__ __forceinline__ float norm_factor(float sum, const NormParams &p) {
    return __frcp_rn(__fsqrt_rn(__fadd_rn(__fdiv_rn(sum, (float)p.width), p.eps)));
}

__device__ __forceinline__ uint32_t add_pair(uint32_t a, uint32_t b, __nv_bfloat16) {
    const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t add_pair(uint32_t a, uint32_t b, __half) {
    const __half2 v = __hadd2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t add_pair(uint32_t a, uint32_t b, float) { return __float_as_uint(__fadd_rn(__uint_as_float(a), __uint_as_float(b))); }
template <class T> __device__ __forceinline__ uint4 add_pack(uint4 a, uint4 b) {
    return make_uint4(add_pair(a.x, b.x, T()), add_pair(a.y, b.y, T()), add_pair(a.z, b.z, T()), add_pair(a.w, b.w, T()));
}

// A row by `blockDim.x` threads (y: rows of a block, more than one for rows of a single warp).  Each thread holds NV packs of 16
// bytes, as products with the gain.  NORM = false: codes of the rows themselves.
template <class T, class G, int NV, bool NORM>
__global__ void __launch_bounds__(NV == 1 ? 1024 : 512, NV == 2 ? 3 : 1) norm_rows_kernel(const NormParams p) {
    __shared__ float parts[2][32];
    start_next();
    wait_for_previous();
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;                                      // (whole warps: blocks of several rows have one warp a row)
    typedef Octets<T> O;
    constexpr int V = O::V;
    const int packs = p.width / V, step = blockDim.x;
    const uint4 *x = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.x) + row * p.ldx);
    uint4 h[NV], r[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = threadIdx.x + j * step;
        h[j] = i < packs ? x[i] : make_uint4(0, 0, 0, 0);
    }
    if (NORM && p.residual) {
        const uint4 *res = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.residual) + row * p.ldr);
        uint4 *out = reinterpret_cast<uint4 *>(static_cast<T *>(p.h) + row * p.ldh);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = threadIdx.x + j * step;
            r[j] = i < packs ? res[i] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = threadIdx.x + j * step;
            h[j] = add_pack<T>(h[j], r[j]);
            if (i < packs) out[i] = h[j];
        }
    }
    constexpr int SUMS = NV == 2 ? 2 : 1;                           // (NV is 1 or 2 by the number of rows)
    float v[NV][V], sums[SUMS] = {}, most = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        float &sum = sums[j % SUMS];
        O::get(h[j], v[j]);
        if constexpr (NORM) {
            float g[V];
            gain_of_pack<T, G>(p.gain, min((int)threadIdx.x + j * step, packs - 1), g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sum = __fmaf_rn(v[j][e], v[j][e], sum);
                v[j][e] = __fmul_rn(v[j][e], g[e]);
            }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) most = max_or_nan(most, fabsf(v[j][e]));
    }
    block_sum_and_max<NORM>(sums, most, parts);
    float rstd = 1.0f;
    if constexpr (NORM) {
        rstd = norm_factor(sums[0], p);
        if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
        most = __fmul_rn(most, rstd);
        if (p.y) {
            uint4 *y = reinterpret_cast<uint4 *>(static_cast<T *>(p.y) + row * p.ldy);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int i = threadIdx.x + j * step;
                float o[V];
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] = __fmul_rn(v[j][e], rstd);
                if (i < packs) y[i] = O::put(o);
            }
        }
    }
    if (!NORM || p.codes) {
        const RowScale s(most);
        if (threadIdx.x == 0) p.scales[row] = s.scale;
        uint32_t *codes = reinterpret_cast<uint32_t *>(p.codes + row * p.ldc);
        auto encode = [&](auto raised) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int i = threadIdx.x + j * step;
                uint32_t c[V];
#pragma unroll
                for (int e = 0; e < V; ++e) c[e] = s.code<raised>(NORM ? __fmul_rn(v[j][e], rstd) : v[j][e]);
                if (i < packs) {
                    if constexpr (V == 8)
                        reinterpret_cast<uint2 *>(codes)[i] = make_uint2(s.word(c[0], c[1], c[2], c[3]), s.word(c[4], c[5], c[6], c[7]));
                    else
                        codes[i] = s.word(c[0], c[1], c[2], c[3]);
                }
            }
        };
        if (s.is_raised()) encode(std::true_type());
        else encode(std::false_type());
    }
}

// Rows whose start, stride or width is not a multiple of 16 bytes: element by element, NE of them a thread, `blockDim.x` apart, so that
// a warp's accesses lie together whatever the row's alignment.
template <class T, class G, int NE, bool NORM>
__global__ void __launch_bounds__(512, NE <= 16 ? 2 : 1) norm_elements_kernel(const NormParams p) {
    __shared__ float parts[2][32];
    start_next();
    wait_for_previous();
    const int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= p.rows) return;                                      // (whole warps: blocks of several rows have one warp a row)
    const int step = blockDim.x, width = p.width, first = threadIdx.x;
    const T *x = static_cast<const T *>(p.x) + row * p.ldx + first;
    const G *gain = static_cast<const G *>(p.gain) + first;
    T h[NE], r[NE];
    float v[NE], sums[1] = {}, most = 0.0f;
    float &sum = sums[0];
#pragma unroll
    for (int j = 0; j < NE; ++j) h[j] = first + j * step < width ? x[j * step] : from_f32<T>(0.0f);
    if (NORM && p.residual) {
        const T *res = static_cast<const T *>(p.residual) + row * p.ldr + first;
        T *out = static_cast<T *>(p.h) + row * p.ldh + first;
#pragma unroll
        for (int j = 0; j < NE; ++j) r[j] = first + j * step < width ? res[j * step] : from_f32<T>(0.0f);
#pragma unroll
        for (int j = 0; j < NE; ++j) {
            h[j] = from_f32<T>(__fadd_rn(to_f32(h[j]), to_f32(r[j])));
            if (first + j * step < width) out[j * step] = h[j];
        }
    }
#pragma unroll
    for (int j = 0; j < NE; ++j) {
        v[j] = to_f32(h[j]);
        if constexpr (NORM) {
            sum = __fmaf_rn(v[j], v[j], sum);
            v[j] = first + j * step < width ? __fmul_rn(v[j], to_f32(gain[j * step])) : 0.0f;
        }
        most = max_or_nan(most, fabsf(v[j]));
    }
    block_sum_and_max<NORM>(sums, most, parts);
    float rstd = 1.0f;
    if constexpr (NORM) {
        rstd = norm_factor(sum, p);
        if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
        most = __fmul_rn(most, rstd);
        if (p.y) {
            T *y = static_cast<T *>(p.y) + row * p.ldy + first;
#pragma unroll
            for (int j = 0; j < NE; ++j)
                if (first + j * step < width) y[j * step] = from_f32<T>(__fmul_rn(v[j], rstd));
        }
    }
    if (!NORM || p.codes) {
        const RowScale s(most);
        if (threadIdx.x == 0) p.scales[row] = s.scale;
        int8_t *codes = p.codes + row * p.ldc + first;
        auto encode = [&](auto raised) {
#pragma unroll
            for (int j = 0; j < NE; ++j) {
                const uint32_t c = s.code<raised>(NORM ? __fmul_rn(v[j], rstd) : v[j]);
                if (first + j * step < width) codes[j * step] = (int8_t)(s.inverse != 0.0f ? c : 0u);
            }
        };
        if (s.is_raised()) encode(std::true_type());
        else encode(std::false_type());
    }
}

// Rows that do not fit the registers of a block: element by element, read again (from the caches) for the results.
template <class T, class G, bool NORM>
__global__ void __launch_bounds__(1024) norm_wide_kernel(const NormParams p) {
    __shared__ float parts[2][32];
    start_next();
    wait_for_previous();
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + row * p.ldx;
    const G *gain = static_cast<const G *>(p.gain);
    float sums[1] = {}, most = 0.0f;
    float &sum = sums[0];
    if (NORM && p.residual) {
        const T *res = static_cast<const T *>(p.residual) + row * p.ldr;
        T *h = static_cast<T *>(p.h) + row * p.ldh;
#pragma unroll 8
        for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
            const T v = from_f32<T>(__fadd_rn(to_f32(x[i]), to_f32(res[i])));
            const float a = to_f32(v);
            h[i] = v;
            sum = __fmaf_rn(a, a, sum);
            most = max_or_nan(most, fabsf(__fmul_rn(a, to_f32(gain[i]))));
        }
        x = h;                                                      // (each thread reads what it has written itself)
    } else {
#pragma unroll 8
        for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
            float a = to_f32(x[i]);
            if constexpr (NORM) {
                sum = __fmaf_rn(a, a, sum);
                a = __fmul_rn(a, to_f32(gain[i]));
            }
            most = max_or_nan(most, fabsf(a));
        }
    }
    block_sum_and_max<NORM>(sums, most, parts);
    float rstd = 1.0f;
    if constexpr (NORM) {
        rstd = norm_factor(sum, p);
        if (p.rstd && threadIdx.x == 0) p.rstd[row] = rstd;
        most = __fmul_rn(most, rstd);
    }
    const bool coded = !NORM || p.codes;
    const RowScale s(most);
    if (coded && threadIdx.x == 0) p.scales[row] = s.scale;
    int8_t *codes = p.codes + row * p.ldc;
    T *y = static_cast<T *>(p.y) + row * p.ldy;
#pragma unroll 8
    for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
        float a = to_f32(x[i]);
        if constexpr (NORM) a = __fmul_rn(__fmul_rn(a, to_f32(gain[i])), rstd);
        if (NORM && p.y) y[i] = from_f32<T>(a);
        if (coded) codes[i] = (int8_t)(s.inverse != 0.0f ? s.code<true>(a) : 0u);
    }
}

static inline int whole_warps(int threads) { return (threads + 31) / 32 * 32; }
template <class T, class G, int NV, bool NORM>
int norm_launch(const NormParams &p, int packs, cudaStream_t st) {
    const int threads = whole_warps((packs + NV - 1) / NV), together = threads == 32 ? 4 : 1;
    const int64_t blocks = (p.rows + together - 1) / together;
    return launch_early(norm_rows_kernel<T, G, NV, NORM>, dim3((unsigned)blocks), dim3(threads, together), st, p);
}
template <class T, class G, int NE, bool NORM>
int norm_elements_launch(const NormParams &p, cudaStream_t st) {
    const int threads = whole_warps((p.width + NE - 1) / NE), together = threads == 32 ? 4 : 1;
    return launch_early(norm_elements_kernel<T, G, NE, NORM>, dim3((unsigned)((p.rows + together - 1) / together)), dim3(threads, together), st, p);
}
template <class T, class G, bool NORM>
int norm_typed(const NormParams &p, bool vec, cudaStream_t st) {
    if (!vec) {
        if (p.width <= 4096) return norm_elements_launch<T, G, 8, NORM>(p, st);
        if (p.width <= 8192) return norm_elements_launch<T, G, 16, NORM>(p, st);
        if (p.width <= 16384) return norm_elements_launch<T, G, 32, NORM>(p, st);
        return launch_early(norm_wide_kernel<T, G, NORM>, dim3((unsigned)p.rows), dim3(1024), st, p);
    }
    const int packs = p.width / (16 / (int)sizeof(T));
    if (packs > 4096) return launch_early(norm_wide_kernel<T, G, NORM>, dim3((unsigned)p.rows), dim3(1024), st, p);
    if (packs <= 1024 && (p.rows <= 296 || packs <= 32)) return norm_launch<T, G, 1, NORM>(p, packs, st);
    if (packs <= 1024) return norm_launch<T, G, 2, NORM>(p, packs, st);
    if (packs <= 2048) return norm_launch<T, G, 4, NORM>(p, packs, st);
    return norm_launch<T, G, 8, NORM>(p, packs, st);
}

int check_real(const void *p, int type, int64_t ld, int width) {
    if (!p || ld < width) return QNN_E_ARG;
    return qnn_aligned(p, g4_type_bytes(type)) ? QNN_OK : QNN_E_ALIGN;
}
int check_codes(const int8_t *codes, const float *scales, int64_t ldc, int width) {
    if (!codes || !scales || ldc < width) return QNN_E_ARG;
    return qnn_aligned(codes, 16) && ldc % 16 == 0 && qnn_aligned(scales, 4) ? QNN_OK : QNN_E_ALIGN;
}
// Can rows be accessed 16 bytes at a time?
bool in_packs(const void *p, int type, int64_t ld) { return qnn_aligned(p, 16) && ld * g4_type_bytes(type) % 16 == 0; }

// ------------------------------------------------------------------------------------------------ codes back to numbers

// A byte as a number: xor 128 makes it 0 .. 255, which the mantissa of 2^23 takes as it is.
__device__ __forceinline__ float byte_value(uint32_t word, int i) {
    return __fadd_rn(__uint_as_float(__byte_perm(word ^ 0x80808080u, 0x4B000000u, 0x7540 + i)), -8388736.0f);      // 2^23 + 128
}
// The codes of one 16-byte pack of results in each of ROWS rows by a thread, all loaded first.  (A pack a thread: with two, a warp's
// stores cover half sectors, and 16384 x 4096 take 43 us instead of 31.)
template <class T, int ROWS>
__global__ void __launch_bounds__(256) decode_kernel(const int8_t *codes, const float *scales, int64_t rows, int width, int64_t ldc, T *out, int64_t ldo) {
    start_next();
    wait_for_previous();
    typedef Octets<T> O;
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i * O::V >= width) return;
    for (int64_t row = (int64_t)blockIdx.y * ROWS; row < rows; row += (int64_t)gridDim.y * ROWS) {
        uint32_t c[ROWS][O::V / 4];
        float s[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t at = row + r < rows ? row + r : rows - 1;
            const uint32_t *src = reinterpret_cast<const uint32_t *>(codes + at * ldc);
            if constexpr (O::V == 8) {
                const uint2 w = reinterpret_cast<const uint2 *>(src)[i];
                c[r][0] = w.x;
                c[r][1] = w.y;
            } else {
                c[r][0] = src[i];
            }
            s[r] = scales[at];
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row + r >= rows) break;
            float f[O::V];
#pragma unroll
            for (int e = 0; e < O::V; ++e) f[e] = __fmul_rn(byte_value(c[r][e / 4], e % 4), s[r]);
            reinterpret_cast<uint4 *>(out + (row + r) * ldo)[i] = O::put(f);
        }
    }
}
template <class T>
__global__ void __launch_bounds__(256) decode_any_kernel(const int8_t *codes, const float *scales, int64_t rows, int width, int64_t ldc, T *out, int64_t ldo) {
    start_next();
    wait_for_previous();
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const float s = scales[row];
#pragma unroll 4
        for (int i = blockIdx.x * 256 + threadIdx.x; i < width; i += gridDim.x * 256) out[row * ldo + i] = from_f32<T>(__fmul_rn((float)codes[row * ldc + i], s));
    }
}
template <class T>
int decode(const int8_t *codes, const float *scales, int64_t rows, int width, int64_t ldc, void *out, int64_t ldo, bool vec, cudaStream_t st) {
    T *o = static_cast<T *>(out);
    if (!vec) {
        const unsigned ys = (unsigned)(rows < 65535 ? rows : 65535);
        return launch_early(decode_any_kernel<T>, dim3((width + 1023) / 1024, ys), dim3(256), st, codes, scales, rows, width, ldc, o, ldo);
    }
    const int packs = width / Octets<T>::V, threads = packs < 256 ? (packs + 31) / 32 * 32 : 256;
    const unsigned xs = (unsigned)((packs + threads - 1) / threads);
    if (rows < 4 * 148) return launch_early(decode_kernel<T, 1>, dim3(xs, (unsigned)rows), dim3(threads), st, codes, scales, rows, width, ldc, o, ldo);
    const int64_t ys = (rows + 3) / 4;
    return launch_early(decode_kernel<T, 4>, dim3(xs, (unsigned)(ys < 65535 ? ys : 65535)), dim3(threads), st, codes, scales, rows, width, ldc, o, ldo);
}

// ------------------------------------------------------------------------------------------------ backward products

// dx = rstd * a - h * rstd^3 * mean(a * h) + dh with a = dy * gain; dgain = sum over the rows of dy * h * rstd.
// A block takes every gridDim.x-th row and keeps dgain of its columns in registers; the blocks' sums are added in a fixed order
// by a second kernel, so results repeat bit for bit.  Bound: HBM (8192 x 4096 bf16 with dh 50 us, 5.4 TB/s, 4 of them the second
// kernel; loads into registers, two rows of an SM at a time, took 81).
struct NormBackParams {
    const void *dy, *h, *gain, *dh;           // dh NULL: no gradient reaches h by another way
    const float *rstd;
    int64_t lddy, ldh, lddh, lddx, rows;
    int width;
    void *dx;
    float *sums;                              // [gridDim.x][width]
    unsigned int *err;
    unsigned int wait_limit;
};

// What a pack of a row adds to the row's sum, and its u = h * rstd.
template <class T> struct BackPack {
    static constexpr int V = Octets<T>::V;
    float dy[V], u[V];
    __device__ __forceinline__ void get(const uint4 &d, const uint4 &h, float r) {
        Octets<T>::get(d, dy);
        Octets<T>::get(h, u);
#pragma unroll
        for (int e = 0; e < V; ++e) u[e] = __fmul_rn(u[e], r);
    }
    __device__ __forceinline__ void add(const float (&g)[V], float &dot, float (&sum)[V]) const {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            dot = __fmaf_rn(__fmul_rn(dy[e], g[e]), u[e], dot);
            sum[e] = __fmaf_rn(dy[e], u[e], sum[e]);
        }
    }
    __device__ __forceinline__ uint4 result(const float (&g)[V], float mean, float r, const uint4 &other) const {
        float o[V], dh[V];
        Octets<T>::get(other, dh);                              // (zeros where there is none)
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = __fadd_rn(__fmul_rn(__fmaf_rn(-u[e], mean, __fmul_rn(dy[e], g[e])), r), dh[e]);
        return Octets<T>::put(o);
    }
};

// Rows of up to 32 * NV packs, a warp each: no barrier but the last, which adds the warps' sums of the gain in order.  A row stays in its
// own type and is unpacked twice; with four packs a lane the gain is read again (from L1) for each row, so that all fits the registers.
constexpr int BACK_WARPS = 8;
template <class T, class G, int NV>
__global__ void __launch_bounds__(BACK_WARPS * 32, 2) norm_back_warps_kernel(const NormBackParams p) {
    extern __shared__ float all[];                              // [BACK_WARPS][32 * NV * V]
    start_next();
    wait_for_previous();
    constexpr int V = Octets<T>::V, WIDE = 32 * NV * V;
    const int packs = p.width / V, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    float kept[NV > 2 ? 1 : NV][V], sum[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        if constexpr (NV <= 2) gain_of_pack<T, G>(p.gain, min(lane + 32 * j, packs - 1), kept[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[j][e] = 0.0f;
    }
    auto gain = [&](int j, float (&g)[V]) {
        if constexpr (NV <= 2) {
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = kept[j][e];
        } else {
            gain_of_pack<T, G>(p.gain, min(lane + 32 * j, packs - 1), g);
        }
    };
    for (int64_t row = (int64_t)blockIdx.x * BACK_WARPS + warp; row < p.rows; row += (int64_t)gridDim.x * BACK_WARPS) {
        const uint4 *dys = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.dy) + row * p.lddy);
        const uint4 *hs = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.h) + row * p.ldh);
        const uint4 *dhs = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.dh) + row * p.lddh);
        uint4 *dxs = reinterpret_cast<uint4 *>(static_cast<T *>(p.dx) + row * p.lddx);
        const float r = p.rstd[row];
        uint4 dy[NV], h[NV], dh[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = lane + 32 * j;
            dy[j] = i < packs ? dys[i] : zero;
            h[j] = i < packs ? hs[i] : zero;
            dh[j] = p.dh && i < packs ? dhs[i] : zero;
        }
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            BackPack<T> b;
            float g[V];
            b.get(dy[j], h[j], r);
            gain(j, g);
            b.add(g, dot, sum[j]);
        }
        const float mean = __fdiv_rn(warp_sum(dot), (float)p.width);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            BackPack<T> b;
            float g[V];
            b.get(dy[j], h[j], r);
            gain(j, g);
            const uint4 out = b.result(g, mean, r, dh[j]);
            if (lane + 32 * j < packs) dxs[lane + 32 * j] = out;
        }
    }
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) all[warp * WIDE + (lane + 32 * j) * V + e] = sum[j][e];
    __syncthreads();
    for (int c = threadIdx.x; c < p.width; c += BACK_WARPS * 32) {
        float s = all[c];
#pragma unroll
        for (int w = 1; w < BACK_WARPS; ++w) s = __fadd_rn(s, all[w * WIDE + c]);
        p.sums[(int64_t)blockIdx.x * p.width + c] = s;
    }
}

// Wider rows, a block each, NV packs a thread.  Rows come through a ring in shared memory by bulk copies, issued as soon as a stage
// has been read, so that the next rows are under way while one is summed over the block's barrier.
template <class T, class G, int NV>
__global__ void __launch_bounds__(512) norm_back_kernel(const NormBackParams p, int stages, int stage_bytes) {
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ float parts[2][16];
    __shared__ uint64_t full[8];
    __shared__ uint32_t abort_word;
    constexpr int V = Octets<T>::V;
    const int packs = p.width / V, step = blockDim.x, row_bytes = p.width * (int)sizeof(T);
    volatile uint32_t *abort_flag = &abort_word;
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) mbar_init(&full[s], 1);
        *abort_flag = 0;
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    start_next();
    wait_for_previous();
    auto load = [&](int64_t row, int s) {                       // by one thread
        uint8_t *dst = ring + s * stage_bytes;
        mbar_expect_tx(&full[s], (p.dh ? 3 : 2) * row_bytes);
        bulk_load(dst, static_cast<const T *>(p.dy) + row * p.lddy, row_bytes, &full[s]);
        bulk_load(dst + row_bytes, static_cast<const T *>(p.h) + row * p.ldh, row_bytes, &full[s]);
        if (p.dh) bulk_load(dst + 2 * row_bytes, static_cast<const T *>(p.dh) + row * p.lddh, row_bytes, &full[s]);
    };
    if (threadIdx.x == 0)
        for (int s = 0; s < stages && blockIdx.x + (int64_t)s * gridDim.x < p.rows; ++s) load(blockIdx.x + (int64_t)s * gridDim.x, s);
    const uint4 zero = make_uint4(0, 0, 0, 0);
    float g[NV][V], sum[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        gain_of_pack<T, G>(p.gain, min((int)threadIdx.x + j * step, packs - 1), g[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[j][e] = 0.0f;
    }
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    Ring at;
    int side = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, side ^= 1) {
        const float r = p.rstd[row];
        bool ok = short_wait(&full[at.s], at.ph, abort_flag, 1, p.err, p.wait_limit);
        const uint32_t src = smem_u32(ring) + at.s * stage_bytes;
        uint4 dh[NV];
        BackPack<T> b[NV];
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = threadIdx.x + j * step;
            const bool in = i < packs;
            b[j].get(in ? lds_128(src + i * 16) : zero, in ? lds_128(src + row_bytes + i * 16) : zero, r);
            dh[j] = in && p.dh ? lds_128(src + 2 * row_bytes + i * 16) : zero;
            b[j].add(g[j], dot, sum[j]);
        }
        dot = warp_sum(dot);
        if (lane == 0) parts[side][warp] = dot;                 // (two sides: the next row's sums do not wait for this one's readers)
        if (!__syncthreads_and(ok)) break;                      // all leave together; the copies in flight have been waited for or ...
        if (threadIdx.x == 0 && row + (int64_t)stages * gridDim.x < p.rows) load(row + (int64_t)stages * gridDim.x, at.s);
        at.next(stages);
        const float mean = __fdiv_rn(warp_sum(lane < warps ? parts[side][lane] : 0.0f), (float)p.width);
        uint4 *dxs = reinterpret_cast<uint4 *>(static_cast<T *>(p.dx) + row * p.lddx);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int i = threadIdx.x + j * step;
            if (i < packs) dxs[i] = b[j].result(g[j], mean, r, dh[j]);
        }
    }
    // ... get some time to land
    if (*abort_flag)
#pragma unroll 1
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int i = threadIdx.x + j * step;
        if (i < packs)
#pragma unroll
            for (int e = 0; e < V; ++e) p.sums[(int64_t)blockIdx.x * p.width + i * V + e] = sum[j][e];
    }
}

// The same for narrow rows that cannot be accessed in packs: NE elements a lane, 32 apart.
template <class T, class G, int NE>
__global__ void __launch_bounds__(BACK_WARPS * 32, 2) norm_back_warp_elements_kernel(const NormBackParams p) {
    __shared__ float all[BACK_WARPS][32 * NE];
    start_next();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, width = p.width;
    const G *gain = static_cast<const G *>(p.gain) + lane;
    float g[NE], sum[NE];
#pragma unroll
    for (int j = 0; j < NE; ++j) {
        g[j] = lane + 32 * j < width ? to_f32(gain[32 * j]) : 0.0f;
        sum[j] = 0.0f;
    }
    for (int64_t row = (int64_t)blockIdx.x * BACK_WARPS + warp; row < p.rows; row += (int64_t)gridDim.x * BACK_WARPS) {
        const T *dys = static_cast<const T *>(p.dy) + row * p.lddy + lane, *hs = static_cast<const T *>(p.h) + row * p.ldh + lane;
        const T *dhs = static_cast<const T *>(p.dh) + row * p.lddh + lane;
        T *dxs = static_cast<T *>(p.dx) + row * p.lddx + lane;
        const float r = p.rstd[row];
        const T zero = from_f32<T>(0.0f);
        T dy[NE], h[NE], dh[NE];
#pragma unroll
        for (int j = 0; j < NE; ++j) {
            const bool in = lane + 32 * j < width;
            dy[j] = in ? dys[32 * j] : zero;
            h[j] = in ? hs[32 * j] : zero;
            dh[j] = in && p.dh ? dhs[32 * j] : zero;
        }
        float dot = 0.0f;
#pragma unroll
        for (int j = 0; j < NE; ++j) {
            const float d = to_f32(dy[j]), u = __fmul_rn(to_f32(h[j]), r);
            dot = __fmaf_rn(__fmul_rn(d, g[j]), u, dot);
            sum[j] = __fmaf_rn(d, u, sum[j]);
        }
        const float mean = __fdiv_rn(warp_sum(dot), (float)width);
#pragma unroll
        for (int j = 0; j < NE; ++j) {
            const float u = __fmul_rn(to_f32(h[j]), r);
            const float d = __fadd_rn(__fmul_rn(__fmaf_rn(-u, mean, __fmul_rn(to_f32(dy[j]), g[j])), r), to_f32(dh[j]));
            if (lane + 32 * j < width) dxs[32 * j] = from_f32<T>(d);
        }
    }
#pragma unroll
    for (int j = 0; j < NE; ++j) all[warp][lane + 32 * j] = sum[j];
    __syncthreads();
    for (int c = threadIdx.x; c < width; c += BACK_WARPS * 32) {
        float s = all[0][c];
#pragma unroll
        for (int w = 1; w < BACK_WARPS; ++w) s = __fadd_rn(s, all[w][c]);
        p.sums[(int64_t)blockIdx.x * width + c] = s;
    }
}

// Wider rows that cannot be accessed in packs, element by element, NE of them a thread, blockDim.x apart; ROWS rows for each barrier.
template <class T, class G, int NE, int ROWS>
__global__ void __launch_bounds__(ROWS > 1 ? 256 : 512, NE <= 8 ? 2 : 1) norm_back_elements_kernel(const NormBackParams p) {
    __shared__ float parts[2][ROWS][16];
    start_next();
    wait_for_previous();
    const int step = blockDim.x, width = p.width, first = threadIdx.x;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const G *gain = static_cast<const G *>(p.gain) + first;
    float g[NE], sum[NE];
#pragma unroll
    for (int j = 0; j < NE; ++j) {
        g[j] = first + j * step < width ? to_f32(gain[j * step]) : 0.0f;
        sum[j] = 0.0f;
    }
    int side = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += ROWS * (int64_t)gridDim.x, side ^= 1) {
        const T zero = from_f32<T>(0.0f);
        T dy[ROWS][NE], h[ROWS][NE], dh[ROWS][NE];
        float r[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {                        // (rows past the last are rows of zeros, and not stored)
            const int64_t at = row + k * (int64_t)gridDim.x;
            const bool there = at < p.rows;
            const T *dys = static_cast<const T *>(p.dy) + at * p.lddy + first, *hs = static_cast<const T *>(p.h) + at * p.ldh + first;
            const T *dhs = static_cast<const T *>(p.dh) + at * p.lddh + first;
            r[k] = there ? p.rstd[at] : 0.0f;
#pragma unroll
            for (int j = 0; j < NE; ++j) {
                const bool in = there && first + j * step < width;
                dy[k][j] = in ? dys[j * step] : zero;
                h[k][j] = in ? hs[j * step] : zero;
                dh[k][j] = in && p.dh ? dhs[j * step] : zero;
            }
        }
        float dot[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            dot[k] = 0.0f;
#pragma unroll
            for (int j = 0; j < NE; ++j) {
                const float d = to_f32(dy[k][j]), u = __fmul_rn(to_f32(h[k][j]), r[k]);
                dot[k] = __fmaf_rn(__fmul_rn(d, g[j]), u, dot[k]);
                sum[j] = __fmaf_rn(d, u, sum[j]);
            }
            dot[k] = warp_sum(dot[k]);
            if (lane == 0) parts[side][k][warp] = dot[k];       // (two sides: the next rows' sums do not wait for these ones' readers)
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t at = row + k * (int64_t)gridDim.x;
            const float mean = __fdiv_rn(warp_sum(lane < warps ? parts[side][k][lane] : 0.0f), (float)width);
            T *dxs = static_cast<T *>(p.dx) + at * p.lddx + first;
#pragma unroll
            for (int j = 0; j < NE; ++j) {
                const float u = __fmul_rn(to_f32(h[k][j]), r[k]);
                const float d = __fadd_rn(__fmul_rn(__fmaf_rn(-u, mean, __fmul_rn(to_f32(dy[k][j]), g[j])), r[k]), to_f32(dh[k][j]));
                if (at < p.rows && first + j * step < width) dxs[j * step] = from_f32<T>(d);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < NE; ++j)
        if (first + j * step < width) p.sums[(int64_t)blockIdx.x * width + first + j * step] = sum[j];
}

// Wider ones than that has registers for: a thread's sums are in shared memory, and rows are read twice.
template <class T, class G>
__global__ void __launch_bounds__(512) norm_back_any_kernel(const NormBackParams p) {
    extern __shared__ float sums[];
    __shared__ float parts[2][32];
    start_next();
    wait_for_previous();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const G *gain = static_cast<const G *>(p.gain);
    for (int i = threadIdx.x; i < p.width; i += blockDim.x) sums[i] = 0.0f;
    int side = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, side ^= 1) {
        const T *dy = static_cast<const T *>(p.dy) + row * p.lddy, *h = static_cast<const T *>(p.h) + row * p.ldh;
        const T *dh = static_cast<const T *>(p.dh) + row * p.lddh;
        T *dx = static_cast<T *>(p.dx) + row * p.lddx;
        const float r = p.rstd[row];
        float dot = 0.0f;
#pragma unroll 4
        for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
            const float d = to_f32(dy[i]), u = __fmul_rn(to_f32(h[i]), r);
            dot = __fmaf_rn(__fmul_rn(d, to_f32(gain[i])), u, dot);
            sums[i] = __fmaf_rn(d, u, sums[i]);
        }
        dot = warp_sum(dot);
        if (lane == 0) parts[side][warp] = dot;
        __syncthreads();
        const float mean = __fdiv_rn(warp_sum(lane < warps ? parts[side][lane] : 0.0f), (float)p.width);
#pragma unroll 4
        for (int i = threadIdx.x; i < p.width; i += blockDim.x) {
            const float u = __fmul_rn(to_f32(h[i]), r);
            float d = __fmul_rn(__fmaf_rn(-u, mean, __fmul_rn(to_f32(dy[i]), to_f32(gain[i]))), r);
            if (p.dh) d = __fadd_rn(d, to_f32(dh[i]));
            dx[i] = from_f32<T>(d);
        }
    }
    for (int i = threadIdx.x; i < p.width; i += blockDim.x) p.sums[(int64_t)blockIdx.x * p.width + i] = sums[i];
}

// dgain[c] = sum over `parts` rows of sums.  A thread adds every 32nd of them, with twelve loads under way; 32 threads a column, whose sums
// are added in order.
constexpr int BACK_PARTS = 296;
__global__ void __launch_bounds__(1024) norm_gain_kernel(const float *sums, int parts, int width, float *dgain) {
    __shared__ float part[32][33];
    start_next();
    wait_for_previous();
    const int c = blockIdx.x * 32 + threadIdx.x;
    float sum = 0.0f;
    for (int q0 = threadIdx.y; q0 < parts; q0 += 32 * 12) {
        float v[12];
#pragma unroll
        for (int i = 0; i < 12; ++i) v[i] = c < width && q0 + 32 * i < parts ? sums[(int64_t)(q0 + 32 * i) * width + c] : 0.0f;
#pragma unroll
        for (int i = 0; i < 12; ++i) sum = __fadd_rn(sum, v[i]);
    }
    part[threadIdx.y][threadIdx.x] = sum;
    __syncthreads();
    const float total = warp_sum(part[threadIdx.x][threadIdx.y]);         // warp y takes column y
    if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < width) dgain[blockIdx.x * 32 + threadIdx.y] = total;
}

// Blocks of the backward kernel; sized for 148 SMs, so that workspace queries and calls agree.
int back_blocks(int64_t rows) { return (int)(rows < BACK_PARTS ? rows : BACK_PARTS); }

template <class T, class G, int NV>
int back_launch(const NormBackParams &p, int packs, cudaStream_t st) {
    const int stage = (p.dh ? 3 : 2) * p.width * (int)sizeof(T), fit = 100 * 1024 / stage, stages = fit < 2 ? 2 : fit < 8 ? fit : 8;
    if (!allow_shared_memory<norm_back_kernel<T, G, NV>>(200 * 1024)) return QNN_E_CUDA;
    LaunchAttrs attrs(1);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(back_blocks(p.rows));
    cfg.blockDim = dim3(whole_warps((packs + NV - 1) / NV));
    cfg.dynamicSmemBytes = stages * stage;
    cfg.stream = st;
    cfg.attrs = attrs.a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, norm_back_kernel<T, G, NV>, p, stages, stage) == cudaSuccess) return QNN_OK;
    cudaGetLastError();
    return QNN_E_CUDA;
}
template <class T, class G, int NV>
int back_warps_launch(const NormBackParams &p, cudaStream_t st) {
    LaunchAttrs attrs(1);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(back_blocks(p.rows));
    cfg.blockDim = dim3(BACK_WARPS * 32);
    cfg.dynamicSmemBytes = BACK_WARPS * 32 * NV * Octets<T>::V * sizeof(float);      // (at most 32 KB)
    cfg.stream = st;
    cfg.attrs = attrs.a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, norm_back_warps_kernel<T, G, NV>, p) == cudaSuccess) return QNN_OK;
    cudaGetLastError();
    return QNN_E_CUDA;
}
template <class T, class G, int NE, int ROWS>
int back_elements_launch(const NormBackParams &p, cudaStream_t st) {
    return launch_early(norm_back_elements_kernel<T, G, NE, ROWS>, dim3(back_blocks(p.rows)), dim3(whole_warps((p.width + NE - 1) / NE)), st, p);
}
template <class T, class G>
int back_any_launch(const NormBackParams &p, cudaStream_t st) {
    const int smem = p.width * (int)sizeof(float);
    if (!allow_shared_memory<norm_back_any_kernel<T, G>>(NORM_MAX_WIDTH * (int)sizeof(float))) return QNN_E_CUDA;
    LaunchAttrs attrs(1);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(back_blocks(p.rows));
    cfg.blockDim = dim3(p.width <= 512 ? whole_warps(p.width) : 512);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attrs.a;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, norm_back_any_kernel<T, G>, p) == cudaSuccess) return QNN_OK;
    cudaGetLastError();
    return QNN_E_CUDA;
}
template <class T, class G>
int back_typed(const NormBackParams &p, bool vec, float *dgain, cudaStream_t st) {
    const int packs = p.width / (16 / (int)sizeof(T));
    int rc;
    if (!vec && p.width <= 512) rc = launch_early(norm_back_warp_elements_kernel<T, G, 16>, dim3(back_blocks(p.rows)), dim3(BACK_WARPS * 32), st, p);
    else if (!vec && p.width <= 4096) rc = p.width <= 2048 ? back_elements_launch<T, G, 8, 2>(p, st) : back_elements_launch<T, G, 8, 1>(p, st);
    else if (!vec && p.width <= 8192) rc = back_elements_launch<T, G, 16, 1>(p, st);
    else if (!vec || packs > 2048) rc = back_any_launch<T, G>(p, st);
    else if (packs <= 32) rc = back_warps_launch<T, G, 1>(p, st);
    else if (packs <= 64) rc = back_warps_launch<T, G, 2>(p, st);
    else if (packs <= 128) rc = back_warps_launch<T, G, 4>(p, st);
    else if (packs <= 256) rc = back_launch<T, G, 1>(p, packs, st);
    else if (packs <= 1024) rc = back_launch<T, G, 2>(p, packs, st);
    else rc = back_launch<T, G, 4>(p, packs, st);
    if (rc != QNN_OK) return rc;
    return launch_early(norm_gain_kernel, dim3((p.width + 31) / 32), dim3(32, 32), st, p.sums, back_blocks(p.rows), p.width, dgain);
}

// f(T, G) for the element type and the gain's (that type or fp32)
template <class F> int by_types(int type, int gain_type, F f) {
    if (type == QNN_F32) return f(float(), float());
    if (type == QNN_BF16) return gain_type == QNN_F32 ? f(__nv_bfloat16(), float()) : f(__nv_bfloat16(), __nv_bfloat16());
    return gain_type == QNN_F32 ? f(__half(), float()) : f(__half(), __half());
}
int check_gain(const void *gain, int gain_type, int type) {
    if (!gain || !(gain_type == type || gain_type == QNN_F32)) return QNN_E_ARG;
    return qnn_aligned(gain, g4_type_bytes(gain_type)) ? QNN_OK : QNN_E_ALIGN;
}

}  // namespace

extern "C" int qnn_rms_norm(const void *x, int type, int64_t rows, int width, int64_t ldx, const void *residual, int64_t ldr, const void *gain,
                            int gain_type, float eps, void *h, int64_t ldh, void *y, int64_t ldy, int8_t *codes, int64_t ldc, float *scales,
                            float *rstd, void *stream) {
    if (!g4_type_ok(type) || rows < 0 || width < 1 || !(eps >= 0.0f && eps <= 3.0e38f)) return QNN_E_ARG;
    if (width > NORM_MAX_WIDTH || rows > ROWS_MAX) return QNN_E_RANGE;
    int rc = check_gain(gain, gain_type, type);
    if (rc != QNN_OK || rows == 0) return rc;
    if (!y && !codes) return QNN_E_ARG;
    if ((rc = check_real(x, type, ldx, width)) != QNN_OK) return rc;
    if (residual && (rc = check_real(residual, type, ldr, width)) != QNN_OK) return rc;
    if (residual && (rc = check_real(h, type, ldh, width)) != QNN_OK) return rc;
    if (y && (rc = check_real(y, type, ldy, width)) != QNN_OK) return rc;
    if (codes && (rc = check_codes(codes, scales, ldc, width)) != QNN_OK) return rc;
    if (rstd && !qnn_aligned(rstd, 4)) return QNN_E_ALIGN;
    const bool vec = width * g4_type_bytes(type) % 16 == 0 && in_packs(x, type, ldx) && qnn_aligned(gain, 16) &&
                     (!residual || (in_packs(residual, type, ldr) && in_packs(h, type, ldh))) && (!y || in_packs(y, type, ldy));
    const NormParams p{x, residual, gain, ldx, ldr, ldh, ldy, ldc, rows, width, eps, h, y, codes, scales, rstd};
    return by_types(type, gain_type, [&](auto t, auto g) { return norm_typed<decltype(t), decltype(g), true>(p, vec, static_cast<cudaStream_t>(stream)); });
}

extern "C" int qnn_i8_quantize(const void *x, int type, int64_t rows, int width, int64_t ldx, int8_t *codes, int64_t ldc, float *scales,
                               void *stream) {
    if (!g4_type_ok(type) || rows < 0 || width < 1) return QNN_E_ARG;
    if (width > CODES_MAX_WIDTH || rows > ROWS_MAX) return QNN_E_RANGE;
    if (rows == 0) return QNN_OK;
    int rc = check_real(x, type, ldx, width);
    if (rc == QNN_OK) rc = check_codes(codes, scales, ldc, width);
    if (rc != QNN_OK) return rc;
    const bool vec = width * g4_type_bytes(type) % 16 == 0 && in_packs(x, type, ldx);
    NormParams p{};
    p.x = x; p.ldx = ldx; p.rows = rows; p.width = width; p.codes = codes; p.ldc = ldc; p.scales = scales;
    return by_types(type, type, [&](auto t, auto) { return norm_typed<decltype(t), decltype(t), false>(p, vec, static_cast<cudaStream_t>(stream)); });
}

extern "C" int qnn_i8_decode(const int8_t *codes, const float *scales, int64_t rows, int width, int64_t ldc, int type, void *out, int64_t ldo,
                             void *stream) {
    if (!g4_type_ok(type) || rows < 0 || width < 1) return QNN_E_ARG;
    if (width > CODES_MAX_WIDTH || rows > ROWS_MAX) return QNN_E_RANGE;
    if (rows == 0) return QNN_OK;
    int rc = check_codes(codes, scales, ldc, width);
    if (rc == QNN_OK) rc = check_real(out, type, ldo, width);
    if (rc != QNN_OK) return rc;
    const bool vec = width * g4_type_bytes(type) % 16 == 0 && in_packs(out, type, ldo);
    return by_types(type, type, [&](auto t, auto) { return decode<decltype(t)>(codes, scales, rows, width, ldc, out, ldo, vec, static_cast<cudaStream_t>(stream)); });
}

extern "C" size_t qnn_rms_norm_backward_workspace(int64_t rows, int width) {
    if (rows < 1 || rows > ROWS_MAX || width < 1 || width > NORM_MAX_WIDTH) return 0;
    return ((size_t)back_blocks(rows) * (size_t)width * sizeof(float) + 255) / 256 * 256;
}

extern "C" int qnn_rms_norm_backward(const void *dy, int type, int64_t rows, int width, int64_t lddy, const void *h, int64_t ldh,
                                     const void *gain, int gain_type, const float *rstd, const void *dh, int64_t lddh, void *dx, int64_t lddx,
                                     float *dgain, void *workspace, size_t workspace_bytes, void *stream) {
    if (!g4_type_ok(type) || rows < 0 || width < 1 || !dgain) return QNN_E_ARG;
    if (width > NORM_MAX_WIDTH || rows > ROWS_MAX) return QNN_E_RANGE;
    if (!qnn_aligned(dgain, 4)) return QNN_E_ALIGN;
    int rc = check_gain(gain, gain_type, type);
    if (rc != QNN_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) return cudaMemsetAsync(dgain, 0, (size_t)width * sizeof(float), st) == cudaSuccess ? QNN_OK : QNN_E_CUDA;
    if (!rstd) return QNN_E_ARG;
    if ((rc = check_real(dy, type, lddy, width)) != QNN_OK || (rc = check_real(h, type, ldh, width)) != QNN_OK ||
        (rc = check_real(dx, type, lddx, width)) != QNN_OK || (dh && (rc = check_real(dh, type, lddh, width)) != QNN_OK))
        return rc;
    if (!workspace || workspace_bytes < qnn_rms_norm_backward_workspace(rows, width)) return QNN_E_ARG;
    if (!qnn_aligned(workspace, 256) || !qnn_aligned(rstd, 4)) return QNN_E_ALIGN;
    const bool vec = width * g4_type_bytes(type) % 16 == 0 && in_packs(dy, type, lddy) && in_packs(h, type, ldh) && in_packs(dx, type, lddx) &&
                     (!dh || in_packs(dh, type, lddh)) && qnn_aligned(gain, 16);
    const NormBackParams p{dy, h, gain, dh, rstd, lddy, ldh, lddh, lddx, rows, width, dx, static_cast<float *>(workspace), qnn_tc_error_word(), WAIT_LIMIT};
    if (!p.err) return QNN_E_CUDA;
    return by_types(type, gain_type, [&](auto t, auto g) { return back_typed<decltype(t), decltype(g)>(p, vec, dgain, st); });
}
