// Rows of real numbers as the row-wise kernels (rms_norm.cu, route.cu, i8_gemm.cu) see them: element types, 16 bytes of them in one
// access, and the code of a value in 8 bits.
#pragma once
#include <type_traits>
#include "g4_format.cuh"

constexpr int64_t ROWS_MAX = (1ll << 31) - 1;      // rows of a call

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// 16 bytes of a row as fp32 numbers, and back.
template <class T> struct Octets {
    static constexpr int V = 8;
    __device__ static __forceinline__ void get(const uint4 &w, float (&f)[8]) {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                f[2 * i] = __uint_as_float(u[i] << 16);
                f[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
            } else {
                const float2 v = __half22float2(*reinterpret_cast<const __half2 *>(&u[i]));
                f[2 * i] = v.x;
                f[2 * i + 1] = v.y;
            }
        }
    }
    __device__ static __forceinline__ uint4 put(const float (&f)[8]) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                u[i] = *reinterpret_cast<const uint32_t *>(&v);
            } else {
                const __half2 v = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
                u[i] = *reinterpret_cast<const uint32_t *>(&v);
            }
        }
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <> struct Octets<float> {
    static constexpr int V = 4;
    __device__ static __forceinline__ void get(const uint4 &w, float (&f)[4]) {
        f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
    }
    __device__ static __forceinline__ uint4 put(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
};
// Numbers of a gain of type G that go with pack i of rows of T.
template <class T, class G> __device__ __forceinline__ void gain_of_pack(const void *gain, int i, float (&f)[Octets<T>::V]) {
    if constexpr (std::is_same<T, G>::value) {
        Octets<T>::get(static_cast<const uint4 *>(gain)[i], f);
    } else {
        const uint4 *g = static_cast<const uint4 *>(gain) + 2 * i;              // fp32 beside a 2-byte type
        float lo[4], hi[4];
        Octets<float>::get(g[0], lo);
        Octets<float>::get(g[1], hi);
#pragma unroll
        for (int e = 0; e < 4; ++e) { f[e] = lo[e]; f[4 + e] = hi[e]; }
    }
}

// The larger one; NaN if either is (fmaxf would drop it).
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// A row's scale from its largest magnitude m: m / 127, at least the smallest normal number, so that 1 / scale is finite and a row
// of zeros decodes to zeros.  NaN for a row that holds an infinity or NaN.
constexpr float TO_NEAREST = 12582912.0f;          // 1.5 * 2^23: a sum with it holds the nearest whole number in its low bits
//
// A code is rint(y / scale), the quotient rounded to fp32, and comes without a division: q0 = y * inverse, corrected by its residual,
// q = q0 + (y - q0 * scale) * inverse.  Only where y / scale is next to a border, half a step of fp32 off a half H, could q fall on the
// border's other side.  With scale = S * 2^a, 2^23 < S < 2^24 (all is exact for S = 2^23), y and H * scale are multiples of 2^(a-1), so that
// a quotient lies j / 2S steps off its border with a whole j, never 0.  There q0, whose product is off by 0.993 steps before it is rounded, is
// one of the border's two neighbours and the residual is exact; the inverse, off by S * 2^-48 (relative), makes the sum off by
// (S + j) * 2^-49 steps at most: less than j / 2S, as S * (S + j) < j * 2^48.  (Farther off, from j = 7, it is off by 3 * 2^-24 steps at most.)
// The residual has to be a normal number: rows of small scales are raised by a power of two, which changes no quotient.  |y| <= 127 scale:
// no clamp is needed.
struct RowScale {
    float scale, up, raised, inverse;              // up: 1, or what small scales are raised by; raised = scale * up; inverse of that
    __device__ __forceinline__ explicit RowScale(float m) {
        const bool finite = m <= 3.402823466e38f;
        scale = finite ? fmaxf(__fdiv_rn(m, 127.0f), 1.17549435e-38f) : __int_as_float(0x7FC00000);
        up = scale < 8.67361738e-19f ? 1.8446744e19f : 1.0f;        // 2^-60, 2^64
        raised = __fmul_rn(scale, up);
        inverse = finite ? __frcp_rn(raised) : 0.0f;
    }
    // The code of y as the low byte of a word; any byte where the scale is NaN.  RAISED: whether the row is one that has to be raised (a
    // multiplication more for each code, so that rows take their own side of a branch).
    __device__ __forceinline__ bool is_raised() const { return up != 1.0f; }
    template <bool RAISED> __device__ __forceinline__ uint32_t code(float y) const {
        const float a = RAISED ? __fmul_rn(y, up) : y, q = __fmul_rn(a, inverse), r = __fmaf_rn(-q, raised, a);
        return __float_as_uint(__fadd_rn(__fmaf_rn(r, inverse, q), TO_NEAREST));
    }
    // Bytes of codes, zeros where the scale is NaN.
    __device__ __forceinline__ uint32_t word(uint32_t a, uint32_t b, uint32_t c, uint32_t d) const {
        const uint32_t w = __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
        return inverse != 0.0f ? w : 0u;
    }
};
