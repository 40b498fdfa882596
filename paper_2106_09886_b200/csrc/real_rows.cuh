// Rows of real numbers as the row-wise kernels (rms_norm.cu, route.cu, i8_gemm.cu) see them: element types, packs of elements
// that move in one access, and the code of a value in 8 bits.
#pragma once
#include "g4_format.cuh"

constexpr int64_t ROWS_MAX = (1ll << 31) - 1;      // rows of a call

// N elements that are read and written in one access.
template <class T, int N> struct alignas(N * sizeof(T)) Pack {
    T e[N];
};
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// The larger one; NaN if either is (fmaxf would drop it).
__device__ __forceinline__ float max_or_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// A row's scale from its largest magnitude m: m / 127, at least the smallest normal number, so that 1 / scale is finite and a row
// of zeros decodes to zeros.  NaN for a row that holds an infinity or NaN.
struct RowScale {
    float scale, inverse;
    __device__ __forceinline__ explicit RowScale(float m) {
        const bool finite = m <= 3.402823466e38f;
        scale = finite ? fmaxf(__fdiv_rn(m, 127.0f), 1.17549435e-38f) : __int_as_float(0x7FC00000);
        inverse = finite ? __frcp_rn(scale) : 0.0f;
    }
    // rint(v / scale), the quotient rounded to fp32: the product with the inverse is off by at most 2^-23 of 127, so that only a
    // quotient next to a half needs the division itself.  0 where the scale is NaN.
    __device__ __forceinline__ int code(float v) const {
        const float t = __fmul_rn(v, inverse);
        float r = rintf(t);
        if (fabsf(__fadd_rn(t, -r)) > 0.4999f) r = rintf(__fdiv_rn(v, scale));
        return min(max(__float2int_rn(r), -127), 127);
    }
};
