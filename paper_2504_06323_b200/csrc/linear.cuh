// Shared by the matrix products of linear.cu and the elementwise passes around them.
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"

namespace mosaic {

#ifdef __CUDACC__
__device__ __forceinline__ float bf16_to_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t f32_to_bf16(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }

// Logistic function 1 / (1 + e^-z).  The hardware's exponential and reciprocal are off by about 2^-22 near zero and by
// 2^-16 at z = -80 (the exponential's error grows with its argument): below the bf16 rounding of whatever is made of
// it.  From z = -87.3 down, where it is under 10^-37, it is 0.
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

// (1 + erf(z / sqrt 2)) / 2, the normal distribution's integral up to z, from bell = e^(-z^2 / 2).  As a sum it would
// cancel for negative z (at z = -5 a few bits are left), so it is the tail beyond |z|, or 1 minus that:
//     tail = bell t p(t),  t = 1 / (1 + 5/16 |z|),
// p a polynomial fitted to the smooth quotient (relative error 2^-22 for |z| <= 14; beyond, the tail is under 10^-43).
// Calls of erfc instead filled the epilogues' straight code and made 14336 outputs of 2048 tokens 15 % slower.
__device__ __forceinline__ float normal_cdf(float z, float bell) {
    const float t = __fdividef(1.0f, __fmaf_rn(0.3125f, fabsf(z), 1.0f));
    float p = 0.035262212f;
    p = __fmaf_rn(p, t, -0.13551591f);
    p = __fmaf_rn(p, t, 0.13984019f);
    p = __fmaf_rn(p, t, -0.0040229424f);
    p = __fmaf_rn(p, t, 0.105123475f);
    p = __fmaf_rn(p, t, 0.10976139f);
    p = __fmaf_rn(p, t, 0.124888316f);
    p = __fmaf_rn(p, t, 0.124663375f);
    const float tail = bell * (t * p);
    return z < 0.0f ? tail : 1.0f - tail;
}
__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case MOSAIC_ACT_RELU: return z > 0.0f || z != z ? z : 0.0f;
        case MOSAIC_ACT_GELU: return z * normal_cdf(z, __expf(-0.5f * z * z));
        case MOSAIC_ACT_SILU: return z * logistic(z);
        default: return z;
    }
}
// The same for a lane's run of values: one branch, then straight code.
template <int N> __device__ __forceinline__ void activate_all(float (&v)[N], int act) {
    if (act == MOSAIC_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], MOSAIC_ACT_RELU);
    } else if (act == MOSAIC_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], MOSAIC_ACT_SILU);
    } else if (act == MOSAIC_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = activate(v[e], MOSAIC_ACT_GELU);
    }
}
// d activate(z) / dz
__device__ __forceinline__ float activate_slope(float z, int act) {
    switch (act) {
        case MOSAIC_ACT_RELU: return z > 0.0f ? 1.0f : (z != z ? z : 0.0f);
        case MOSAIC_ACT_GELU: {
            const float bell = __expf(-0.5f * z * z);
            return normal_cdf(z, bell) + z * bell * 0.39894228040143268f;
        }
        case MOSAIC_ACT_SILU: {
            const float s = logistic(z);
            return s * (1.0f + z * (1.0f - s));
        }
        default: return 1.0f;
    }
}
template <int N> __device__ __forceinline__ void slope_all(float (&z)[N], int act) {
    if (act == MOSAIC_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = activate_slope(z[e], MOSAIC_ACT_RELU);
    } else if (act == MOSAIC_ACT_SILU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = activate_slope(z[e], MOSAIC_ACT_SILU);
    } else if (act == MOSAIC_ACT_GELU) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = activate_slope(z[e], MOSAIC_ACT_GELU);
    }
}
#endif
}  // namespace mosaic
