// Shared by the matrix products of linear.cu and the elementwise passes around them.
#pragma once
#include <cuda_bf16.h>

#include "common.cuh"

namespace mosaic {

#ifdef __CUDACC__
__device__ __forceinline__ float bf16_to_f32(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ uint16_t f32_to_bf16(float f) { return __bfloat16_as_ushort(__float2bfloat16_rn(f)); }

// Logistic function 1 / (1 + e^-z).  The hardware's exponential and reciprocal (relative error about 2^-22)
// are far below the bf16 rounding of whatever is made of it.
__device__ __forceinline__ float logistic(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case MOSAIC_ACT_RELU: return z > 0.0f || z != z ? z : 0.0f;
        case MOSAIC_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
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
        case MOSAIC_ACT_GELU:
            return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * __expf(-0.5f * z * z) * 0.39894228040143268f;
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
