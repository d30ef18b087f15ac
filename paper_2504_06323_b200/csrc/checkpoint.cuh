// Activations in 8 bits: 16 adjacent columns of a row share an exponent.
//     E = biased exponent of the largest finite magnitude of the group, at least 1
//     code = x 2^(133 - E) rounded to the nearest whole number (ties to even), within +-127; -128 for NaN and infinities
//     value = code 2^(E - 133)
// A bf16 value has eight significant bits, a code seven and a sign: the group's largest values lose at most their last bit, and
// what clamps is at most 127.5.  Powers of two make every step exact but the one rounding: codes do not depend on how they are
// computed, and a value is a bf16 number again (seven significant bits, no exponent below bf16's).
#pragma once
#include "lanes.cuh"

namespace mosaic {
constexpr int kSavedGroup = 16;

// A checkpoint's matrix, checked: codes on 16-byte boundaries with room for whole groups, exponents row by row.
struct Saved {
    int8_t* codes;
    int64_t ldc;
    uint8_t* exponents;
    int64_t lde;
};
inline int64_t saved_groups(int64_t cols) { return (cols + kSavedGroup - 1) / kSavedGroup; }
inline size_t saved_code_bytes(const Saved& s, int64_t rows, int64_t cols) {
    return rows > 0 ? (size_t)(rows - 1) * (size_t)s.ldc + (size_t)(saved_groups(cols) * kSavedGroup) : 0u;
}
inline size_t saved_exponent_bytes(const Saved& s, int64_t rows, int64_t cols) {
    return rows > 0 ? (size_t)(rows - 1) * (size_t)s.lde + (size_t)saved_groups(cols) : 0u;
}
int check_saved(const mosaic_checkpoint* c, int64_t rows, int64_t cols);
inline Saved as_saved(const mosaic_checkpoint* c) {
    return {static_cast<int8_t*>(c->codes), c->ldc, static_cast<uint8_t*>(c->exponents), c->lde};
}
// Enqueue the conversions (arguments checked).
int store_saved(const void* X, int64_t ldx, int64_t rows, int64_t cols, const Saved& out, cudaStream_t st);
int load_saved(const Saved& in, int64_t rows, int64_t cols, void* X, int64_t ldx, cudaStream_t st);

#ifdef __CUDACC__
// The exponent of a group from its largest finite magnitude (bf16 bits without the sign).
__device__ __forceinline__ uint32_t saved_exponent(uint32_t largest) { return largest >> 7 > 1u ? largest >> 7 : 1u; }
// Magnitude bits that count for the exponent.
__device__ __forceinline__ uint32_t finite_bits(uint32_t half) { return (half & 0x7F80u) == 0x7F80u ? 0u : half & 0x7FFFu; }
// 2^(133 - E) as a product of two factors that are normal numbers.
struct SavedScale {
    float first, second;
    __device__ __forceinline__ explicit SavedScale(uint32_t E) {
        first = __uint_as_float((E >= 6u ? 260u - E : 254u) << 23);
        second = E >= 6u ? 1.0f : __uint_as_float((133u - E) << 23);
    }
};
__device__ __forceinline__ int saved_code(float x, const SavedScale& s) {
    const float y = __fmul_rn(__fmul_rn(x, s.first), s.second);
    const int q = min(127, max(-127, __float2int_rn(y)));
    return fabsf(x) <= 3.4e38f ? q : -128;
}
__device__ __forceinline__ float saved_value(int code, uint32_t E) {
    const float v = __fmul_rn(__fmul_rn((float)code, 0.015625f), __uint_as_float(E << 23));
    return code == -128 ? __uint_as_float(0x7FC00000u) : v;
}
// Eight values of a lane from their codes.
__device__ __forceinline__ void saved_values8(uint2 codes, uint32_t E, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = saved_value((int)(int8_t)((e < 4 ? codes.x : codes.y) >> (8 * (e & 3))), E);
}
#endif
}  // namespace mosaic
