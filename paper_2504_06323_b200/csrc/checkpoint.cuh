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
// The largest magnitude's bits among eight values, infinities and NaN above all numbers; and among the finite ones.
__device__ __forceinline__ uint32_t largest8(const uint32_t (&w)[4]) {
    const uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7FFF7FFFu, w[1] & 0x7FFF7FFFu), __vmaxu2(w[2] & 0x7FFF7FFFu, w[3] & 0x7FFF7FFFu));
    return max(m & 0xFFFFu, m >> 16);
}
constexpr uint32_t kNotFinite = 0x7F80u;
__device__ __forceinline__ uint32_t finite_bits(uint32_t half) { return (half & kNotFinite) == kNotFinite ? 0u : half & 0x7FFFu; }
__device__ __forceinline__ uint32_t largest_finite8(const uint32_t (&w)[4]) {
    uint32_t largest = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) largest = max(largest, max(finite_bits(w[e] & 0xFFFFu), finite_bits(w[e] >> 16)));
    return largest;
}
__device__ __forceinline__ uint32_t saved_exponent(uint32_t largest) { return largest >> 7 > 1u ? largest >> 7 : 1u; }

// Eight values' codes.  One fma scales (exactly) and rounds: adding 3 2^22 leaves a small number's whole part in the float's low
// bits, ties to even.  The eight sums are packed by multiplying them into place and taking off what the exponents' bits add
// up to.  128 more in each keeps borrows out, and comes off as the bytes' top bits.  finite: all eight are.
__device__ __forceinline__ uint2 saved_codes8(const uint32_t (&w)[4], uint32_t E, bool finite) {
    constexpr float kRound = 12582912.0f + 128.0f;
    constexpr uint32_t kBits = 0x4B400000u, kAll = kBits * 0x01010101u;
    uint32_t q[2] = {0u, 0u};
    const float up = __uint_as_float((E >= 6u ? 260u - E : 254u) << 23);   // 2^(133 - E), or as much of it as a float holds
    if (E >= 6u) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {   // +-127.5 is the one that would leave the range
            const float y = fminf(fmaxf(__fmaf_rn(half_of(w, e), up, kRound), kRound - 127.0f), kRound + 127.0f);
            q[e >> 2] += __float_as_uint(y) << (8 * (e & 3));
        }
    } else {
        const float more = __uint_as_float((133u - E) << 23);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = fminf(fmaxf(__fmaf_rn(__fmul_rn(half_of(w, e), up), more, kRound), kRound - 127.0f), kRound + 127.0f);
            q[e >> 2] += __float_as_uint(y) << (8 * (e & 3));
        }
    }
    q[0] = (q[0] - kAll) ^ 0x80808080u;
    q[1] = (q[1] - kAll) ^ 0x80808080u;
    if (!finite) {   // rare
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t half = (e & 1) ? w[e >> 1] >> 16 : w[e >> 1];
            if ((half & kNotFinite) == kNotFinite) q[e >> 2] = (q[e >> 2] & ~(0xFFu << (8 * (e & 3)))) | (0x80u << (8 * (e & 3)));
        }
    }
    return make_uint2(q[0], q[1]);
}

// Eight values from their codes, exactly: a byte in the middle of a float of exponent 2^15 makes it 2^15 + code + 128, and one fma
// takes the 32896 off and scales.
__device__ __forceinline__ void saved_values8(uint2 codes, uint32_t E, float (&v)[8]) {
    const uint32_t u[2] = {codes.x ^ 0x80808080u, codes.y ^ 0x80808080u};
    if (E < 230u) {
        // 2^(E - 133): a normal number from E = 7 on, below a subnormal one
        const float step = __uint_as_float(E >= 7u ? (E - 6u) << 23 : (E == 0u ? 0u : 1u << (E + 16u))), less = __fmul_rn(step, -32896.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmaf_rn(__uint_as_float(__byte_perm(u[e >> 2], 0x47000000u, 0x7404 | ((e & 3) << 4))), step, less);
    } else {   // what is taken off would leave a float's range
        const float step = __uint_as_float((E - 6u) << 23);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = __fmul_rn(__fsub_rn(__uint_as_float(__byte_perm(u[e >> 2], 0x47000000u, 0x7404 | ((e & 3) << 4))), 32896.0f), step);
    }
    const auto no_zero = [](uint32_t x) { return ((x - 0x01010101u) & ~x & 0x80808080u) == 0u; };
    if (!no_zero(u[0]) || !no_zero(u[1])) {   // a zero byte is the code of what was not finite: rare
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (((u[e >> 2] >> (8 * (e & 3))) & 0xFFu) == 0u) v[e] = __uint_as_float(0x7FC00000u);
    }
}
// Two values that are bf16 numbers.
__device__ __forceinline__ uint32_t pack_exact(float lo, float hi) { return __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632); }
#endif
}  // namespace mosaic
