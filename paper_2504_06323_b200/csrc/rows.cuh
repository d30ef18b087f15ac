// Rows of logits in registers: how the kernels over a model's output distribution (top logits,
// distillation) read a row of any length, alignment and leading dimension, and the running maximum
// and sum of a softmax over it.
//
// A row is cut into 16-byte vectors that start on 16-byte boundaries; the first and the last may hold
// fewer than a whole vector's elements (an odd vocabulary, a dense matrix whose rows start anywhere).
// Whole vectors are one 16-byte load, the two ragged ones are read element by element, and the places
// outside the row are filled with -inf: nothing outside the row is read.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace mosaic {

constexpr int kRowThreads = 512;   // threads of a CTA
constexpr int kRowVecs = 8;        // vectors a thread holds in registers (128 bytes: 64 KB of a row per CTA)
constexpr int kRowWarps = kRowThreads / 32;
constexpr int kMaxTop = 1024;      // kept logits per row
constexpr int64_t kMaxRow = 0x7FFFFF00;   // elements of a row: column and vector numbers fit 32 bits with room to spare
constexpr int kMaxCluster = 8;     // CTAs that share one row (the portable cluster size)

// ---------------------------------------------------------------- host side
// CTAs per row.  A CTA holds kRowThreads * kRowVecs vectors of a row in registers (read once); a longer
// row is shared by a cluster, and where the rows alone would leave SMs idle a row is spread further, as
// long as every thread keeps a vector.
inline int row_cluster(int64_t rows, int64_t vectors) {
    int c = 1;
    while (c < kMaxCluster && vectors > (int64_t)c * kRowThreads * kRowVecs) c *= 2;
    while (c < kMaxCluster && rows * c < sm_count() && vectors >= (int64_t)2 * c * kRowThreads) c *= 2;
    return c;
}
// Most vectors a row of `cols` elements can be cut into, whatever its alignment.
inline int64_t row_vectors(int64_t cols, int dtype) {
    const int64_t per = 16 / (int64_t)elem_size(dtype);
    return (cols + 2 * per - 2) / per;
}

#ifdef __CUDACC__
// 2^x by the hardware's approximation (relative error about 2^-22, results below 2^-126 become 0).
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int DT> struct RowVec;
template <> struct RowVec<MOSAIC_BF16> {
    static constexpr int kElems = 8;
    using Elem = uint16_t;
    static constexpr uint32_t kFill = 0xFF80FF80u;   // -inf, -inf
    __device__ static __forceinline__ float widen(uint32_t bits) { return __uint_as_float(bits << 16); }
    __device__ static __forceinline__ float get(const uint4& v, int e) {
        const uint32_t w = (e >> 1) == 0 ? v.x : (e >> 1) == 1 ? v.y : (e >> 1) == 2 ? v.z : v.w;
        return __uint_as_float((e & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
    __device__ static __forceinline__ Elem narrow(float f) {   // one rounding to nearest, ties to even
        return __bfloat16_as_ushort(__float2bfloat16_rn(f));
    }
    __device__ static __forceinline__ uint32_t pair(float lo, float hi) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
        return (uint32_t)__bfloat16_as_ushort(p.x) | ((uint32_t)__bfloat16_as_ushort(p.y) << 16);
    }
    __device__ static __forceinline__ uint4 pack(const float (&f)[8]) {
        return make_uint4(pair(f[0], f[1]), pair(f[2], f[3]), pair(f[4], f[5]), pair(f[6], f[7]));
    }
    __device__ static __forceinline__ void put(uint4& v, int e, Elem b) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
        w[e >> 1] = (e & 1) ? ((w[e >> 1] & 0xFFFFu) | ((uint32_t)b << 16)) : ((w[e >> 1] & 0xFFFF0000u) | b);
    }
};
template <> struct RowVec<MOSAIC_F32> {
    static constexpr int kElems = 4;
    using Elem = uint32_t;
    static constexpr uint32_t kFill = 0xFF800000u;
    __device__ static __forceinline__ float widen(uint32_t bits) { return __uint_as_float(bits); }
    __device__ static __forceinline__ float get(const uint4& v, int e) {
        return __uint_as_float(e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w);
    }
    __device__ static __forceinline__ Elem narrow(float f) { return __float_as_uint(f); }
    __device__ static __forceinline__ uint4 pack(const float (&f)[4]) {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    __device__ static __forceinline__ void put(uint4& v, int e, Elem b) { reinterpret_cast<uint32_t*>(&v)[e] = b; }
};

// One row and the part of its vectors that this CTA of the row's cluster owns.
template <int DT> struct RowPart {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    const Elem* row;
    int cols;
    int off;              // elements between the first vector's boundary and the row's first element
    int v_lo, v_hi;   // this CTA's vectors

    __device__ __forceinline__ RowPart(const void* base, int64_t r, int64_t ld, int cols_, int rank, int n_ctas) : cols(cols_) {
        row = reinterpret_cast<const Elem*>(base) + r * ld;
        off = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(Elem));
        const int nv = (cols + off + RV::kElems - 1) / RV::kElems;
        const int per = (nv + n_ctas - 1) / n_ctas;
        v_lo = rank * per < nv ? rank * per : nv;
        v_hi = v_lo + per < nv ? v_lo + per : nv;
    }
    __device__ __forceinline__ int first(int vec) const { return vec * RV::kElems - off; }   // column of its element 0
    __device__ __forceinline__ bool whole(int vec) const {
        const int j = first(vec);
        return j >= 0 && j + RV::kElems <= cols;
    }
    __device__ __forceinline__ bool owns(int col) const {
        const int v = (col + off) / RV::kElems;
        return v >= v_lo && v < v_hi;
    }
    __device__ __forceinline__ float at(int col) const { return RV::widen(row[col]); }
    __device__ __forceinline__ uint4 load(int vec) const {
        const int j = first(vec);
        if (j >= 0 && j + RV::kElems <= cols) return ld_stream16(row + j);
        uint4 v = make_uint4(RV::kFill, RV::kFill, RV::kFill, RV::kFill);
#pragma unroll
        for (int e = 0; e < RV::kElems; ++e)
            if (j + e >= 0 && j + e < cols) RV::put(v, e, row[j + e]);
        return v;
    }
    // The thread's vectors of one pass, all loads issued before the first is used.
    __device__ __forceinline__ void load_pass(int base, uint4 (&raw)[kRowVecs]) const {
#pragma unroll
        for (int i = 0; i < kRowVecs; ++i) {
            const int v = base + (int)threadIdx.x + i * kRowThreads;
            raw[i] = v < v_hi ? load(v) : make_uint4(RV::kFill, RV::kFill, RV::kFill, RV::kFill);
        }
    }
};

// Running maximum m and sum s of 2^(c (x - m)) over some entries of a row; an infinite m counts as 0
// inside the sum, so that a row of -inf has the sum 0, +inf the sum +inf, and NaN stays NaN.
struct SoftStat {
    float m, s;
};
__device__ __forceinline__ float soft_ref(float m) { return fabsf(m) <= 3.402823466e38f ? m : 0.0f; }
__device__ __forceinline__ float soft_scale(float m, float to, float c) { return m == to ? 1.0f : exp2_fast((m - to) * c); }
__device__ __forceinline__ SoftStat soft_merge(SoftStat a, SoftStat b, float c) {
    const float m = fmaxf(a.m, b.m);
    return {m, __fadd_rn(__fmul_rn(a.s, soft_scale(a.m, m, c)), __fmul_rn(b.s, soft_scale(b.m, m, c)))};
}
// Between two passes over the registers: the compiler may not carry widened copies of the 64 entries across
// (they do not fit beside the vectors and were spilled).
__device__ __forceinline__ void keep_packed(uint4 (&raw)[kRowVecs]) {
#pragma unroll
    for (int i = 0; i < kRowVecs; ++i) asm volatile("" : "+r"(raw[i].x), "+r"(raw[i].y), "+r"(raw[i].z), "+r"(raw[i].w));
}
// The thread's statistics of the vectors of one pass, merged into `st`.
template <int DT> __device__ __forceinline__ void soft_pass(uint4 (&raw)[kRowVecs], float c, SoftStat& st) {
    using RV = RowVec<DT>;
    float m = st.m;
#pragma unroll
    for (int i = 0; i < kRowVecs; ++i)
#pragma unroll
        for (int e = 0; e < RV::kElems; ++e) m = fmaxf(m, RV::get(raw[i], e));
    keep_packed(raw);
    // (x - m) first, then the factor: near the maximum the difference is exact, so the factor's rounding
    // costs next to nothing there; folded into one multiply-add, m * c would shift every term alike.
    const float ref = soft_ref(m);
    float s = __fmul_rn(st.s, soft_scale(st.m, m, c));
#pragma unroll
    for (int i = 0; i < kRowVecs; ++i) {
        float t = 0.0f;   // a vector's sum first: fewer roundings at the size of the total
#pragma unroll
        for (int e = 0; e < RV::kElems; ++e) t = __fadd_rn(t, exp2_fast(__fmul_rn(__fsub_rn(RV::get(raw[i], e), ref), c)));
        s = __fadd_rn(s, t);
    }
    st.m = m;
    st.s = s;
}
// The warp's statistics in every lane.
__device__ __forceinline__ SoftStat soft_warp(SoftStat st, float c) {
    float m = st.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    float s = __fmul_rn(st.s, soft_scale(st.m, m, c));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s = __fadd_rn(s, __shfl_xor_sync(0xFFFFFFFFu, s, o));
    return {m, s};
}
// Merges n statistics in their order; every thread that calls it gets the same value.
__device__ __forceinline__ SoftStat soft_all(const SoftStat* part, int n, float c) {
    SoftStat a = part[0];
    for (int i = 1; i < n; ++i) a.m = fmaxf(a.m, part[i].m);
    a.s = 0.0f;
    for (int i = 0; i < n; ++i) a.s = __fadd_rn(a.s, __fmul_rn(part[i].s, soft_scale(part[i].m, a.m, c)));
    return a;
}
// log sum exp(x / T) of a row, from its statistics (c = log2(e) / T).
__device__ __forceinline__ double soft_lse(SoftStat st, double inv_t) { return (double)soft_ref(st.m) * inv_t + log((double)st.s); }
#endif
}  // namespace mosaic
