// Rows of logits in registers: how the kernels over a model's output distribution (top logits,
// distillation) read a row of any length, alignment and leading dimension, and the running maximum
// and sum of a softmax over it.
//
// A row is its whole 16-byte vectors on 16-byte boundaries, one 16-byte load each, and at most a vector's
// worth of single elements on either side of them (an odd vocabulary, a dense matrix whose rows start
// anywhere), which the first threads of the row's first CTA take one each.  Nothing outside the row is read.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace mosaic {

constexpr int kRowThreads = 512;   // threads of a CTA
constexpr int kRowVecs = 8;        // vectors a thread holds in registers (128 bytes: 64 KB of a row per CTA)
constexpr int kRowCtasPerSm = 2;
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
// Vectors of a row (at most; one fewer if it starts off a boundary).
inline int64_t row_vectors(int64_t cols, int dtype) { return cols * (int64_t)elem_size(dtype) / 16; }

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
};

// One row and the part of it that this CTA of the row's cluster owns.
template <int DT> struct RowPart {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    const Elem* row;
    int cols;
    int head, tail;       // single elements before and after the whole vectors
    int v_lo, v_hi;       // this CTA's vectors
    bool first_cta;

    __device__ __forceinline__ RowPart(const void* base, int64_t r, int64_t ld, int cols_, int rank, int n_ctas) : cols(cols_) {
        row = reinterpret_cast<const Elem*>(base) + r * ld;
        const int mis = (int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(Elem));
        head = mis == 0 ? 0 : (RV::kElems - mis < cols ? RV::kElems - mis : cols);
        const int nv = (cols - head) / RV::kElems;
        tail = cols - head - nv * RV::kElems;
        const int per = (nv + n_ctas - 1) / n_ctas;
        v_lo = rank * per < nv ? rank * per : nv;
        v_hi = v_lo + per < nv ? v_lo + per : nv;
        first_cta = rank == 0;
    }
    __device__ __forceinline__ int first(int vec) const { return head + vec * RV::kElems; }   // column of its element 0
    // The column of the single element this thread takes, or -1.
    __device__ __forceinline__ int single() const {
        const int t = (int)threadIdx.x;
        return first_cta && t < head + tail ? (t < head ? t : cols - tail + (t - head)) : -1;
    }
    __device__ __forceinline__ bool owns(int col) const {
        if (col < head || col >= cols - tail) return first_cta;
        const int v = (col - head) / RV::kElems;
        return v >= v_lo && v < v_hi;
    }
    __device__ __forceinline__ float at(int col) const { return RV::widen(row[col]); }
    // The thread's vectors of one pass, all loads issued before the first is used; -inf where there is none.
    __device__ __forceinline__ void load_pass(int base, uint4 (&raw)[kRowVecs]) const {
        const Elem* p = row + head;
#pragma unroll
        for (int i = 0; i < kRowVecs; ++i) {
            const int v = base + (int)threadIdx.x + i * kRowThreads;
            raw[i] = make_uint4(RV::kFill, RV::kFill, RV::kFill, RV::kFill);
            if (v < v_hi) raw[i] = ld_stream16(p + (int64_t)v * RV::kElems);
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
// The largest of a thread's entries (NaN aside).
template <int DT> __device__ __forceinline__ float pass_max(const uint4 (&raw)[kRowVecs]) {
    using RV = RowVec<DT>;
    if constexpr (DT == MOSAIC_BF16) {   // two entries an instruction
        uint32_t m = raw[0].x;
#pragma unroll
        for (int i = 0; i < kRowVecs; ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[e]));
        }
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    } else {
        float m = RV::get(raw[0], 0);
#pragma unroll
        for (int i = 0; i < kRowVecs; ++i)
#pragma unroll
            for (int e = 0; e < RV::kElems; ++e) m = fmaxf(m, RV::get(raw[i], e));
        return m;
    }
}
// One entry's statistics.
__device__ __forceinline__ SoftStat soft_one(float x, float c) { return {x, exp2_fast(__fmul_rn(__fsub_rn(x, soft_ref(x)), c))}; }
// The thread's statistics of the vectors of one pass, merged into `st`.
template <int DT> __device__ __forceinline__ void soft_pass(uint4 (&raw)[kRowVecs], float c, SoftStat& st) {
    using RV = RowVec<DT>;
    const float m = fmaxf(st.m, pass_max<DT>(raw));
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
// A whole part: its vectors (the first pass's are already in `raw`) and the thread's single element x (-inf: none).
template <int DT>
__device__ __forceinline__ SoftStat soft_part(const RowPart<DT>& part, uint4 (&raw)[kRowVecs], float x, float c) {
    SoftStat st = {-INFINITY, 0.0f};
    soft_pass<DT>(raw, c, st);
    for (int b = part.v_lo + kRowThreads * kRowVecs; b < part.v_hi; b += kRowThreads * kRowVecs) {
        part.load_pass(b, raw);
        soft_pass<DT>(raw, c, st);
    }
    return part.single() >= 0 ? soft_merge(st, soft_one(x, c), c) : st;
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
// The merged statistics of n <= 32 parts, by a whole warp, in every lane.
__device__ __forceinline__ SoftStat soft_all(const SoftStat* part, int n, float c) {
    SoftStat st = {-INFINITY, 0.0f};
    if ((int)(threadIdx.x & 31) < n) st = part[threadIdx.x & 31];
    return soft_warp(st, c);
}
// log sum exp(x / T) of a row, from its statistics (c = log2(e) / T).
__device__ __forceinline__ double soft_lse(SoftStat st, double inv_t) { return (double)soft_ref(st.m) * inv_t + log((double)st.s); }
#endif
}  // namespace mosaic
