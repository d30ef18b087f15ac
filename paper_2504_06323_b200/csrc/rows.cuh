// Rows of logits: how the kernels over a model's output distribution (top logits, distillation) read a row of
// any length, alignment and leading dimension, and the running maximum and sum of a softmax over it.
//
// A row is its whole 16-byte vectors on 16-byte boundaries, one 16-byte load each, and at most a vector's
// worth of single elements on either side of them (an odd vocabulary, a dense matrix whose rows start
// anywhere), which the first threads of the row's first CTA take one each.  Nothing outside the row is read.
// A thread streams over its vectors, kBatch loads in flight, and holds none in registers.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "common.cuh"

namespace mosaic {

constexpr int kThreads = 512;                // threads of a CTA
constexpr int kWarps = kThreads / 32;
constexpr int kBatch = 4;                    // vectors a thread has in flight
constexpr int kRowCtas = 3;                  // CTAs an SM holds
constexpr int kPartVecs = 4096;              // vectors of a row that a CTA takes before the row is shared by more
constexpr int kMaxTop = 1024;      // kept logits per row
constexpr int64_t kMaxRow = 0x7FFFFF00;   // elements of a row: column and vector numbers fit 32 bits with room to spare
constexpr int kMaxCluster = 8;     // CTAs that share one row (the portable cluster size)

// ---------------------------------------------------------------- host side
// CTAs per row: one for every kPartVecs vectors (64 KB), and where the rows alone would leave SMs idle a row is
// spread further, as long as every thread keeps a vector.
inline int row_cluster(int64_t rows, int64_t vectors) {
    int c = 1;
    while (c < kMaxCluster && vectors > (int64_t)c * kPartVecs) c *= 2;
    while (c < kMaxCluster && rows * c < sm_count() && vectors >= (int64_t)2 * c * kThreads) c *= 2;
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

// 2^((x - ref) c) of both.  (x - ref) first, then the factor: near the maximum the difference is exact, so the
// factor's rounding costs next to nothing there; folded into one multiply-add, ref * c would shift every term
// alike, and overflow for logits near the type's ends.
__device__ __forceinline__ Pair soft_pair(float x0, float x1, Pair minus_ref, Pair c) {
    float y0, y1;
    split(mul2(add2(pair_of(x0, x1), minus_ref), c), y0, y1);
    return pair_of(exp2_fast(y0), exp2_fast(y1));
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
    __device__ static __forceinline__ float any(const uint4& v, int e) {   // e not known at compile time
        const uint32_t a = (e & 4) ? v.z : v.x, b = (e & 4) ? v.w : v.y, w = (e & 2) ? b : a;
        return __uint_as_float((e & 1) ? (w & 0xFFFF0000u) : (w << 16));
    }
    __device__ static __forceinline__ Elem bits(const uint4& v, int e) {
        const uint32_t w = (e >> 1) == 0 ? v.x : (e >> 1) == 1 ? v.y : (e >> 1) == 2 ? v.z : v.w;
        return (Elem)((e & 1) ? w >> 16 : w & 0xFFFFu);
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
    __device__ static __forceinline__ float any(const uint4& v, int e) {
        const uint32_t a = (e & 2) ? v.z : v.x, b = (e & 2) ? v.w : v.y;
        return __uint_as_float((e & 1) ? b : a);
    }
    __device__ static __forceinline__ Elem bits(const uint4& v, int e) { return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w; }
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
    __device__ __forceinline__ float at(int col) const { return RV::widen(row[col]); }
    __device__ __forceinline__ const Elem* vec(int v) const { return row + head + (int64_t)v * RV::kElems; }
    // kBatch vectors from v on, a block's stride (T threads) apart, all loads issued before the first is used; -inf where there is none.
    template <int T = kThreads> __device__ __forceinline__ void load(int v, uint4 (&raw)[kBatch]) const {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            raw[i] = make_uint4(RV::kFill, RV::kFill, RV::kFill, RV::kFill);
            if (v + i * T < v_hi) raw[i] = ld_stream16(vec(v + i * T));
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
// Bit e: entry e of the vector is not below `least` (NaN included).
template <int DT> __device__ __forceinline__ uint32_t reach_mask(const uint4& v, float least) {
    using RV = RowVec<DT>;
    uint32_t mask = 0u;
#pragma unroll
    for (int e = 0; e < RV::kElems; ++e) mask |= !(RV::get(v, e) < least) ? 1u << e : 0u;
    return mask;
}
// The largest entry of a batch (NaN aside).
template <int DT> __device__ __forceinline__ float batch_max(const uint4 (&raw)[kBatch]) {
    using RV = RowVec<DT>;
    if constexpr (DT == MOSAIC_BF16) {   // two entries an instruction
        uint32_t m = raw[0].x;
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) asm("max.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(w[e]));
        }
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    } else {
        float m = RV::get(raw[0], 0);
#pragma unroll
        for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int e = 0; e < RV::kElems; ++e) m = fmaxf(m, RV::get(raw[i], e));
        return m;
    }
}
// One entry's statistics.
__device__ __forceinline__ SoftStat soft_one(float x, float c) { return {x, exp2_fast(__fmul_rn(__fsub_rn(x, soft_ref(x)), c))}; }
// A batch's statistics merged into the thread's; `most`: its largest entry.
template <int DT> __device__ __forceinline__ void soft_batch(const uint4 (&raw)[kBatch], float most, float c, SoftStat& st) {
    using RV = RowVec<DT>;
    const float m = fmaxf(st.m, most);
    const float ref = soft_ref(m);
    const Pair minus_ref = pair_of(-ref, -ref), cc = pair_of(c, c);
    Pair sum = pair_of(0.0f, 0.0f);   // the batch's sum first: fewer roundings at the size of the total
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
#pragma unroll
        for (int e = 0; e < RV::kElems; e += 2) sum = add2(sum, soft_pair(RV::get(raw[i], e), RV::get(raw[i], e + 1), minus_ref, cc));
    float s0, s1;
    split(sum, s0, s1);
    st.s = __fadd_rn(__fmul_rn(st.s, soft_scale(st.m, m, c)), __fadd_rn(s0, s1));
    st.m = m;
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
