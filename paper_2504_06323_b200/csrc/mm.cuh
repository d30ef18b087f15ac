// The matrix products of the linear and gated calls on the tensor cores (bf16 in, fp32 sums), the kernel for few tokens,
// and the elementwise passes around them.
//
// One kernel computes all of them as   out[j, i] = sum_c A[i, c] B[j, c]:  the matrix instruction's 128 rows run
// along the CONTIGUOUS dimension of the output, its columns along the rows of the output.  The accumulator of a
// fixed column is then a run of adjacent output elements across the lanes of a warp: the epilogue reads and writes
// 64 adjacent bytes per instruction whatever the alignment, the bias is one register per lane, and few tokens mean
// a narrow instruction instead of one mostly filled with nothing.
//     forward    A = W  (contraction contiguous)   B = X   (contraction contiguous)
//     dX         A = W  (contraction = rows)       B = dZ  (contraction contiguous)
//     dW         A = X  (contraction = rows)       B = dZ  (contraction = rows)
// "Contraction = rows" operands are MN-major for tcgen05.mma; nothing is transposed.
#pragma once
#include <cooperative_groups.h>

#include "checkpoint.cuh"
#include "umma.cuh"

namespace cg = cooperative_groups;

namespace mosaic {
namespace {

constexpr int kMI = 128;               // rows of the matrix instruction: adjacent output elements
constexpr int kMC = 64;                // contraction steps per stage (128 bytes: one swizzle row)
constexpr int kMMaxSplit = 8;          // CTAs (one cluster) that share one tile's contraction
constexpr uint32_t kMBox = 64 * 64 * 2;   // an MN-major box: 64 elements x 64 contraction steps

struct MmArgs {
    int64_t n_i, n_j, n_c;             // extents
    int tiles_i, tiles_j, stages, split;
    int first_pair;                    // >= 0: the tiles are quarters of the pair kernel's tiles from this one on
    int pair_i, pair_j;                // its tiles
    uint16_t* out;
    int64_t ld_out;
    const uint16_t* bias;              // [n_i] or null
    const uint16_t* resid;             // [n_j, n_i] or null
    int64_t ld_resid;
    uint16_t* z;                       // [n_j, n_i] or null: the value before the activation
    int64_t ld_z;
    int act;
    int pairs;                         // out, resid and z (those there are) take two elements a word: 4-byte bases, even ld
    int* status;
};

// What a product is made of:
//   kPlain  out = A B
//   kGate   out = act(A B + bias) * (A2 B + bias2) with z and u, the two before the activation.  A tile's rows are 64 of A and the
//           same 64 of A2: n_i counts output elements, of which a tile of the matrix instruction then has half as many.
//           Two warps hold 32 elements of z and of u, exchange half of their columns through shared memory and make half
//           of the output each; the loads, the instructions and their rate are those of the plain product.
//   kSum    out = A B + A2 B2: one contraction after the other into the same accumulator
//   kTwin   out = A B, out2 = A B2 of the same extents in one launch: the tiles' second half
enum Mode { kPlain = 0, kGate, kSum, kTwin };
struct GateArgs {
    const uint16_t* w;                 // A2, for the kernel that reads it without a tensor map
    int64_t ld_w;
    const uint16_t* bias;              // [n_i] or null
    uint16_t* u;                       // [n_j, n_i] or null
    int64_t ld_u;
    Saved z8, u8;                      // or, in 8 bits, both of them (codes null: not)
};
template <int MODE> struct Second {};
template <> struct Second<kGate> {
    CUtensorMap a;
    GateArgs g;
};
template <> struct Second<kSum> {
    CUtensorMap a, b;
};
template <> struct Second<kTwin> {
    CUtensorMap b;
    uint16_t* out;
    int64_t ld_out;
};

// Two adjacent output elements a word.  A lane holds element i of rows j and j + 1 (lo, hi); after the exchange with its
// neighbour an even lane holds elements i, i + 1 of row j, an odd one i - 1, i of row j + 1.  Its own inverse.
__device__ __forceinline__ uint32_t exchange(uint32_t w, bool odd) {
    const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, w, 1);
    return odd ? __byte_perm(other, w, 0x7632) : __byte_perm(w, other, 0x5410);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return (uint32_t)__bfloat16_as_ushort(p.x) | ((uint32_t)__bfloat16_as_ushort(p.y) << 16);
}

// N accumulator columns of a warp into the output: v[e] belongs to element (i, j + e), e < n; i0 is lane 0's i.
template <int N> __device__ __forceinline__ void epilogue(const MmArgs& a, float (&v)[N], float bias, int64_t i0, int64_t j, int n) {
    const int lane = (int)threadIdx.x & 31;
    const int64_t i = i0 + lane;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = __fadd_rn(v[e], bias);
    if (a.pairs && i0 + 32 <= a.n_i) {   // whole words: half the instructions of the element by element form below
        const bool odd = (lane & 1) != 0;
        const int64_t at = i & ~(int64_t)1, row = j + (lane & 1);
        uint32_t r[N / 2];
        if (a.resid != nullptr) {
            const uint16_t* p = a.resid + row * a.ld_resid + at;
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_resid) r[e / 2] = e + (lane & 1) < n ? *reinterpret_cast<const uint32_t*>(p) : 0u;
        }
        if (a.z != nullptr) {
            uint16_t* p = a.z + row * a.ld_z + at;
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_z) {
                const uint32_t w = exchange(pack2(v[e], v[e + 1]), odd);
                if (e + (lane & 1) < n) *reinterpret_cast<uint32_t*>(p) = w;
            }
        }
        if (a.act != MOSAIC_ACT_NONE) activate_all(v, a.act);
        if (a.resid != nullptr) {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const uint32_t w = exchange(r[e / 2], odd);
                v[e] = __fadd_rn(v[e], __uint_as_float(w << 16));
                v[e + 1] = __fadd_rn(v[e + 1], __uint_as_float(w & 0xFFFF0000u));
            }
        }
        uint16_t* p = a.out + row * a.ld_out + at;
        if (n >= N) {
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_out) *reinterpret_cast<uint32_t*>(p) = exchange(pack2(v[e], v[e + 1]), odd);
        } else {
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_out) {
                const uint32_t w = exchange(pack2(v[e], v[e + 1]), odd);
                if (e + (lane & 1) < n) *reinterpret_cast<uint32_t*>(p) = w;
            }
        }
        return;
    }
    if (i >= a.n_i) return;
    if (a.z != nullptr) {
        uint16_t* p = a.z + j * a.ld_z + i;
#pragma unroll
        for (int e = 0; e < N; ++e, p += a.ld_z)
            if (e < n) *p = f32_to_bf16(v[e]);
    }
    if (a.act != MOSAIC_ACT_NONE) activate_all(v, a.act);
    if (a.resid != nullptr) {
        const uint16_t* p = a.resid + j * a.ld_resid + i;
#pragma unroll
        for (int h = 0; h < N; h += N / 2) {   // half of them on their way before the first is used
            uint16_t r[N / 2];
#pragma unroll
            for (int e = 0; e < N / 2; ++e) {
                r[e] = 0;
                if (h + e < n) asm volatile("ld.global.u16 %0, [%1];" : "=h"(r[e]) : "l"(p));   // volatile: not one by one with the additions
                p += a.ld_resid;
            }
#pragma unroll
            for (int e = 0; e < N / 2; ++e) v[h + e] = __fadd_rn(v[h + e], bf16_to_f32(r[e]));
        }
    }
    uint16_t* p = a.out + j * a.ld_out + i;
#pragma unroll
    for (int e = 0; e < N; ++e, p += a.ld_out)
        if (e < n) *p = f32_to_bf16(v[e]);
}
// 16 accumulator columns of a warp whose lanes hold 32 adjacent channels, two groups, from i0 on, v[at + e] in column (token) e < n:
// the groups in 8 bits, as store_saved would make them of the bf16 values.  Words of two tokens' magnitudes are maximised
// over the group's lanes, each lane ending with the two of one word (so it has their exponents to write); four tokens' codes are
// turned round among four lanes, so that a lane writes four channels of a token.
template <int N> __device__ __forceinline__ void keep16(const Saved& to, const float (&v)[N], int at, int64_t i0, int64_t n_i, int64_t j, int n) {
    const int lane = (int)threadIdx.x & 31, l = lane & 15;
    i0 += lane & 16;                   // the lane's group
    const bool there = i0 + l < n_i;   // behind the last channel rows of zeros, whose sums are NaN where X is not finite
    uint32_t h[8], m[8], any = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        h[k] = there ? pack2(v[at + 2 * k], v[at + 2 * k + 1]) : 0u;
        m[k] = h[k] & 0x7FFF7FFFu;
        any = __vmaxu2(any, m[k]);
    }
    if (max(any & 0xFFFFu, any >> 16) >= kNotFinite) {   // rare
#pragma unroll
        for (int k = 0; k < 8; ++k) m[k] = finite_bits(h[k] & 0xFFFFu) | (finite_bits(h[k] >> 16) << 16);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) m[k] = __vmaxu2(m[k], __shfl_xor_sync(0xFFFFFFFFu, m[k], 8));
#pragma unroll
    for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < o; ++k) {
            const bool upper = (lane & o) != 0;
            const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, upper ? m[k] : m[k + o], o);
            m[k] = __vmaxu2(upper ? m[k + o] : m[k], other);
        }
    const uint32_t E2 = saved_exponent(m[0] & 0xFFFFu) | (saved_exponent(m[0] >> 16) << 16);   // of tokens 2 (l & 7) and the next
    const int64_t group = i0 / kSavedGroup;
    if (l < 8 && i0 < n_i) {
        if (2 * l < n) to.exponents[(j + 2 * l) * to.lde + group] = (uint8_t)E2;
        if (2 * l + 1 < n) to.exponents[(j + 2 * l + 1) * to.lde + group] = (uint8_t)(E2 >> 16);
    }
    constexpr float kRound = 12582912.0f + 128.0f;
#pragma unroll
    for (int t = 0; t < 16; t += 4) {
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t pair = __shfl_sync(0xFFFFFFFFu, E2, (lane & 16) | ((t + e) >> 1)), E = (e & 1) ? pair >> 16 : pair & 0xFFFFu;
            const uint32_t half = (e & 1) ? h[(t + e) >> 1] >> 16 : h[(t + e) >> 1] & 0xFFFFu;
            const float up = __uint_as_float((E >= 6u ? 260u - E : 254u) << 23), more = E >= 6u ? 1.0f : __uint_as_float((133u - E) << 23);
            const float y = fminf(fmaxf(__fmaf_rn(__fmul_rn(__uint_as_float(half << 16), more), up, kRound), kRound - 127.0f), kRound + 127.0f);
            word |= ((half & kNotFinite) == kNotFinite ? 0u : __float_as_uint(y) & 0xFFu) << (8 * e);   // code + 128; 0: not finite
        }
        word ^= 0x80808080u;
        const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, word, 2);
        word = (lane & 2) ? __byte_perm(word, other, 0x3276) : __byte_perm(word, other, 0x5410);
        const uint32_t next = __shfl_xor_sync(0xFFFFFFFFu, word, 1);
        word = (lane & 1) ? __byte_perm(word, next, 0x3715) : __byte_perm(word, next, 0x6240);
        const int token = t + (lane & 3);
        if (token < n && i0 < n_i) *reinterpret_cast<uint32_t*>(to.codes + (j + token) * to.ldc + i0 + (l & 12)) = word;
    }
}

// The same for kGate, by two warps: one holds z of 32 elements from i0 on, the other (`up`) u of the same.  Each keeps what it holds,
// then they exchange halves of the columns through `swap` (kSwap floats of shared memory, theirs alone), and each makes the output
// of a half.  Both warps call with the same columns; `id` is their barrier.
constexpr int kSwap = 2 * 32 * 16;   // 16 columns of either warp
template <int N> __device__ __forceinline__ void gate_epilogue(const MmArgs& a, const GateArgs& g, float (&v)[N], float bias, int64_t i0, int64_t j, int n, bool up,
                                                               float4* swap, int id) {
    const int lane = (int)threadIdx.x & 31;
    const int64_t i = i0 + lane;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = __fadd_rn(v[e], bias);
    const bool odd = (lane & 1) != 0, words = a.pairs && i0 + 32 <= a.n_i;
    uint16_t* kept = up ? g.u : a.z;
    const int64_t ld_kept = up ? g.ld_u : a.ld_z;
    if (kept != nullptr) {
        if (words) {
            uint16_t* p = kept + (j + (lane & 1)) * ld_kept + (i & ~(int64_t)1);
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * ld_kept) {
                const uint32_t w = exchange(pack2(v[e], v[e + 1]), odd);
                if (e + (lane & 1) < n) *reinterpret_cast<uint32_t*>(p) = w;
            }
        } else if (i < a.n_i) {
            uint16_t* p = kept + j * ld_kept + i;
#pragma unroll
            for (int e = 0; e < N; ++e, p += ld_kept)
                if (e < n) *p = f32_to_bf16(v[e]);
        }
    }
    if (g.z8.codes != nullptr && i0 < a.n_i) {
        __syncwarp();
#pragma unroll
        for (int at = 0; at < N; at += 16)
            if (at < n) keep16(up ? g.u8 : g.z8, v, at, i0, a.n_i, j + at, n - at);
    }
    float4 *mine = swap + (up ? kSwap / 8 : 0) + lane, *theirs = swap + (up ? 0 : kSwap / 8) + lane;
    float x[N / 2];                    // this warp's values of the columns that it goes on with
#pragma unroll
    for (int e = 0; e < N / 2; e += 4) {
        mine[e * 8] = up ? make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]) : make_float4(v[N / 2 + e], v[N / 2 + e + 1], v[N / 2 + e + 2], v[N / 2 + e + 3]);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[e + k] = up ? v[N / 2 + e + k] : v[e + k];
    }
    __syncwarp();
    two_warps_meet(id);
    float z[N / 2], u[N / 2];
#pragma unroll
    for (int e = 0; e < N / 2; e += 4) {
        const float4 f = theirs[e * 8];
        const float other[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            z[e + k] = up ? other[k] : x[e + k];
            u[e + k] = up ? x[e + k] : other[k];
        }
    }
    two_warps_meet(id);                // read, before the next columns are written there
    activate_all(z, a.act);
#pragma unroll
    for (int e = 0; e < N / 2; ++e) z[e] = __fmul_rn(z[e], u[e]);
    const int first = up ? N / 2 : 0;  // this warp's first column
    if (words) {
        uint16_t* p = a.out + (j + first + (lane & 1)) * a.ld_out + (i & ~(int64_t)1);
#pragma unroll
        for (int e = 0; e < N / 2; e += 2, p += 2 * a.ld_out) {
            const uint32_t w = exchange(pack2(z[e], z[e + 1]), odd);
            if (first + e + (lane & 1) < n) *reinterpret_cast<uint32_t*>(p) = w;
        }
    } else if (i < a.n_i) {
        uint16_t* p = a.out + (j + first) * a.ld_out + i;
#pragma unroll
        for (int e = 0; e < N / 2; ++e, p += a.ld_out)
            if (first + e < n) *p = f32_to_bf16(z[e]);
    }
}
// Of the 128 lanes of tensor memory, a warp's quarter q: its first output element from the tile's, for kGate whether it holds u.
template <int MODE> __device__ __forceinline__ int quarter_first(int q) { return MODE == kGate ? (q & 1) * 32 : q * 32; }
template <int MODE> __device__ __forceinline__ bool quarter_up(int q) { return MODE == kGate && q >= 2; }
__device__ __forceinline__ int quarter_barrier(int set, int q) { return 1 + set * 2 + (q & 1); }
template <int N> __device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[N]) {
    if constexpr (N == 16) tmem_load16(addr, v);
    else tmem_load32(addr, v);
}
__device__ __forceinline__ void pair_tile(int tile, int tiles_i, int tiles_j, int* ti, int* tj);
// A tile's arguments: the kernel's own (read where they lie: a copy costs registers), but for the twin's output.
template <int MODE> __device__ __forceinline__ decltype(auto) twin_args(const MmArgs& args, const Second<MODE>& second, bool twin) {
    if constexpr (MODE == kTwin) {
        MmArgs a = args;
        if (twin) {
            a.out = second.out;
            a.ld_out = second.ld_out;
        }
        return a;
    } else {
        return (args);
    }
}
// The bias of a lane's accumulator row; i0 is the first element of the warp, quarter q of the lanes.
template <int MODE> __device__ __forceinline__ float lane_bias(const MmArgs& a, const Second<MODE>& second, int64_t i0, int q) {
    const uint16_t* bias = a.bias;
    if constexpr (MODE == kGate) {
        if (quarter_up<MODE>(q)) bias = second.g.bias;
    }
    const int64_t i = i0 + ((int)threadIdx.x & 31);
    return bias != nullptr && i < a.n_i ? bf16_to_f32(bias[i]) : 0.0f;
}
// The map of B (and for kSum of A) that a step reads.
template <int MODE> __device__ __forceinline__ const CUtensorMap* map_a(const CUtensorMap& a_map, const Second<MODE>& second, bool other) {
    if constexpr (MODE == kSum) return other ? &second.a : &a_map;
    return &a_map;
}
template <int MODE> __device__ __forceinline__ const CUtensorMap* map_b(const CUtensorMap& b_map, const Second<MODE>& second, bool other) {
    if constexpr (MODE == kSum || MODE == kTwin) return other ? &second.b : &b_map;
    return &b_map;
}
template <int MODE> __device__ __forceinline__ void prefetch_second(const Second<MODE>& second) {
    if constexpr (MODE == kGate || MODE == kSum) prefetch_map(&second.a);
    if constexpr (MODE == kSum || MODE == kTwin) prefetch_map(&second.b);
}
// Four adjacent elements, or the first n of them.
__device__ __forceinline__ void store4(uint16_t* p, const float (&y)[4], bool words, int64_t n) {
    if (words) {
        reinterpret_cast<uint32_t*>(p)[0] = pack2(y[0], y[1]);
        reinterpret_cast<uint32_t*>(p)[1] = pack2(y[2], y[3]);
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h)
            if (h < n) p[h] = f32_to_bf16(y[h]);
    }
}

constexpr int kGateRows = kMI / 2;   // rows of A, then of A2, in kGate's tiles
constexpr uint32_t kGateBox = kGateRows * kMC * 2;
template <int MODE> constexpr int kTileI = MODE == kGate ? kMI / 2 : kMI;   // output elements of a tile's 128 rows
constexpr int kMSub = 2;     // 64 contraction steps each a stage: eight instructions a barrier
constexpr int kMRoles = 2;   // loader, MMA issue; then the epilogue: four warps (a quarter of tensor memory's lanes each), eight for wide tiles
__host__ __device__ constexpr int mm_warps(int bn) { return bn >= 256 ? 16 : bn >= 64 ? 8 : 4; }
__host__ __device__ constexpr int mm_threads(int bn) { return 32 * (kMRoles + mm_warps(bn)); }

// A complete accumulator of kMI rows and BN columns, n_cols of them of the output: into the output, or, of a contraction that
// `split` CTAs share, into the shared memory of the CTAs that add it up, each `per` columns.  By warps kMRoles on, SETS of them
// a quarter of tensor memory's lanes, which take chunks in turn.
template <int BN, int MODE, int SETS>
__device__ __forceinline__ void tile_out(const MmArgs& a, const Second<MODE>& second, uint32_t tmem, float* part, int per, int rank, int split, int n_cols,
                                         int64_t i0, int64_t j0) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, q = warp & 3;
    constexpr int kChunk = BN < 32 ? 16 : 32;   // warps of a quarter take chunks in turn
    const int set = (warp - kMRoles) >> 2;
    const int64_t iw = i0 + quarter_first<MODE>(q);
    const float bias = lane_bias(a, second, iw, q);
#pragma unroll 1
    for (int c0 = set * kChunk; c0 < n_cols; c0 += SETS * kChunk) {
        float v[kChunk];
        tmem_load<kChunk>(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c0, v);
        if (split > 1) {
            int owner = c0 / per, at = c0 - owner * per;
            uint32_t to = cluster_addr(part + ((size_t)rank * per + at) * kMI + q * 32 + lane, owner);
#pragma unroll
            for (int e = 0; e < kChunk; ++e) {
                if (c0 + e < n_cols) store_remote(to, v[e]);
                to += kMI * 4;
                if (++at == per) {
                    at = 0;
                    ++owner;
                    to = cluster_addr(part + (size_t)rank * per * kMI + q * 32 + lane, owner < split ? owner : 0);
                }
            }
        } else {
            if constexpr (MODE == kGate)   // the stages are free, and no partial sums come
                gate_epilogue<kChunk>(a, second.g, v, bias, iw, j0 + c0, n_cols - c0, quarter_up<MODE>(q),
                                      reinterpret_cast<float4*>(part) + (set * 2 + (q & 1)) * (kSwap / 4), quarter_barrier(set, q));
            else epilogue<kChunk>(a, v, bias, iw, j0 + c0, n_cols - c0);
            __syncwarp();
        }
    }
}
// Whether a warp's accumulator is there (`done`), and for kGate that of the warp beside it: they meet within the epilogue.
template <int MODE> __device__ __forceinline__ bool tile_done(bool done) {
    if constexpr (MODE == kGate) {
        const int warp = threadIdx.x >> 5;
        __syncwarp();
        if (warp >= kMRoles) done = two_warps_agree(quarter_barrier((warp - kMRoles) >> 2, warp & 3), done);
    }
    return done;
}

// A group of 16 channels in 8 bits by four adjacent lanes, four channels each from oi on (all four lanes are there, or none).
__device__ __forceinline__ void keep4(const Saved& to, const float (&x)[4], int64_t oi, int64_t oj, int64_t n_i) {
    const int lane = (int)threadIdx.x & 31;
    const uint32_t four = 0xFu << (lane & 28);
    uint32_t half[4], largest = 0;
#pragma unroll
    for (int h = 0; h < 4; ++h) {
        half[h] = oi + h < n_i ? f32_to_bf16(x[h]) : 0u;
        largest = max(largest, finite_bits(half[h]));
    }
    largest = max(largest, __shfl_xor_sync(four, largest, 1));
    largest = max(largest, __shfl_xor_sync(four, largest, 2));
    if (oi / kSavedGroup * kSavedGroup >= n_i) return;   // the group is not of the matrix
    const uint32_t E = saved_exponent(largest), w[4] = {half[0] | (half[1] << 16), half[2] | (half[3] << 16), 0u, 0u};
    const bool finite = max(max(half[0] & 0x7FFFu, half[1] & 0x7FFFu), max(half[2] & 0x7FFFu, half[3] & 0x7FFFu)) < kNotFinite;
    *reinterpret_cast<uint32_t*>(to.codes + oj * to.ldc + oi) = saved_codes8(w, E, finite).x;
    if ((oi & (kSavedGroup - 1)) == 0) to.exponents[oj * to.lde + oi / kSavedGroup] = (uint8_t)E;
}

// The sum of the CTAs' parts of this CTA's columns, and its epilogue.  Between it and tile_out the CTAs arrive at their barrier.
template <int MODE, int THREADS>
__device__ __forceinline__ void tile_join(const MmArgs& a, const Second<MODE>& second, const float* part, int per, int rank, int split, int n_cols, int64_t i0,
                                          int64_t j0) {
    if constexpr (MODE == kGate) {
        // Four adjacent elements a thread and turn, from the partial sums of both matrices.
        __syncwarp();
        cluster_wait();
        const int mine = n_cols - rank * per < per ? n_cols - rank * per : per;
        for (int e = (int)threadIdx.x; e < mine * (kMI / 8); e += THREADS) {
            const int col = e / (kMI / 8), quad = e % (kMI / 8);   // 16 quads of either matrix a column
            const float4* from = reinterpret_cast<const float4*>(part) + col * (kMI / 4) + quad;
            float z[4] = {}, u[4] = {};
            for (int p = 0; p < split; ++p) {   // in the CTAs' order
                const float4 zp = from[p * per * (kMI / 4)], up = from[p * per * (kMI / 4) + kMI / 8];
                z[0] = __fadd_rn(z[0], zp.x);
                z[1] = __fadd_rn(z[1], zp.y);
                z[2] = __fadd_rn(z[2], zp.z);
                z[3] = __fadd_rn(z[3], zp.w);
                u[0] = __fadd_rn(u[0], up.x);
                u[1] = __fadd_rn(u[1], up.y);
                u[2] = __fadd_rn(u[2], up.z);
                u[3] = __fadd_rn(u[3], up.w);
            }
            const int64_t oi = i0 + 4 * quad, oj = j0 + rank * per + col;
            const bool words = a.pairs && oi + 4 <= a.n_i;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                if (oi + h >= a.n_i) break;
                if (a.bias != nullptr) z[h] = __fadd_rn(z[h], bf16_to_f32(a.bias[oi + h]));
                if (second.g.bias != nullptr) u[h] = __fadd_rn(u[h], bf16_to_f32(second.g.bias[oi + h]));
            }
            if (second.g.z8.codes != nullptr) {   // four lanes hold a group
                keep4(second.g.z8, z, oi, oj, a.n_i);
                keep4(second.g.u8, u, oi, oj, a.n_i);
            }
            if (a.z != nullptr) store4(a.z + oj * a.ld_z + oi, z, words, a.n_i - oi);
            if (second.g.u != nullptr) store4(second.g.u + oj * second.g.ld_u + oi, u, words, a.n_i - oi);
            activate_all(z, a.act);
#pragma unroll
            for (int h = 0; h < 4; ++h) z[h] = __fmul_rn(z[h], u[h]);
            store4(a.out + oj * a.ld_out + oi, z, words, a.n_i - oi);
        }
        return;
    }
    // Four adjacent elements a thread and turn; the residual's are on their way while the partial sums come in.
    constexpr int kTurns = 4;
    const int mine = n_cols - rank * per < per ? n_cols - rank * per : per, quads = mine > 0 ? mine * (kMI / 4) : 0;
    uint32_t r[kTurns][2];
    const auto fetch = [&](int e0) {
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int e = e0 + u * THREADS;
            const int64_t oi = i0 + 4 * (e % (kMI / 4)), oj = j0 + rank * per + e / (kMI / 4);
            r[u][0] = r[u][1] = 0;
            if (a.resid == nullptr || e >= quads || oi >= a.n_i) continue;
            const uint16_t* p = a.resid + oj * a.ld_resid + oi;
            if (a.pairs && oi + 4 <= a.n_i) {
                r[u][0] = reinterpret_cast<const uint32_t*>(p)[0];
                r[u][1] = reinterpret_cast<const uint32_t*>(p)[1];
            } else {
                r[u][0] = p[0] | (oi + 1 < a.n_i ? (uint32_t)p[1] << 16 : 0u);
                r[u][1] = (oi + 2 < a.n_i ? (uint32_t)p[2] : 0u) | (oi + 3 < a.n_i ? (uint32_t)p[3] << 16 : 0u);
            }
        }
    };
    fetch((int)threadIdx.x);
    __syncwarp();
    cluster_wait();
    for (int e0 = (int)threadIdx.x; e0 < quads; e0 += kTurns * THREADS) {
        if (e0 != (int)threadIdx.x) fetch(e0);
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            const int e = e0 + u * THREADS;
            if (e >= quads) break;
            const float4* from = reinterpret_cast<const float4*>(part) + e;
            const float4 first = *from;
            float y[4] = {first.x, first.y, first.z, first.w};
            for (int p = 1; p < split; ++p) {   // in the CTAs' order
                const float4 more = from[p * per * (kMI / 4)];
                y[0] = __fadd_rn(y[0], more.x);
                y[1] = __fadd_rn(y[1], more.y);
                y[2] = __fadd_rn(y[2], more.z);
                y[3] = __fadd_rn(y[3], more.w);
            }
            const int64_t oi = i0 + 4 * (e % (kMI / 4)), oj = j0 + rank * per + e / (kMI / 4);
            const bool words = a.pairs && oi + 4 <= a.n_i;
            if (a.bias != nullptr) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    if (oi + h < a.n_i) y[h] = __fadd_rn(y[h], bf16_to_f32(a.bias[oi + h]));
            }
            if (a.z != nullptr) store4(a.z + oj * a.ld_z + oi, y, words, a.n_i - oi);
            activate_all(y, a.act);
            if (a.resid != nullptr) {
#pragma unroll
                for (int h = 0; h < 4; ++h)
                    y[h] = __fadd_rn(y[h], __uint_as_float((h & 1) ? r[u][h / 2] & 0xFFFF0000u : r[u][h / 2] << 16));
            }
            store4(a.out + oj * a.ld_out + oi, y, words, a.n_i - oi);
        }
    }
}

// One output tile of kMI x BN per cluster; its contraction is split over the cluster's CTAs.  Each of them adds up and writes
// an equal share of the tile's columns: the others push their partial sums of it into its shared memory (the stages, free
// by then), and it adds them in the CTAs' order.  Bound by the loads of a tile's operands into one SM (about 110 GB/s an
// SM for wide tiles) or, with few tokens, by the weights' stream: 37 tokens, 4096 outputs from 8807, 17 us against
// 11.2 of the weights alone; 512 tokens, 4096 from 4096, 19 us.  One CTA an SM (its stages fill shared memory), so a CTA
// never waits for tensor memory that another one of this kernel holds.
template <bool A_MN, bool B_MN, int BN, int MODE>
__global__ void __launch_bounds__(mm_threads(BN)) mm_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                                                       const __grid_constant__ MmArgs args, const __grid_constant__ Second<MODE> second) {
    static_assert(MODE != kGate || (!A_MN && !B_MN), "the gated product is the forward one");
    constexpr uint32_t kABytes = kMI * kMC * 2, kBBytes = BN * kMC * 2, kHalf = kABytes + kBBytes, kStage = kMSub * kHalf;
    constexpr uint32_t kCols = BN < 32 ? 32 : BN;
    constexpr uint32_t kDesc = instr_desc(A_MN, B_MN, kMI, BN);
    extern __shared__ unsigned char mm_smem_raw[];
    __shared__ uint64_t full[8], empty[8], acc_full;
    __shared__ uint32_t tmem_slot;
    __shared__ int err_word;
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(mm_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    volatile int* err = &err_word;
    const int split = args.split, rank = (int)(blockIdx.x % (unsigned)split);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = (int)(blockIdx.x / (unsigned)split);
    int64_t i0 = (int64_t)(tile % args.tiles_i) * kTileI<MODE>, j0 = (int64_t)(tile / args.tiles_i) * BN;
    bool twin = false;
    if (BN == 128 && args.first_pair >= 0) {   // what is left over of the pair kernel's tiles
        int ti, tj;
        pair_tile(args.first_pair + tile / 4, args.pair_i, MODE == kTwin ? 2 * args.pair_j : args.pair_j, &ti, &tj);
        if (MODE == kTwin && tj >= args.pair_j) {
            twin = true;
            tj -= args.pair_j;
        }
        i0 = (int64_t)ti * (2 * kTileI<MODE>) + (tile & 1) * kTileI<MODE>;
        j0 = (int64_t)tj * 256 + ((tile >> 1) & 1) * 128;
    } else if (MODE == kTwin && tile / args.tiles_i >= args.tiles_j) {
        twin = true;
        j0 -= (int64_t)args.tiles_j * BN;
    }
    const auto& a = twin_args(args, second, twin);
    const int64_t part_steps = (a.n_c + kMSub * kMC - 1) / (kMSub * kMC), steps = MODE == kSum ? 2 * part_steps : part_steps;
    const int s0 = (int)(steps * rank / split), s1 = (int)(steps * (rank + 1) / split);   // split <= steps: never empty

    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        prefetch_second(second);
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1u);
            mbar_init(&empty[s], 1u);
        }
        mbar_init(&acc_full, 1u);
        *err = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    uint32_t issued = 0;
    allow_next_kernel();   // not before this CTA has its tensor memory: the next kernel's CTAs wait for it with theirs in hand
    await_previous_kernel();

    if (warp == 0) {
        if (lane == 0) {
            for (int s = s0; s < s1; ++s) {
                const uint32_t it = (uint32_t)(s - s0), slot = it % (uint32_t)a.stages, ph = (it / (uint32_t)a.stages) & 1u;
                if (!mbar_wait(&empty[slot], ph ^ 1u, err)) break;
                mbar_expect_tx(&full[slot], kStage);
                const bool later = MODE == kSum && s >= (int)part_steps;
                const CUtensorMap *am = map_a(a_map, second, later), *bm = map_b(b_map, second, MODE == kSum ? later : twin);
#pragma unroll
                for (int h = 0; h < kMSub; ++h) {
                    unsigned char* sa = ring + (size_t)slot * kStage + (size_t)h * kHalf;
                    unsigned char* sb = sa + kABytes;
                    const int c = ((later ? s - (int)part_steps : s) * kMSub + h) * kMC;
                    if constexpr (MODE == kGate) {
                        tma_load_box(sa, am, &full[slot], c, (int)i0);
                        tma_load_box(sa + kGateBox, &second.a, &full[slot], c, (int)i0);
                    } else if (A_MN) {
#pragma unroll
                        for (int b = 0; b < kMI / 64; ++b) tma_load_box(sa + (size_t)b * kMBox, am, &full[slot], (int)i0 + b * 64, c);
                    } else {
                        tma_load_box(sa, am, &full[slot], c, (int)i0);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int b = 0; b < BN / 64; ++b) tma_load_box(sb + (size_t)b * kMBox, bm, &full[slot], (int)j0 + b * 64, c);
                    } else {
                        tma_load_box(sb, bm, &full[slot], c, (int)j0);
                    }
                }
                issued = it + 1u;
            }
        }
    } else if (warp == 1) {
        // all lanes alike, one of them issues (umma.cuh, elect_one)
        const bool issue = elect_one();
        const uint32_t acc = __shfl_sync(0xFFFFFFFFu, tmem, 0), ring0 = __shfl_sync(0xFFFFFFFFu, smem_u32(ring), 0);
        bool ok = true;
        uint32_t slot = 0, ph = 0;
        for (int s = s0; s < s1; ++s) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&full[slot], ph, err));
            if (!ok) break;
            tc_fence_after();
            const uint32_t stage = ring0 + slot * kStage;
            if (issue) {
#pragma unroll
                for (int k = 0; k < kMSub * kMC / 16; ++k) {
                    // 16 contraction steps further: 16 swizzle rows (MN-major) or 32 bytes along one (K-major)
                    const uint32_t sa = stage + (uint32_t)(k / (kMC / 16)) * kHalf, sb = sa + kABytes, kk = (uint32_t)(k % (kMC / 16));
                    const uint64_t da = operand_desc(sa + kk * (A_MN ? 2048u : 32u), A_MN ? kMBox : 16u);
                    const uint64_t db = operand_desc(sb + kk * (B_MN ? 2048u : 32u), B_MN ? kMBox : 16u);
                    umma_bf16(acc, da, db, kDesc, (s > s0 || k > 0) ? 1u : 0u);
                }
                umma_commit(&empty[slot]);
            }
            __syncwarp();
            if (++slot == (uint32_t)a.stages) {
                slot = 0;
                ph ^= 1u;
            }
        }
        if (ok && issue) umma_commit(&acc_full);
    }
    __syncwarp();
    const bool done = tile_done<MODE>(warp >= kMRoles && mbar_wait(&acc_full, 0u, err));
    tc_fence_after();
    const int n_cols = (int)(a.n_j - j0 < BN ? (a.n_j > j0 ? a.n_j - j0 : 0) : BN);
    const int per = (n_cols + split - 1) / split;   // columns of the tile that a CTA of the cluster adds up and writes
    float* part = reinterpret_cast<float*>(ring);   // [split][per][kMI]: the cluster's partial sums of this CTA's columns
    if (split > 1) {
        // Every CTA's accumulator is complete, so its loads have been consumed, before its stages take partial sums.
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (done) tile_out<BN, MODE, mm_warps(BN) / 4>(a, second, tmem, part, per, rank, split, n_cols, i0, j0);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
    }
    if (threadIdx.x == 0 && *err != 0) {
        // a role gave up: let the loads of the last stages land before shared memory is reused or left (bounded)
        for (uint32_t back = 1; back <= (uint32_t)a.stages && back <= issued; ++back) {
            const uint32_t it = issued - back, slot = it % (uint32_t)a.stages, ph = (it / (uint32_t)a.stages) & 1u;
            const long long t0 = clock64();
            while (!mbar_try_wait(&full[slot], ph) && clock64() - t0 < kWaitCycles) {
            }
        }
        if (a.status != nullptr) atomicExch(a.status, 1);
    }
    if (split > 1) {
        __syncwarp();
        cluster_arrive();
        tile_join<MODE, mm_threads(BN)>(a, second, part, per, rank, split, n_cols, i0, j0);
    }
}

// ---------------------------------------------------------------- large products
// Two CTAs (a cluster, two SMs) share each matrix instruction: 256 x 256 output elements, each CTA holding its half
// of both operands in shared memory (64 KB a stage for 256 x 256 x 128 products: half of what a CTA alone would have
// to load for the same work) and 128 x 256 of the accumulator in its tensor memory, twice: the epilogue of a tile
// runs under the products of the next.  Persistent: a pair takes tile after tile.  The tiles go band by band
// (kPBand tiles of output rows), so that the tiles in flight share operands in L2.  Bound by the tensor pipe, 86 % busy at
// 14336 gated outputs from 4096 and 2048 tokens with Z and U (324 us, of which 289 are the flop at the measured peak; the plain
// product of as many outputs 320).
constexpr int kPTile = 256, kPHalf = 128;
constexpr int kPSub = 2;   // 64 contraction steps each: eight instructions a barrier (with four, 1377 instead of 1505 Tflop/s at 4096 x 13824 x 5120)
constexpr int kPStages = 3;
constexpr uint32_t kPOperand = kPHalf * kMC * 2, kPStage = kPSub * 2 * kPOperand;
constexpr int kPEpiWarps = 16;   // four per quarter of the lanes
constexpr int kPThreads = 64 + 32 * kPEpiWarps;
constexpr int kPBand = 8;
template <int MODE> constexpr size_t kPSmem = (size_t)kPStages * kPStage + 1024 + (MODE == kGate ? kPEpiWarps / 2 * kSwap * 4 : 0);

__device__ __forceinline__ void pair_tile(int tile, int tiles_i, int tiles_j, int* ti, int* tj) {
    const int band = tile / (kPBand * tiles_i), in = tile - band * kPBand * tiles_i;
    const int width = tiles_j - band * kPBand < kPBand ? tiles_j - band * kPBand : kPBand;
    *ti = in / width;
    *tj = band * kPBand + in % width;
}

template <bool A_MN, bool B_MN, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPThreads, 1)
    mm_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ MmArgs a,
                   const __grid_constant__ Second<MODE> second, int tiles) {
    static_assert(MODE != kGate || (!A_MN && !B_MN), "the gated product is the forward one");
    constexpr int kOwn = kTileI<MODE>;   // output elements of this CTA's half of a tile
    constexpr uint32_t kDesc = instr_desc(A_MN, B_MN, kPTile, kPTile);
    extern __shared__ unsigned char pair_smem_raw[];
    __shared__ uint64_t full[kPStages], empty[kPStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int err_word;
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(pair_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    volatile int* err = &err_word;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
    const int part_steps = (int)((a.n_c + kPSub * kMC - 1) / (kPSub * kMC)), steps = MODE == kSum ? 2 * part_steps : part_steps;
    const int all_j = MODE == kTwin ? 2 * a.tiles_j : a.tiles_j;

    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        prefetch_second(second);
        for (int s = 0; s < kPStages; ++s) {
            mbar_init(&full[s], 1u);    // first CTA's: both CTAs' loads of a stage have landed
            mbar_init(&empty[s], 1u);   // the products reading a stage have completed
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1u);
            mbar_init(&acc_empty[b], 2u * kPEpiWarps);   // first CTA's: both epilogues have read the accumulator
        }
        *err = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    cluster.sync();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    uint32_t issued = 0;
    allow_next_kernel();   // not before this CTA has its tensor memory: the next kernel's CTAs wait for it with theirs in hand
    await_previous_kernel();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int tile = pair; tile < tiles && ok; tile += pairs) {
                int ti, tj;
                pair_tile(tile, a.tiles_i, all_j, &ti, &tj);
                const bool twin = MODE == kTwin && tj >= a.tiles_j;
                const int i0 = ti * (2 * kOwn) + rank * kOwn, j0 = (twin ? tj - a.tiles_j : tj) * kPTile + rank * kPHalf;
                for (int s = 0; s < steps; ++s, ++it) {
                    const uint32_t slot = it % kPStages, ph = (it / kPStages) & 1u;
                    if (!mbar_wait(&empty[slot], ph ^ 1u, err)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_expect_tx(&full[slot], 2u * kPStage);
                    const uint32_t bar = cluster_addr(&full[slot], 0u);
                    const bool later = MODE == kSum && s >= part_steps;
                    const CUtensorMap *am = map_a(a_map, second, later), *bm = map_b(b_map, second, MODE == kSum ? later : twin);
#pragma unroll
                    for (int h = 0; h < kPSub; ++h) {
                        unsigned char* sa = ring + (size_t)slot * kPStage + (size_t)h * 2u * kPOperand;
                        unsigned char* sb = sa + kPOperand;
                        const int c = ((later ? s - part_steps : s) * kPSub + h) * kMC;
                        if constexpr (MODE == kGate) {
                            tma_load_box_pair(sa, am, bar, c, i0);
                            tma_load_box_pair(sa + kGateBox, &second.a, bar, c, i0);
                        } else if (A_MN) {
                            tma_load_box_pair(sa, am, bar, i0, c);
                            tma_load_box_pair(sa + kMBox, am, bar, i0 + 64, c);
                        } else {
                            tma_load_box_pair(sa, am, bar, c, i0);
                        }
                        if (B_MN) {
                            tma_load_box_pair(sb, bm, bar, j0, c);
                            tma_load_box_pair(sb + kMBox, bm, bar, j0 + 64, c);
                        } else {
                            tma_load_box_pair(sb, bm, bar, c, j0);
                        }
                    }
                }
            }
            issued = it;
        }
    } else if (warp == 1) {
        if (rank == 0) {   // all lanes alike, one of them issues
            const bool issue = elect_one();
            const uint32_t acc = __shfl_sync(0xFFFFFFFFu, tmem, 0), ring0 = __shfl_sync(0xFFFFFFFFu, smem_u32(ring), 0);
            uint32_t slot = 0, ph = 0, n = 0;
            bool ok = true;
            for (int tile = pair; tile < tiles && ok; tile += pairs, ++n) {
                const uint32_t buf = n & 1u;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(&acc_empty[buf], ((n >> 1) & 1u) ^ 1u, err));
                if (!ok) break;
                tc_fence_after();
                for (int s = 0; s < steps; ++s) {
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(&full[slot], ph, err));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t stage = ring0 + slot * kPStage;
                    if (issue) {
#pragma unroll
                        for (int k = 0; k < kPSub * kMC / 16; ++k) {
                            const uint32_t sa = stage + (uint32_t)(k / (kMC / 16)) * 2u * kPOperand, sb = sa + kPOperand, kk = (uint32_t)(k % (kMC / 16));
                            const uint64_t da = operand_desc(sa + kk * (A_MN ? 2048u : 32u), A_MN ? kMBox : 16u);
                            const uint64_t db = operand_desc(sb + kk * (B_MN ? 2048u : 32u), B_MN ? kMBox : 16u);
                            umma_bf16_pair(acc + buf * 256u, da, db, kDesc, (s > 0 || k > 0) ? 1u : 0u);
                        }
                        umma_commit_pair(&empty[slot]);
                    }
                    __syncwarp();
                    if (++slot == (uint32_t)kPStages) {
                        slot = 0;
                        ph ^= 1u;
                    }
                }
                if (ok && issue) umma_commit_pair(&acc_full[buf]);
                __syncwarp();
            }
        }
    } else {
        const int q = warp & 3, set = (warp - 2) >> 2;   // quarter of the lanes, quarter of the columns
        uint32_t n = 0;
        for (int tile = pair; tile < tiles; tile += pairs, ++n) {
            int ti, tj;
            pair_tile(tile, a.tiles_i, all_j, &ti, &tj);
            const bool twin = MODE == kTwin && tj >= a.tiles_j;
            if (twin) tj -= a.tiles_j;
            const auto& o = twin_args(a, second, twin);
            const uint32_t buf = n & 1u;
            const int64_t i0 = (int64_t)ti * (2 * kOwn) + rank * kOwn + quarter_first<MODE>(q), j0 = (int64_t)tj * kPTile;
            const int n_cols = (int)(a.n_j - j0 < kPTile ? a.n_j - j0 : kPTile);
            const float bias = lane_bias(a, second, i0, q);
            if (!tile_done<MODE>(mbar_wait(&acc_full[buf], (n >> 1) & 1u, err))) break;
            tc_fence_after();
#pragma unroll 1
            for (int c0 = set * 64; c0 < set * 64 + 64 && c0 < n_cols; c0 += 32) {
                float v[32];
                tmem_load32(tmem + ((uint32_t)(q * 32) << 16) + buf * 256u + (uint32_t)c0, v);
                if constexpr (MODE == kGate)
                    gate_epilogue<32>(o, second.g, v, bias, i0, j0 + c0, n_cols - c0, quarter_up<MODE>(q),
                                      reinterpret_cast<float4*>(ring + kPStages * kPStage) + (set * 2 + (q & 1)) * (kSwap / 4), quarter_barrier(set, q));
                else epilogue<32>(o, v, bias, i0, j0 + c0, n_cols - c0);
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(cluster_addr(&acc_empty[buf], 0u));
        }
    }
    __syncwarp();
    tc_fence_before();
    cluster.sync();   // all products and reads of both CTAs are done, or a wait ran out and every role has left
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (threadIdx.x == 0) {
        const bool failed = *err != 0 || *cluster.map_shared_rank(&err_word, rank ^ 1) != 0;
        if (failed && rank == 0) {   // let both CTAs' last loads land before shared memory is left (bounded)
            for (uint32_t back = 1; back <= (uint32_t)kPStages && back <= issued; ++back) {
                const uint32_t it = issued - back, slot = it % kPStages, ph = (it / kPStages) & 1u;
                const long long t0 = clock64();
                while (!mbar_try_wait(&full[slot], ph) && clock64() - t0 < kWaitCycles) {
                }
            }
        }
        if (failed && a.status != nullptr) atomicExch(a.status, 1);
    }
    cluster.sync();   // the error words have been read, the loads have landed
}

// Eight elements of a row from c on; zeros past the last column, which nothing is read of.  Ordinary loads here and in the
// kernels below, no read-only ones (nor __restrict__, which lets the compiler make them so): they may start while the
// kernel that writes what they read still runs, and nothing orders read-only loads behind the wait for it.
template <bool VEC> __device__ __forceinline__ void load8(const uint16_t* row, int64_t c, int64_t cols, uint32_t (&w)[4]) {
    if (VEC) {   // rows on 16-byte boundaries
        if (c + 8 <= cols) {
            const uint4 v = ld_stream16(row + c);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = c + 2 * e < cols ? row[c + 2 * e] : 0u, hi = c + 2 * e + 1 < cols ? row[c + 2 * e + 1] : 0u;
        w[e] = lo | (hi << 16);
    }
}

// ---------------------------------------------------------------- few tokens
// A decoding step's one or two tokens (up to kFewTokens where rows are not aligned): the weights are read once for next
// to no arithmetic, so what counts is that they stream.  A CTA takes kFewRows weight rows and a quarter to an eighth of the contraction per warp; a lane
// multiplies 16 bytes of each row (VEC: rows on 16-byte boundaries; else element by element, any alignment) with the
// tokens' values from L1.  fp32 sums: per lane in order, over the lanes by a butterfly, over the warps in their order.
// Bound by memory; no shared-memory ring, tensor memory or cluster to set up.
// 11008 outputs from 4096, one token: 16.3 us, 5.5 TB/s, against 19.3 us on the tensor cores; three tokens 23.7 against
// 19.2, so from there on only rows that TMA cannot read come here (46 us at four; copying them first costs more).
constexpr int kFewTokens = 4, kFewVector = 2, kFewRows = 4, kFewWarps = 8;
// GATE: half of a CTA's weight rows are the second matrix's.
template <int M, bool VEC, bool GATE>
__global__ void __launch_bounds__(32 * kFewWarps, VEC && M == 1 ? 5 : M <= 2 ? 4 : 3) few_kernel(const uint16_t* X, int64_t ldx, const uint16_t* W, int64_t ldw,
                                                             const __grid_constant__ MmArgs a, const __grid_constant__ GateArgs g) {
    constexpr int kOutputs = GATE ? kFewRows / 2 : kFewRows;
    __shared__ float part[kFewWarps][kFewRows][M];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t o0 = (int64_t)blockIdx.x * kOutputs;
    float acc[kFewRows][M] = {};
    await_previous_kernel();
    const uint16_t* w[kFewRows];
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) {
        const int64_t o = o0 + r % kOutputs, at = o < a.n_i ? o : o0;   // past the end: the first row again, not stored
        w[r] = r < kOutputs ? W + at * ldw : g.w + at * g.ld_w;
    }
    if (VEC) {
        // chunks of 256 contraction steps, dealt to the warps in turn; even and odd steps are summed apart
        Pair two[kFewRows][M];
#pragma unroll
        for (int r = 0; r < kFewRows; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) two[r][m] = pair_of(0.0f, 0.0f);
#pragma unroll 1
        for (int64_t c = warp * 256 + lane * 8; c < a.n_c; c += kFewWarps * 256) {
            uint32_t x[M][4], y[kFewRows][4];
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) load8<true>(w[r], c, a.n_c, y[r]);
#pragma unroll
            for (int m = 0; m < M; ++m) load8<true>(X + m * ldx, c, a.n_c, x[m]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                Pair xe[M];
#pragma unroll
                for (int m = 0; m < M; ++m) xe[m] = widen2(x[m][e]);
#pragma unroll
                for (int r = 0; r < kFewRows; ++r) {
                    const Pair ye = widen2(y[r][e]);
#pragma unroll
                    for (int m = 0; m < M; ++m) two[r][m] = fma2(ye, xe[m], two[r][m]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kFewRows; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) {
                float lo, hi;
                split(two[r][m], lo, hi);
                acc[r][m] = __fadd_rn(lo, hi);
            }
    } else {
#pragma unroll 8
        for (int64_t c = warp * 32 + lane; c < a.n_c; c += kFewWarps * 32) {
            float x[M];
#pragma unroll
            for (int m = 0; m < M; ++m) x[m] = bf16_to_f32(X[m * ldx + c]);
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) {
                const float y = bf16_to_f32(w[r][c]);
#pragma unroll
                for (int m = 0; m < M; ++m) acc[r][m] = __fmaf_rn(y, x[m], acc[r][m]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float v = acc[r][m];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
            if (lane == 0) part[warp][r][m] = v;
        }
    __syncthreads();
    if (threadIdx.x >= kOutputs * M) return;
    const int r = threadIdx.x % kOutputs, m = threadIdx.x / kOutputs;
    const int64_t i = o0 + r;
    if (i >= a.n_i) return;
    float v = 0.0f;
    for (int k = 0; k < kFewWarps; ++k) v = __fadd_rn(v, part[k][r][m]);
    v = __fadd_rn(v, a.bias != nullptr ? bf16_to_f32(a.bias[i]) : 0.0f);
    if (a.z != nullptr) a.z[m * a.ld_z + i] = f32_to_bf16(v);
    v = activate(v, a.act);
    if constexpr (GATE) {
        float u = 0.0f;
        for (int k = 0; k < kFewWarps; ++k) u = __fadd_rn(u, part[k][r + kOutputs][m]);
        u = __fadd_rn(u, g.bias != nullptr ? bf16_to_f32(g.bias[i]) : 0.0f);
        if (g.u != nullptr) g.u[m * g.ld_u + i] = f32_to_bf16(u);
        v = __fmul_rn(v, u);
    }
    if (a.resid != nullptr) v = __fadd_rn(v, bf16_to_f32(a.resid[m * a.ld_resid + i]));
    a.out[m * a.ld_out + i] = f32_to_bf16(v);
}

// ---------------------------------------------------------------- elementwise passes
// dst[r, c] = src[r, c] * act'(z[r, c]) (z null: a plain copy), dst with rows on 16-byte boundaries; column sums of
// the unrounded values over the rows of this CTA's band into partial[band, c], or, of the only band, into db[c] if wanted.  A warp
// takes 256 columns, a lane eight of them (16 bytes where src and z have 16-byte rows), the CTA's eight warps every eighth
// row; the warps' sums meet in shared memory in their order.  Bound by the latency of a row's loads at the occupancy
// that the slopes' registers leave: 1001 x 8807 with silu 18 us from cold caches (gelu 21), an instruction issued in 64 %
// of the cycles, 8 us of them the bytes.  In a row of launches, with the column sums, 16 (gelu 19, no activation 13); four
// rows' loads at once (128 registers) cost 2.4 more.
constexpr int kSlopeWarps = 8, kSlopeCols = 256;
template <bool VEC>
__global__ void __launch_bounds__(32 * kSlopeWarps) slope_kernel(const uint16_t* src, int64_t ld_src, const uint16_t* z, int64_t ld_z, int act, uint16_t* dst,
                                                                 int64_t ld_dst, int64_t rows, int64_t cols, int64_t band, float* partial, uint16_t* db) {
    __shared__ float sums[kSlopeWarps][kSlopeCols];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * kSlopeCols + lane * 8;
    const int64_t r0 = (int64_t)blockIdx.y * band, r1 = r0 + band < rows ? r0 + band : rows;
    await_previous_kernel();
    float sum[8] = {};
    if (c < cols) {
        for (int64_t r = r0 + warp; r < r1; r += kSlopeWarps) {
            uint32_t w[4], y[4];
            load8<VEC>(src + r * ld_src, c, cols, w);
            if (z != nullptr) load8<VEC>(z + r * ld_z, c, cols, y);
            float v[8], s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((e & 1) ? (w[e >> 1] & 0xFFFF0000u) : (w[e >> 1] << 16));
            if (z != nullptr) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = __uint_as_float((e & 1) ? (y[e >> 1] & 0xFFFF0000u) : (y[e >> 1] << 16));
                slope_all(s, act);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], s[e]);
                // dZ is rounded to bf16 here because the tensor cores take bf16; the column sums are not
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2(v[2 * e], v[2 * e + 1]);
            }
            if (dst != nullptr) *reinterpret_cast<uint4*>(dst + r * ld_dst + c) = make_uint4(w[0], w[1], w[2], w[3]);   // rows are padded to whole vectors
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = __fadd_rn(sum[e], v[e]);
        }
    }
    if (partial == nullptr && db == nullptr) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][lane * 8 + e] = sum[e];
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * kSlopeCols + threadIdx.x;
    if (col >= cols) return;
    float total = 0.0f;
    for (int w = 0; w < kSlopeWarps; ++w) total = __fadd_rn(total, sums[w][threadIdx.x]);
    if (db != nullptr) db[col] = f32_to_bf16(total);
    else partial[(int64_t)blockIdx.y * cols + col] = total;
}
constexpr int kSumCols = 128;
__global__ void __launch_bounds__(kSumCols) column_sum_kernel(const float* partial, int64_t bands, int64_t cols, uint16_t* out) {
    allow_next_kernel();
    await_previous_kernel();
    const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x;
    if (c >= cols) return;
    float sum = 0.0f;
#pragma unroll 8
    for (int64_t b = 0; b < bands; ++b) sum = __fadd_rn(sum, partial[b * cols + c]);
    out[c] = f32_to_bf16(sum);
}

// ---------------------------------------------------------------- host side
// Nanoseconds, measured with the contractions' lengths from 16 to 138 steps: 64 contraction steps of a pair's 256 x 256,
// of a CTA's 128 x 256, 128 x 128 and narrower tiles; an epilogue's column; a launch or a further wave; a shared contraction.
constexpr int64_t kPairStep = 350, kPairFixed = 6900, kWideStep = 454, kMidStep = 294, kNarrowStep = 260, kTileColumn = 5, kFixed = 3600,
                  kSplitFixed = 2000, kSplitColumn = 10, kSecondLaunch = 2000;

struct Matrix {
    const void* p;
    int64_t rows, cols, ld;
    size_t bytes() const { return rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * 2u : 0u; }
    bool tma_ok() const { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld % 8 == 0); }
    int64_t padded_ld() const { return (cols + 7) / 8 * 8; }
    size_t padded_bytes() const { return align_up((size_t)rows * (size_t)padded_ld() * 2u, 256); }
};

// Bands of rows: a CTA's eight warps take four rows each of the shortest; at most 64 bands.
int64_t band_rows(int64_t rows) { return rows <= 32 * 64 ? 32 : (rows + 63) / 64; }
int64_t bands_of(int64_t rows) { return (rows + band_rows(rows) - 1) / band_rows(rows); }

// A launch that may start under the one before it; `cluster` CTAs a cluster.
struct Launch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    Launch(dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster = 1) {
        attr[0] = early_start();
        attr[1] = cluster_of(cluster);
        cfg.gridDim = grid;
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 2 : 1;
    }
};

int run_slope(const Matrix& src, const void* z, int64_t ld_z, int act, void* dst, int64_t ld_dst, float* partial, void* db, cudaStream_t st) {
    const int64_t bands = bands_of(src.rows);
    if (bands > 0) {
        Launch l(dim3((unsigned)((src.cols + kSlopeCols - 1) / kSlopeCols), (unsigned)bands), 32 * kSlopeWarps, 0, st);
        const Matrix zm{z, src.rows, src.cols, ld_z};
        const bool vec = src.tma_ok() && (z == nullptr || zm.tma_ok());
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, vec ? slope_kernel<true> : slope_kernel<false>, static_cast<const uint16_t*>(src.p), src.ld,
                                           static_cast<const uint16_t*>(z), ld_z, act, static_cast<uint16_t*>(dst), ld_dst, src.rows, src.cols,
                                           band_rows(src.rows), partial, bands == 1 ? static_cast<uint16_t*>(db) : nullptr));
    }
    if (db != nullptr && bands != 1) {   // of one band the sums are final
        Launch l(dim3((unsigned)((src.cols + kSumCols - 1) / kSumCols)), kSumCols, 0, st);
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, column_sum_kernel, static_cast<const float*>(partial), bands, src.cols, static_cast<uint16_t*>(db)));
    }
    return MOSAIC_OK;
}

// A matrix TMA can read: itself, or a copy at *ws (advanced) with rows on 16-byte boundaries.
int readable(Matrix& m, char** ws, cudaStream_t st) {
    if (m.rows == 0 || m.tma_ok()) return MOSAIC_OK;
    const int rc = run_slope(m, nullptr, 0, MOSAIC_ACT_NONE, *ws, m.padded_ld(), nullptr, nullptr, st);
    if (rc != MOSAIC_OK) return rc;
    m.p = *ws;
    m.ld = m.padded_ld();
    *ws += m.padded_bytes();
    return MOSAIC_OK;
}

template <bool A_MN, bool B_MN> int encode_operands(CUtensorMap* a_map, CUtensorMap* b_map, const Matrix& A, const Matrix& B, int rows_a, int rows_b) {
    const bool a_ok = A_MN ? encode_bf16(a_map, A.p, A.rows, A.cols, A.ld, kMC, 64) : encode_bf16(a_map, A.p, A.rows, A.cols, A.ld, rows_a, kMC);
    const bool b_ok = B_MN ? encode_bf16(b_map, B.p, B.rows, B.cols, B.ld, kMC, 64) : encode_bf16(b_map, B.p, B.rows, B.cols, B.ld, rows_b, kMC);
    return a_ok && b_ok ? MOSAIC_OK : MOSAIC_ERR_CUDA;
}

template <int BN> constexpr size_t kMRing = 196 * 1024 / ((size_t)(kMI + BN) * kMC * 2 * kMSub) * ((size_t)(kMI + BN) * kMC * 2 * kMSub);   // one CTA an SM
template <bool A_MN, bool B_MN, int BN, int MODE> bool opt_in() {
    static DeviceCache opted;
    return opted.get([]() -> int {
        if (cudaFuncSetAttribute(mm_kernel<A_MN, B_MN, BN, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMRing<BN> + 1024) == cudaSuccess) return 1;
        (void)cudaGetLastError();
        return -1;
    }) > 0;
}

// Clusters of `split` one-an-SM CTAs that run at a time: fewer than the SMs divided by split, as a cluster's SMs are of
// one processing cluster (148 SMs hold 33 clusters of four and 15 of eight).
int64_t resident_clusters(int split) {
    if (split == 1) return sm_count();
    static DeviceCache held[kMMaxSplit + 1];
    return held[split].get([&]() -> int {
        if (opt_in<false, false, 64, kPlain>()) {
            Launch l(dim3((unsigned)split), mm_threads(64), kMRing<64> + 1024, nullptr, split);
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, mm_kernel<false, false, 64, kPlain>, &l.cfg) == cudaSuccess && n > 0) return n;
            (void)cudaGetLastError();
        }
        const int n = sm_count() / split;
        return n > 0 ? n : 1;
    });
}

// What mm_kernel's tiles would take, and the CTAs that share one's contraction (each keeps two stages or more).
struct MmPlan {
    int64_t nanoseconds;
    int split;
};
MmPlan plan_mm(int64_t tiles, int64_t steps, int64_t bn) {
    MmPlan best = {0, 1};
    const int64_t step = bn == 256 ? kWideStep : bn == 128 ? kMidStep : kNarrowStep;
    for (int split = 1; split <= kMMaxSplit && (split == 1 || steps >= 4 * split); ++split) {
        const int64_t held = resident_clusters(split), waves = (tiles + held - 1) / held;
        const int64_t c = waves * ((steps + split - 1) / split * step + bn * kTileColumn + kFixed + (split > 1 ? kSplitFixed + bn * kSplitColumn : 0));
        if (split == 1 || c < best.nanoseconds) best = {c, split};
    }
    return best;
}

// The matrices of a product's second half (kGate: A; kSum: A and B; kTwin: B, out).
struct Also {
    Matrix A, B;
    GateArgs gate;
    uint16_t* out;
    int64_t ld_out;
};
template <bool A_MN, bool B_MN, int MODE> int encode_second(Second<MODE>* second, const Matrix& A, const Also& also, int rows_a, int rows_b) {
    if constexpr (MODE == kGate) {
        second->g = also.gate;
        return encode_bf16(&second->a, also.A.p, also.A.rows, also.A.cols, also.A.ld, kGateRows, kMC) ? MOSAIC_OK : MOSAIC_ERR_CUDA;
    } else if constexpr (MODE == kSum) {
        return encode_operands<A_MN, B_MN>(&second->a, &second->b, also.A, also.B, rows_a, rows_b);
    } else if constexpr (MODE == kTwin) {
        second->out = also.out;
        second->ld_out = also.ld_out;
        const Matrix& B = also.B;
        return (B_MN ? encode_bf16(&second->b, B.p, B.rows, B.cols, B.ld, kMC, 64) : encode_bf16(&second->b, B.p, B.rows, B.cols, B.ld, rows_b, kMC))
                   ? MOSAIC_OK : MOSAIC_ERR_CUDA;
    }
    return MOSAIC_OK;
}

template <bool A_MN, bool B_MN, int BN, int MODE>
int launch_mm(const Matrix& A, const Matrix& B, MmArgs a, const Also& also, int64_t tiles, int split, cudaStream_t st) {
    static_assert(kMRing<BN> >= (size_t)(BN + kMMaxSplit) * kMI * 4, "the partial sums lie where the stages were");
    CUtensorMap a_map, b_map;
    Second<MODE> second;
    if (encode_operands<A_MN, B_MN>(&a_map, &b_map, A, B, MODE == kGate ? kGateRows : kMI, BN) != MOSAIC_OK ||
        encode_second<A_MN, B_MN, MODE>(&second, A, also, kMI, BN) != MOSAIC_OK || !opt_in<A_MN, B_MN, BN, MODE>())
        return MOSAIC_ERR_CUDA;
    a.tiles_i = (int)((a.n_i + kTileI<MODE> - 1) / kTileI<MODE>);
    a.tiles_j = (int)((a.n_j + BN - 1) / BN);
    a.split = split;
    a.stages = (int)(kMRing<BN> / ((size_t)(kMI + BN) * kMC * 2 * kMSub));
    if (tiles * split > 0x7FFFFFFF) return MOSAIC_ERR_INVALID_ARG;
    Launch l(dim3((unsigned)(tiles * split)), mm_threads(BN), kMRing<BN> + 1024, st, split);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, mm_kernel<A_MN, B_MN, BN, MODE>, a_map, b_map, a, second));
    return MOSAIC_OK;
}

template <bool A_MN, bool B_MN, int MODE> int launch_pair(const Matrix& A, const Matrix& B, MmArgs a, const Also& also, int64_t tiles, cudaStream_t st) {
    CUtensorMap a_map, b_map;
    Second<MODE> second;
    if (encode_operands<A_MN, B_MN>(&a_map, &b_map, A, B, MODE == kGate ? kGateRows : kPHalf, kPHalf) != MOSAIC_OK ||
        encode_second<A_MN, B_MN, MODE>(&second, A, also, kPHalf, kPHalf) != MOSAIC_OK)
        return MOSAIC_ERR_CUDA;
    a.tiles_i = a.pair_i;
    a.tiles_j = a.pair_j;
    static DeviceCache opted;
    const int ok = opted.get([&]() -> int {
        if (cudaFuncSetAttribute(mm_pair_kernel<A_MN, B_MN, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPSmem<MODE>) != cudaSuccess) {
            (void)cudaGetLastError();
            return -1;
        }
        return 1;
    });
    if (ok < 0) return MOSAIC_ERR_CUDA;
    const int64_t pairs = sm_count() / 2;
    Launch l(dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), kPThreads, kPSmem<MODE>, st);   // the cluster is the kernel's own
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, mm_pair_kernel<A_MN, B_MN, MODE>, a_map, b_map, a, second, (int)tiles));
    return MOSAIC_OK;
}

// out[j, i] = sum_c A B; A: [n_i, n_c] (or [n_c, n_i] if A_MN), B likewise; the other modes as `also` says.
template <bool A_MN, bool B_MN, int MODE = kPlain> int run_mm(const Matrix& A, const Matrix& B, MmArgs a, cudaStream_t st, const Also& also = {}) {
    const int64_t steps = (MODE == kSum ? 2 : 1) * ((a.n_c + kMC - 1) / kMC), sms = sm_count(), halves = MODE == kTwin ? 2 : 1;
    const auto even = [](const void* p, int64_t ld) { return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 3u) == 0 && ld % 2 == 0); };
    a.pairs = even(a.out, a.ld_out) && even(a.resid, a.ld_resid) && even(a.z, a.ld_z) && even(also.gate.u, also.gate.ld_u) && even(also.out, also.ld_out) ? 1 : 0;
    constexpr int64_t kWide = 2 * kTileI<MODE>;   // output elements of a pair's tile
    const int64_t pi = (a.n_i + kWide - 1) / kWide, pj = (a.n_j + kPTile - 1) / kPTile, large = pi * pj * halves, pairs = sms / 2;
    if (large > 0x0FFFFFFF) return MOSAIC_ERR_INVALID_ARG;
    a.pair_i = (int)pi;
    a.pair_j = (int)pj;
    a.first_pair = -1;
    // Which kernel and tile: what each would take.
    const int64_t ti = (a.n_i + kTileI<MODE> - 1) / kTileI<MODE>;
    MmPlan plan = {0, 1};
    int64_t bn = 0;
    for (int64_t w = B_MN ? 64 : 16; w <= 256; w *= 2) {
        const MmPlan p = plan_mm(halves * ti * ((a.n_j + w - 1) / w), steps, w);
        if (bn == 0 || p.nanoseconds < plan.nanoseconds) {
            plan = p;
            bn = w;
        }
        if (w >= a.n_j) break;
    }
    // The pair kernel, and its last wave, if of few tiles, in quarters whose contraction is shared (14336 x 2048 outputs
    // from 4096, 448 tiles for 74 pairs: 178 instead of 184 us).
    const int64_t waves = large / pairs, rest = large % pairs, wave = steps * kPairStep;
    const MmPlan quarters = plan_mm(rest * 4, steps, 128);
    const bool cut = waves > 0 && rest > 0 && quarters.nanoseconds + kSecondLaunch < wave;
    if (waves * wave + (cut ? quarters.nanoseconds + kSecondLaunch : rest > 0 ? wave : 0) + kPairFixed < plan.nanoseconds) {
        const int rc = launch_pair<A_MN, B_MN, MODE>(A, B, a, also, cut ? waves * pairs : large, st);
        if (rc != MOSAIC_OK || !cut) return rc;
        a.first_pair = (int)(waves * pairs);
        return launch_mm<A_MN, B_MN, 128, MODE>(A, B, a, also, rest * 4, quarters.split, st);
    }
    const int64_t tiles = halves * ti * ((a.n_j + bn - 1) / bn);
    if constexpr (!B_MN) {
        if (bn == 16) return launch_mm<A_MN, B_MN, 16, MODE>(A, B, a, also, tiles, plan.split, st);
        if (bn == 32) return launch_mm<A_MN, B_MN, 32, MODE>(A, B, a, also, tiles, plan.split, st);
    }
    if (bn == 64) return launch_mm<A_MN, B_MN, 64, MODE>(A, B, a, also, tiles, plan.split, st);
    return bn == 128 ? launch_mm<A_MN, B_MN, 128, MODE>(A, B, a, also, tiles, plan.split, st)
                     : launch_mm<A_MN, B_MN, 256, MODE>(A, B, a, also, tiles, plan.split, st);
}

template <bool GATE> int launch_few(const Matrix& x, const Matrix& w, const MmArgs& a, cudaStream_t st, const GateArgs& g = {}) {
    using Kernel = void (*)(const uint16_t*, int64_t, const uint16_t*, int64_t, MmArgs, GateArgs);
    static const Kernel plain[kFewTokens] = {few_kernel<1, false, GATE>, few_kernel<2, false, GATE>, few_kernel<3, false, GATE>, few_kernel<4, false, GATE>};
    static const Kernel vector[kFewVector] = {few_kernel<1, true, GATE>, few_kernel<2, true, GATE>};
    const bool vec = x.tma_ok() && w.tma_ok() && (!GATE || Matrix{g.w, w.rows, w.cols, g.ld_w}.tma_ok());
    const Kernel kernel = vec ? vector[a.n_j - 1] : plain[a.n_j - 1];
    constexpr int kOutputs = GATE ? kFewRows / 2 : kFewRows;
    const int64_t ctas = (a.n_i + kOutputs - 1) / kOutputs;
    Launch l(dim3((unsigned)ctas), 32 * kFewWarps, 0, st);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, kernel, static_cast<const uint16_t*>(x.p), x.ld,
                                       static_cast<const uint16_t*>(w.p), w.ld, a, g));
    return MOSAIC_OK;
}

bool overlap(const Matrix& a, const Matrix& b) {
    const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
    return x != nullptr && y != nullptr && a.bytes() > 0 && b.bytes() > 0 && x < y + b.bytes() && y < x + a.bytes();
}

// null / element alignment / leading dimension of a matrix that is there (rows > 0)
int check_bf16(const Matrix& m) {
    if (m.ld < m.cols) return MOSAIC_ERR_INVALID_ARG;
    if (m.rows > 0 && m.p == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(m.p) & 1u) != 0) return MOSAIC_ERR_MISALIGNED;
    return MOSAIC_OK;
}
constexpr int64_t kMostExtent = 0x7FFFFFFF - 1024;
bool extents_ok(int64_t m, int64_t n, int64_t k) { return m >= 0 && n > 0 && k > 0 && m <= kMostExtent && n <= kMostExtent && k <= kMostExtent; }
bool act_ok(int act) { return act >= MOSAIC_ACT_NONE && act <= MOSAIC_ACT_SILU; }

int check_workspace(const void* ws, size_t ws_bytes, size_t need) {
    if (need == 0) return MOSAIC_OK;
    if (ws == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return MOSAIC_ERR_MISALIGNED;
    return ws_bytes < need ? MOSAIC_ERR_WORKSPACE_TOO_SMALL : MOSAIC_OK;
}

}  // namespace
}  // namespace mosaic
