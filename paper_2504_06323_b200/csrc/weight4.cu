// mosaic_quantize4 / mosaic_dequantize4 and mosaic_linear4 / mosaic_gated_linear4: weights in 4 bits with a scale for every `group`
// adjacent columns of a row, and the products that read them.
//
//     s = (largest magnitude / 7) to five significant bits,  code = w / s to the nearest whole number in -7..7,  w ~ code s
//
// A code has three significant bits and s five, so code * s has eight: it is a bf16 number, exactly, and a matrix in 4 bits
// is a bf16 matrix in less room.  The products below multiply by that number, whichever of them runs.
#include "lanes.cuh"
#include "mm.cuh"

namespace mosaic {
namespace {

struct Weight4 {
    uint8_t* codes;                    // rows on 16-byte boundaries, two codes a byte, 8 added to each, the first in the low half
    int64_t ldc;
    uint16_t* scales;                  // bf16
    int64_t lds;
    int shift;                         // log2 of the group
};

// ---------------------------------------------------------------- packing
// A warp takes 256 columns, a lane eight of them, 4 to 16 lanes a group; kPackRows rows in flight.  Packing is bound by
// instructions: 11008 x 4096 in groups of 128 packed and unpacked in a row 49.5 us, of which 35 are the bytes.
constexpr int kPackWarps = 8, kPackRows = 4;

__device__ __forceinline__ float scale_of(float largest) {
    // a seventh, correctly rounded: a product and one correction (Markstein's division; below 2^-100, where the remainder
    // could underflow, divided)
    const float guess = __fmul_rn(largest, 0.142857149f);
    float ideal = __fmaf_rn(__fmaf_rn(-7.0f, guess, largest), 0.142857149f, guess);
    if (largest < 7.8886091e-31f) ideal = __fdiv_rn(largest, 7.0f);
    if (!(ideal <= 1.0633824e37f)) return ideal != ideal ? ideal : 1.0633824e37f;   // 2^123: 24 s below stays finite
    if (ideal < 1.17549435e-38f) return 0.0f;                                       // below bf16's normal numbers
    uint32_t u = __float_as_uint(ideal);
    u += 0x3FFFFu + ((u >> 19) & 1u);
    return __uint_as_float(u & 0xFFF80000u);
}

// Eight codes, 8 added to each.  w / s from an approximate reciprocal and one correction (Markstein's division): off by a rounding at
// most, and exact where w / s is half a whole number, because the correction's own error is the product of two small
// ones; every other w / s, of eight bits over five, is 2^-11 or more from such a border.  Between the borders of the first
// branch nothing underflows and w / s is below 7.3: s is within 2^-5 of a seventh of the largest.  Adding 3 2^22 rounds to a
// whole number in the float's low bits, ties to even; the eight are packed by multiplying them into place and taking off
// what the exponents' bits add up to.
__device__ __forceinline__ uint32_t codes_of8(const uint32_t (&w)[4], float s) {
    constexpr float kRound = 12582912.0f + 8.0f;
    constexpr uint32_t kBits = 0x4B400000u, kAll = kBits * 0x11111111u;
    uint32_t sum = 0;
    if (s > 7.8886091e-31f && s < 1.0e37f) {   // 2^-100
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = half_of(w, e), y = __fmul_rn(x, r);
            sum += __float_as_uint(__fadd_rn(__fmaf_rn(__fmaf_rn(-y, s, x), r, y), kRound)) << (4 * e);
        }
    } else {
#pragma unroll 1
        for (int e = 0; e < 8; ++e) {
            const uint32_t pair = e < 4 ? (e < 2 ? w[0] : w[1]) : (e < 6 ? w[2] : w[3]);
            const float x = __uint_as_float((e & 1) ? pair & 0xFFFF0000u : pair << 16);
            sum += __float_as_uint(__fadd_rn(fminf(fmaxf(__fdiv_rn(x, s), -7.0f), 7.0f), kRound)) << (4 * e);
        }
    }
    return sum - kAll;
}

template <bool VEC, int SHIFT>
__global__ void __launch_bounds__(32 * kPackWarps) quantize4_kernel(const uint16_t* W, int64_t ldw, int64_t rows, int64_t cols, const __grid_constant__ Weight4 out,
                                                                    unsigned chunks) {
    __shared__ uint4 turns[VEC ? 1 : kPackWarps][kTurn];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* turn = turns[VEC ? 0 : warp];
    const int64_t c0 = ((int64_t)(blockIdx.x % chunks) * kPackWarps + warp) * kWarpCols, c = c0 + lane * kLaneCols;
    const int64_t r0 = (int64_t)(blockIdx.x / chunks) * kPackRows;
    if (c0 >= cols) return;
    await_previous_kernel();
    uint32_t w[kPackRows][4];
#pragma unroll
    for (int r = 0; r < kPackRows; ++r) lane_load8<VEC>(W + (r0 + r < rows ? r0 + r : rows - 1) * ldw, c0, cols, turn, w[r]);
#pragma unroll
    for (int r = 0; r < kPackRows; ++r) {
        // the largest magnitude's bits: infinities and NaN are above all numbers
        const uint32_t m = __vmaxu2(__vmaxu2(w[r][0] & 0x7FFF7FFFu, w[r][1] & 0x7FFF7FFFu), __vmaxu2(w[r][2] & 0x7FFF7FFFu, w[r][3] & 0x7FFF7FFFu));
        uint32_t bits = max(m & 0xFFFFu, m >> 16);
#pragma unroll
        for (int o = 1; o < 1 << (SHIFT - 3); o <<= 1) bits = max(bits, __shfl_xor_sync(0xFFFFFFFFu, bits, o));
        const float s = bits >= 0x7F80u ? __uint_as_float(0x7FC00000u) : scale_of(bf16_to_f32((uint16_t)bits));
        if (r0 + r >= rows || c >= (cols + 31) / 32 * 32) continue;
        *reinterpret_cast<uint32_t*>(out.codes + (r0 + r) * out.ldc + c / 2) = s > 0.0f ? codes_of8(w[r], s) : 0x88888888u;
        if ((c & ((1 << SHIFT) - 1)) == 0 && c < cols) out.scales[(r0 + r) * out.lds + (c >> SHIFT)] = (uint16_t)(__float_as_uint(s) >> 16);
    }
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// -24 s, twice: exact
__device__ __forceinline__ uint32_t minus24(uint32_t s2) { return fma_bf16x2(s2, 0xC1C0C1C0u, 0x80008000u); }
// Codes i and i + 4 of a word (i = 0..3) as two bf16 weights, in three instructions: shifted to bits 3..6 of its half a code goes
// under the exponent of 16, which makes it 16 + n with n = code + 8, and (16 + n) s - 24 s is one fma, exact because s has five
// significant bits, 24 two and the result eight.  s2 and c2 hold s and -24 s twice.
__device__ __forceinline__ uint32_t weights4(uint32_t word, int i, uint32_t s2, uint32_t c2) {
    const uint32_t at = i == 0 ? word << 3 : word >> (4 * i - 3);
    uint32_t sum;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(sum) : "r"(at), "r"(0x00780078u), "r"(0x41804180u));   // and, or: one instruction
    return fma_bf16x2(sum, s2, c2);
}
template <bool VEC>
__global__ void __launch_bounds__(32 * kPackWarps) dequantize4_kernel(const __grid_constant__ Weight4 in, int64_t rows, int64_t cols, uint16_t* W, int64_t ldw,
                                                                      unsigned chunks) {
    __shared__ uint4 turns[VEC ? 1 : kPackWarps][kTurn];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* turn = turns[VEC ? 0 : warp];
    const int64_t c0 = ((int64_t)(blockIdx.x % chunks) * kPackWarps + warp) * kWarpCols, c = c0 + lane * kLaneCols;
    const int64_t r0 = (int64_t)(blockIdx.x / chunks) * kPackRows;
    if (c0 >= cols) return;
    await_previous_kernel();
    uint32_t q[kPackRows];
    uint32_t s[kPackRows];
#pragma unroll
    for (int r = 0; r < kPackRows; ++r) {
        const int64_t row = r0 + r < rows ? r0 + r : rows - 1;
        q[r] = 0x88888888u;
        s[r] = 0u;
        if (c < cols) {
            q[r] = *reinterpret_cast<const uint32_t*>(in.codes + row * in.ldc + c / 2);
            s[r] = in.scales[row * in.lds + (c >> in.shift)];
        }
    }
#pragma unroll
    for (int r = 0; r < kPackRows; ++r) {
        if (r0 + r >= rows) break;
        // a code under the exponent of 16 in each half of a word, then one exact fma; codes e and e + 4 come together
        const uint32_t s2 = s[r] | (s[r] << 16), c2 = minus24(s2);
        uint32_t f[4], w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = weights4(q[r], i, s2, c2);
        w[0] = __byte_perm(f[0], f[1], 0x5410);
        w[1] = __byte_perm(f[2], f[3], 0x5410);
        w[2] = __byte_perm(f[0], f[1], 0x7632);
        w[3] = __byte_perm(f[2], f[3], 0x7632);
        lane_store8<VEC>(W + (r0 + r) * ldw, c0, cols, turn, w);
    }
}

// ---------------------------------------------------------------- few tokens
// The next tokens of up to eight sequences: the weights are read once, and what counts is that they stream.  A tile is 16 weight
// rows - with GATE eight of each matrix, so that one lane has both sums of a channel.  The grid stays, one CTA an SM; `parts`
// warps share a tile's columns in blocks of 128, the CTA's groups of warps take tile after tile.  A lane copies 16 bytes, 32 codes,
// of two rows a block into its own place in shared memory, asynchronously, k4Ahead blocks a group of copies and two groups
// in flight; it reads them back itself, so no thread waits for another.  The matrix instruction (16 rows, 8 tokens, 16
// columns) does not mind which columns it is given as long as both operands agree: a lane's own 32 columns, in the order in
// which codes become weights, so that nothing moves between lanes; X lies in shared memory in that order.  Sums in fp32;
// over a tile's warps in their order.  Bound by instructions, of which the integer pipe takes half at half rate: one token through
// gate and up of 11008 x 4096 13.1 us warm, 17.3 cold, of which 7.1 are the bytes.
constexpr int k4Warps = 24, k4Tokens = 8, k4Rows = 16, k4Block = 128, k4Ahead = 2;
constexpr size_t k4Ring = 2 * k4Ahead * 1024;   // a warp's codes in flight

struct Few4Args {
    const uint16_t* x;                 // rows on 16-byte boundaries
    int64_t ldx, outputs, cols;
    int tokens, tiles, parts;
    Weight4 w, w2;                     // w2: GATE
    const uint16_t *bias, *bias2, *resid;
    int64_t ld_resid;
    int act;
    uint16_t* y;
    int64_t ldy;
};

__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void copy16_async(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <bool GATE>
__global__ void __launch_bounds__(32 * k4Warps) few4_kernel(const __grid_constant__ Few4Args a) {
    constexpr int kOutputs = GATE ? k4Rows / 2 : k4Rows;
    extern __shared__ uint4 smem4[];
    __shared__ float partial[k4Warps][8 * k4Rows];
    allow_next_kernel();
    const int warps = (int)blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int parts = a.parts, groups = warps / parts, part = warp % parts;
    const int blocks = (int)((a.cols + k4Block - 1) / k4Block), steps = (blocks + parts * k4Ahead - 1) / (parts * k4Ahead);
    const int row4 = blocks * 16 + 4, hop = parts * k4Block;          // columns from one of a warp's blocks to its next
    uint4* ring = smem4 + warp * (int)(k4Ring / 16) + lane;            // [group of copies][block][row][lane]
    uint4* x4 = smem4 + warps * (int)(k4Ring / 16);                    // [token][block][word of eight columns][quarter of the block], 64 bytes between tokens
    await_previous_kernel();

    // where the lane reads next: its two rows' codes and scales at a step's first block
    const Weight4& second = GATE ? a.w2 : a.w;
    const int col0 = part * k4Block + t * 32, hop0 = hop >> a.w.shift, hop1 = hop >> second.shift;
    const uint8_t *code0 = nullptr, *code1 = nullptr;
    const uint16_t *scale0 = nullptr, *scale1 = nullptr;
    int left = 0;                      // columns from the lane's first of the step on
    const auto begin = [&](int tile) {
        const int64_t o0 = (int64_t)tile * kOutputs;
        // past the end the tile's first row, not stored
        const int64_t lo = o0 + g < a.outputs ? o0 + g : o0, hi = GATE ? lo : (o0 + g + 8 < a.outputs ? o0 + g + 8 : o0);
        code0 = a.w.codes + lo * a.w.ldc + (col0 >> 1);
        code1 = second.codes + hi * second.ldc + (col0 >> 1);
        scale0 = a.w.scales + lo * a.w.lds + (col0 >> a.w.shift);
        scale1 = second.scales + hi * second.lds + (col0 >> second.shift);
        left = (int)a.cols - col0;
    };
    uint32_t next[k4Ahead];            // both rows' scales of the step on its way; 0 where there are no columns
    const auto fetch = [&](uint4* to) {
#pragma unroll
        for (int u = 0; u < k4Ahead; ++u) {
            next[u] = 0u;
            if (left > u * hop) {
                copy16_async(to + u * 64, code0 + u * (hop / 2));
                copy16_async(to + u * 64 + 32, code1 + u * (hop / 2));
                next[u] = scale0[u * hop0] | ((uint32_t)scale1[u * hop1] << 16);
            }
        }
        copies_commit();
        code0 += k4Ahead * (hop / 2);
        code1 += k4Ahead * (hop / 2);
        scale0 += k4Ahead * hop0;
        scale1 += k4Ahead * hop1;
        left -= k4Ahead * hop;
    };
    const int stride = groups * (int)gridDim.x;
    int tile = (warp / parts) * (int)gridDim.x + (int)blockIdx.x, half = 0;
    if (tile < a.tiles) {
        begin(tile);
        fetch(ring);
    }
    for (int token = 0; token < a.tokens; ++token)
        for (int at = (int)threadIdx.x; at < blocks * 16; at += (int)blockDim.x) {
            uint32_t x[4];
            load8<true>(a.x + token * a.ldx, (int64_t)(at >> 4) * k4Block + (at & 3) * 32 + ((at >> 2) & 3) * 8, a.cols, x);
            // elements (0, 4), (1, 5), (2, 6), (3, 7), as the codes come
            x4[token * row4 + at] = make_uint4(__byte_perm(x[0], x[2], 0x5410), __byte_perm(x[0], x[2], 0x7632), __byte_perm(x[1], x[3], 0x5410),
                                               __byte_perm(x[1], x[3], 0x7632));
        }
    __syncthreads();
    const uint4* mine = x4 + min(g, a.tokens - 1) * row4 + part * 16 + t;   // columns of the product beyond the last token repeat it and are not stored
    const auto store = [&](int token, int64_t o, float v, float u) {
        if (token >= a.tokens || o >= a.outputs) return;
        v = activate(__fadd_rn(v, a.bias != nullptr ? bf16_to_f32(a.bias[o]) : 0.0f), a.act);
        if (GATE) v = __fmul_rn(v, __fadd_rn(u, a.bias2 != nullptr ? bf16_to_f32(a.bias2[o]) : 0.0f));
        if (a.resid != nullptr) v = __fadd_rn(v, bf16_to_f32(a.resid[token * a.ld_resid + o]));
        a.y[token * a.ldy + o] = f32_to_bf16(v);
    };
    for (int first = (int)blockIdx.x; first < a.tiles; first += stride, tile += stride) {   // the same turns for all of the CTA's warps
        float acc[4] = {}, odd[4] = {};
        if (tile < a.tiles) {
#pragma unroll 1
            for (int step = 0; step < steps; ++step, half ^= 1) {
                uint32_t now[k4Ahead];
#pragma unroll
                for (int u = 0; u < k4Ahead; ++u) now[u] = next[u];
                uint4* to = ring + (half ^ 1) * (k4Ahead * 64);
                if (step + 1 < steps) {
                    fetch(to);
                    copies_wait<1>();
                } else if (tile + stride < a.tiles) {
                    begin(tile + stride);
                    fetch(to);
                    copies_wait<1>();
                } else {
                    copies_wait<0>();
                }
                const uint4 *from = ring + half * (k4Ahead * 64), *x = mine + step * (k4Ahead * parts * 16);
#pragma unroll
                for (int u = 0; u < k4Ahead; ++u) {
                    if ((step * k4Ahead + u) * parts + part >= blocks) break;
                    const uint4 qa = from[u * 64], qb = from[u * 64 + 32];   // of no copy where there are no columns: any codes, times a scale of zero
                    const uint32_t sa = __byte_perm(now[u], 0u, 0x1010), sb = __byte_perm(now[u], 0u, 0x3232), ca = minus24(sa), cb = minus24(sb);
#pragma unroll
                    for (int wd = 0; wd < 4; ++wd) {
                        const uint32_t wa = wd == 0 ? qa.x : wd == 1 ? qa.y : wd == 2 ? qa.z : qa.w, wb = wd == 0 ? qb.x : wd == 1 ? qb.y : wd == 2 ? qb.z : qb.w;
                        const uint4 xv = x[u * parts * 16 + wd * 4];
                        mma_16816(acc, weights4(wa, 0, sa, ca), weights4(wb, 0, sb, cb), weights4(wa, 1, sa, ca), weights4(wb, 1, sb, cb), xv.x, xv.y);
                        mma_16816(odd, weights4(wa, 2, sa, ca), weights4(wb, 2, sb, cb), weights4(wa, 3, sa, ca), weights4(wb, 3, sb, cb), xv.z, xv.w);
                    }
                }
            }
        }
        // a lane holds rows g and g + 8 of tokens 2 t and 2 t + 1
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __fadd_rn(acc[e], odd[e]);
        if (parts == 1) {
            if (tile < a.tiles) {
                const int64_t o = (int64_t)tile * kOutputs + g;
                store(2 * t, o, acc[0], acc[2]);
                store(2 * t + 1, o, acc[1], acc[3]);
                if (!GATE) {
                    store(2 * t, o + 8, acc[2], 0.0f);
                    store(2 * t + 1, o + 8, acc[3], 0.0f);
                }
            }
            continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) partial[warp][(2 * t + (e & 1)) * k4Rows + g + (e >> 1) * 8] = acc[e];
        __syncthreads();
        for (int at = part * 32 + lane; at < kOutputs * a.tokens; at += parts * 32) {
            const int token = at / kOutputs, r = at % kOutputs;
            float v = 0.0f, u = 0.0f;
            for (int w = warp - part; w < warp - part + parts; ++w) {
                v = __fadd_rn(v, partial[w][token * k4Rows + r]);
                if (GATE) u = __fadd_rn(u, partial[w][token * k4Rows + r + 8]);
            }
            if (tile < a.tiles) store(token, (int64_t)tile * kOutputs + r, v, u);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- more tokens
// The tensor cores' product with the weights' tile made on the way: mm_kernel's tile, cluster and epilogue (mm.cuh), but of A only
// the codes are loaded, 128 rows x 256 columns a stage in 16 KB; 8 or 12 warps make bf16 of them, a weight row a lane, and put
// them into tensor memory, where the matrix instruction reads its first operand.  The weights so cross shared memory as codes,
// once, instead of as bf16 twice: with them in shared memory its bandwidth would hold the stream to about half of what
// memory gives.  Bound by the widening's instructions, 0.29 us a tile and 128 columns whatever the tokens up to 64, and in small
// calls by start and end (about 5 us with a cluster): 16 tokens, 4096 outputs from 8807, 10.9 us; 64 tokens, 11008 from
// 4096, 13.3 (19 with bf16 weights).
constexpr int kC4Cols = 256;
// Sets of four warps make a stage's weights in turn.
template <int BN> constexpr int kC4Sets = BN == 128 ? 2 : 3;
template <int BN> constexpr int kC4Threads = 32 * (kMRoles + 4 * kC4Sets<BN>);   // code loader, MMA issue; weight makers
constexpr uint32_t kC4Bytes = kMI * kC4Cols / 2, kC4Box = kGateRows * kC4Cols / 2;   // of a stage's codes, of kGate's rows of one matrix
// X comes with the codes it meets: in a ring of its own it waited behind the codes of stages to come (17.3 us for 11.4, 16 tokens,
// 4096 outputs from 8807).
template <int BN> constexpr int kC4Slots = BN == 16 ? 8 : BN == 32 ? 6 : BN == 64 ? 4 : 2;
template <int BN> constexpr uint32_t kC4Slot = kC4Bytes + (uint32_t)BN * kC4Cols * 2u;
constexpr int kC4Made = 3;             // stages made weights of, 128 columns of tensor memory each
// A set waits twice a stage: for its codes (full), and for room, that is for the products of the stage kC4Made before it (used).  A
// wait sees a phase's parity alone: it passes as well while the phase before that one has not completed, so the set must know that
// it has.  Loads land in any order; that a later stage has landed proves nothing.  So the ring whose slots are each one
// set's own comes first - there the set has waited for every phase itself - and its phase then proves the other ring's:
//     room first: the products of stage s - kC4Made are complete, so were issued, so every stage up to it has landed, the one
//         before in the slot of s among them if there are kC4Made slots or more
//     codes first: the load of stage s was issued, so the products of s - slots are complete, so the weights of every stage up to
//         it were made, by sets that had found the room that this set asks about if there are no more slots than kC4Made
template <int BN> constexpr bool kC4RoomFirst = kC4Made % kC4Sets<BN> == 0;
template <int BN> constexpr bool kC4Proved = kC4RoomFirst<BN> ? kC4Slots<BN> >= kC4Made : kC4Slots<BN> % kC4Sets<BN> == 0 && kC4Slots<BN> <= kC4Made;
static_assert(kC4Proved<16> && kC4Proved<32> && kC4Proved<64> && kC4Proved<128>, "a wait's parity tells two phases apart, no more");
template <int BN> constexpr uint32_t kC4Acc = BN < 32 ? 32 : BN;                      // tensor-memory columns of the accumulator
constexpr long long kLandCycles = 20000000ll;   // ten milliseconds: far more than a load takes
// One CTA an SM: it takes all of the tensor memory, and one that waited for it could hold up its cluster.
template <int BN> constexpr size_t kC4Smem = kC4Slots<BN> * (size_t)kC4Slot<BN> + 1024;
static_assert(kC4Smem<16> > 115 * 1024 && kC4Smem<32> > 115 * 1024 && kC4Smem<64> > 115 * 1024 && kC4Smem<128> > 115 * 1024, "one CTA an SM");

struct Scales4 {
    const uint16_t *p, *p2;            // p2: the second matrix's (kGate)
    int64_t ld, ld2;
    int shift, shift2;
    int groups, groups2;               // a row's
    int wide, wide2;                   // a stage's scales of a row may be read as one word
};

// The scales of a row's 256 columns from `col` on, past the last group that one's again; as they are loaded, and then a word for each
// 64 columns, a half for each 32 (apart, so that nothing waits for the loads before their stage).
__device__ __forceinline__ uint4 scales_of(const uint16_t* row, int col, int shift, int groups, bool wide) {
    const int at = col >> shift, n = kC4Cols >> shift;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (wide && at + n <= groups) {
        if (shift == 7) v.x = *reinterpret_cast<const uint32_t*>(row + at);
        else if (shift == 6) {
            const uint2 w = *reinterpret_cast<const uint2*>(row + at);
            v.x = w.x;
            v.y = w.y;
        } else {
            v = *reinterpret_cast<const uint4*>(row + at);
        }
        return v;
    }
    const auto pair = [&](int k) { return (uint32_t)row[min(at + k, groups - 1)] | ((uint32_t)row[min(at + k + 1, groups - 1)] << 16); };
    v.x = pair(0);
    if (shift <= 6) v.y = pair(2);
    if (shift == 5) {
        v.z = pair(4);
        v.w = pair(6);
    }
    return v;
}
__device__ __forceinline__ uint4 scales_spread(uint4 s, int shift) {
    const auto lo = [](uint32_t w) { return __byte_perm(w, 0u, 0x1010); };
    const auto hi = [](uint32_t w) { return __byte_perm(w, 0u, 0x3232); };
    if (shift == 7) return make_uint4(lo(s.x), lo(s.x), hi(s.x), hi(s.x));
    if (shift == 6) return make_uint4(lo(s.x), hi(s.x), lo(s.y), hi(s.y));
    return s;
}
// The eight weights of a word in their order: each byte's codes to bits 3..6 of the halves by one multiplication, then as in weights4.
__device__ __forceinline__ void weights4_in_order(uint32_t word, uint32_t s2, uint32_t c2, uint32_t* w) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t at = __byte_perm(word, 0u, 0x4440 | j) * 0x8008u;
        uint32_t sum;
        asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(sum) : "r"(at), "r"(0x00780078u), "r"(0x41804180u));
        w[j] = fma_bf16x2(sum, s2, c2);
    }
}

template <int BN, int MODE>
__global__ void __launch_bounds__(kC4Threads<BN>) mm4_kernel(const __grid_constant__ CUtensorMap code_map, const __grid_constant__ CUtensorMap x_map,
                                                         const __grid_constant__ MmArgs a, const __grid_constant__ Second<MODE> second,
                                                         const __grid_constant__ Scales4 scales) {
    constexpr int kSlots = kC4Slots<BN>, kSets = kC4Sets<BN>;
    constexpr uint32_t kDesc = instr_desc(false, false, kMI, BN);
    extern __shared__ unsigned char mm4_smem_raw[];
    __shared__ uint64_t full[kSlots], empty[kSlots], ready[kC4Made], used[kC4Made], acc_full;
    __shared__ uint32_t tmem_slot;
    __shared__ int err_word;
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(mm4_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    volatile int* err = &err_word;
    const int split = a.split, rank = (int)(blockIdx.x % (unsigned)split);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = (int)(blockIdx.x / (unsigned)split);
    const int64_t i0 = (int64_t)(tile % a.tiles_i) * kTileI<MODE>, j0 = (int64_t)(tile / a.tiles_i) * BN;
    const int64_t all_steps = (a.n_c + kC4Cols - 1) / kC4Cols;
    const int s0 = (int)(all_steps * rank / split), steps = (int)(all_steps * (rank + 1) / split) - s0;   // split <= steps: never empty

    if (threadIdx.x == 0) {
        prefetch_map(&code_map);
        prefetch_map(&x_map);
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(&full[s], 1u);
            mbar_init(&empty[s], 1u);    // the products of its columns have completed, so its codes have been read
        }
        for (int s = 0; s < kC4Made; ++s) {
            mbar_init(&ready[s], 4u);    // the four warps that make a stage's weights
            mbar_init(&used[s], 1u);     // its products have completed
        }
        mbar_init(&acc_full, 1u);
        *err = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot, tmem_a = tmem + kC4Acc<BN>;
    allow_next_kernel();   // not before this CTA has its tensor memory: the next kernel's CTAs wait for it with theirs in hand
    await_previous_kernel();

    if (warp == 0) {
        if (lane == 0) {
            for (int s = 0; s < steps; ++s) {
                const int slot = s % kSlots;
                if (!mbar_wait(&empty[slot], ((uint32_t)(s / kSlots) & 1u) ^ 1u, err)) break;
                mbar_expect_tx(&full[slot], kC4Slot<BN>);
                unsigned char* codes = ring + slot * kC4Slot<BN>;
                const int c = (s0 + s) * (kC4Cols / 2);
                if constexpr (MODE == kGate) {
                    tma_load_box(codes, &code_map, &full[slot], c, (int)i0);
                    tma_load_box(codes + kC4Box, &second.a, &full[slot], c, (int)i0);
                } else {
                    tma_load_box(codes, &code_map, &full[slot], c, (int)i0);
                }
#pragma unroll
                for (int h = 0; h < kC4Cols / kMC; ++h)
                    tma_load_box(codes + kC4Bytes + h * (BN * kMC * 2), &x_map, &full[slot], (s0 + s) * kC4Cols + h * kMC, (int)j0);
            }
        }
    } else if (warp == 1) {
        // all lanes alike, one of them issues; its pace is the pipeline's
        const bool issue = elect_one();
        const uint32_t acc = __shfl_sync(0xFFFFFFFFu, tmem, 0), made0 = acc + kC4Acc<BN>;
        const uint64_t d0 = operand_desc(smem_u32(ring) + kC4Bytes, 16u);
        const uint32_t hi = (uint32_t)(d0 >> 32), lo0 = __shfl_sync(0xFFFFFFFFu, (uint32_t)d0, 0);
        bool ok = true;
        int slot = 0, made = 0;
        uint32_t slot_ph = 0, made_ph = 0, lo = lo0;
        for (int s = 0; s < steps; ++s) {
            ok = __all_sync(0xFFFFFFFFu, mbar_wait(&full[slot], slot_ph, err) && mbar_wait(&ready[made], made_ph, err));
            if (!ok) break;
            tc_fence_after();
            const uint32_t from = made0 + (uint32_t)made * 128u;
            if (issue) {
#pragma unroll
                for (int k = 0; k < kC4Cols / 16; ++k)
                    umma_bf16_from_tmem(acc, from + (uint32_t)k * 8u, lo + (uint32_t)((k / 4) * (BN * kMC * 2) + (k % 4) * 32) / 16u, hi, kDesc, k > 0 || s > 0);
                umma_commit(&used[made]);
                umma_commit(&empty[slot]);
            }
            __syncwarp();
            if (++made == kC4Made) {
                made = 0;
                made_ph ^= 1u;
            }
            lo += kC4Slot<BN> / 16u;
            if (++slot == kSlots) {
                slot = 0;
                slot_ph ^= 1u;
                lo = lo0;
            }
        }
        if (ok && issue) umma_commit(&acc_full);
    } else {
        // a weight row a lane; sets of four warps take stages in turn
        const int q = warp & 3, set = (warp - kMRoles) >> 2, r = q * 32 + lane;
        int64_t row = i0 + r;
        bool other = false;
        if constexpr (MODE == kGate) {
            other = r >= kGateRows;
            row = i0 + (r & (kGateRows - 1));
        }
        if (row >= a.n_i) row = a.n_i - 1;   // rows past the end: any numbers, not stored
        const uint16_t* at = other ? scales.p2 + row * scales.ld2 : scales.p + row * scales.ld;
        const int shift = other ? scales.shift2 : scales.shift, groups = other ? scales.groups2 : scales.groups;
        const bool wide = (other ? scales.wide2 : scales.wide) != 0;
        uint4 next = make_uint4(0u, 0u, 0u, 0u);
        if (set < steps) next = scales_of(at, (s0 + set) * kC4Cols, shift, groups, wide);
        for (int s = set; s < steps; s += kSets) {
            const int slot = s % kSlots, made = s % kC4Made;
            const uint4 sc = scales_spread(next, shift);
            if (s + kSets < steps) next = scales_of(at, (s0 + s + kSets) * kC4Cols, shift, groups, wide);
            const auto room = [&]() { return mbar_wait(&used[made], ((uint32_t)(s / kC4Made) & 1u) ^ 1u, err); };
            if (kC4RoomFirst<BN> && !room()) break;
            if (!mbar_wait(&full[slot], (uint32_t)(s / kSlots) & 1u, err)) break;
            if (!kC4RoomFirst<BN> && !room()) break;
            __syncwarp();
            tc_fence_after();
            const unsigned char* codes = ring + slot * kC4Slot<BN> + r * 128;
            const uint32_t to = tmem_a + ((uint32_t)(q * 32) << 16) + (uint32_t)made * 128u;
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t w[32];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const uint4 v = *reinterpret_cast<const uint4*>(codes + (((h * 2 + e) ^ (r & 7)) << 4));
                    const uint32_t both = h == 0 ? sc.x : h == 1 ? sc.y : h == 2 ? sc.z : sc.w, s2 = __byte_perm(both, 0u, e == 0 ? 0x1010 : 0x3232), c2 = minus24(s2);
                    weights4_in_order(v.x, s2, c2, w + e * 16);
                    weights4_in_order(v.y, s2, c2, w + e * 16 + 4);
                    weights4_in_order(v.z, s2, c2, w + e * 16 + 8);
                    weights4_in_order(v.w, s2, c2, w + e * 16 + 12);
                }
                tmem_store32(to + (uint32_t)h * 32u, w);
            }
            tmem_stored();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ready[made]);
        }
    }
    __syncwarp();
    const bool done = tile_done<MODE>(warp >= kMRoles && mbar_wait(&acc_full, 0u, err));
    tc_fence_after();
    const int n_cols = (int)(a.n_j - j0 < BN ? a.n_j - j0 : BN);
    const int per = (n_cols + split - 1) / split;
    float* part = reinterpret_cast<float*>(ring);
    if (split > 1) {
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (done) tile_out<BN, MODE, kSets>(a, second, tmem, part, per, rank, split, n_cols, i0, j0);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (threadIdx.x == 0 && *err != 0) {
        // a role gave up: let loads on their way land before shared memory is reused or left (bounded)
        const long long t0 = clock64();
        while (clock64() - t0 < kLandCycles) {
        }
        if (a.status != nullptr) atomicExch(a.status, 1);
    }
    if (split > 1) {
        __syncwarp();
        cluster_arrive();
        tile_join<MODE, kC4Threads<BN>>(a, second, part, per, rank, split, n_cols, i0, j0);
    }
}

// ---------------------------------------------------------------- host side
int64_t code_width(int64_t cols) { return (cols + 31) / 32 * 16; }
int group_shift(int64_t group) { return group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : 0; }
int check_weight4(const mosaic_weight4* w, int64_t rows, int64_t cols) {
    if (w == nullptr) return MOSAIC_ERR_NULL_PTR;
    if (group_shift(w->group) == 0 || w->ldc < code_width(cols) || w->lds < (cols + w->group - 1) / w->group) return MOSAIC_ERR_INVALID_ARG;
    if (rows > 0 && (w->codes == nullptr || w->scales == nullptr)) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(w->codes) & 15u) != 0 || w->ldc % 16 != 0 || (reinterpret_cast<uintptr_t>(w->scales) & 1u) != 0) return MOSAIC_ERR_MISALIGNED;
    return MOSAIC_OK;
}
Weight4 as_weight4(const mosaic_weight4* w) {
    return {static_cast<uint8_t*>(w->codes), w->ldc, static_cast<uint16_t*>(w->scales), w->lds, group_shift(w->group)};
}
struct Spans4 {
    const void *codes, *scales;
    size_t n_codes, n_scales;
    Spans4(const mosaic_weight4* w, int64_t rows, int64_t cols) : codes(w->codes), scales(w->scales) {
        n_codes = rows > 0 ? (size_t)(rows - 1) * (size_t)w->ldc + (size_t)code_width(cols) : 0u;
        n_scales = rows > 0 ? ((size_t)(rows - 1) * (size_t)w->lds + (size_t)((cols + w->group - 1) / w->group)) * 2u : 0u;
    }
    bool meets(const Matrix& m) const { return spans_meet(codes, n_codes, m.p, m.bytes()) || spans_meet(scales, n_scales, m.p, m.bytes()); }
};

struct PackLaunch : Launch {
    unsigned chunks;
    PackLaunch(int64_t rows, int64_t cols, cudaStream_t st) : Launch(dim3(1), 32 * kPackWarps, 0, st) {
        const int64_t wide = kPackWarps * kWarpCols;
        chunks = (unsigned)((cols + wide - 1) / wide);
        cfg.gridDim = dim3((unsigned)(chunks * ((rows + kPackRows - 1) / kPackRows)));
    }
};
int run_dequantize4(const Weight4& in, int64_t rows, int64_t cols, void* W, int64_t ldw, cudaStream_t st) {
    PackLaunch l(rows, cols, st);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, Matrix{W, rows, cols, ldw}.tma_ok() ? dequantize4_kernel<true> : dequantize4_kernel<false>, in, rows, cols,
                                       static_cast<uint16_t*>(W), ldw, l.chunks));
    return MOSAIC_OK;
}
int check_pack(const void* W, int64_t rows, int64_t cols, int64_t ldw, int dtype, const mosaic_weight4* w) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (rows < 0 || cols <= 0 || rows > kMostExtent || cols > kMostExtent || rows * (cols + 2048) > ((int64_t)1 << 41)) return MOSAIC_ERR_INVALID_ARG;
    const Matrix m{W, rows, cols, ldw};
    int rc;
    if ((rc = check_bf16(m)) != MOSAIC_OK || (rc = check_weight4(w, rows, cols)) != MOSAIC_OK) return rc;
    const Spans4 s(w, rows, cols);
    return s.meets(m) || spans_meet(s.codes, s.n_codes, s.scales, s.n_scales) ? MOSAIC_ERR_ALIASING : MOSAIC_OK;
}

// Few tokens are those whose X lies in shared memory beside the codes in flight of all warps: eight of 4096 columns, six of 8807.
// With fewer warps the kernel for more tokens is faster (eight tokens, 4096 outputs from 8807: 12.5 against 10.9 us).
constexpr size_t k4Smem = 212 * 1024;
size_t few4_x_bytes(int64_t tokens, int64_t cols) { return (size_t)tokens * ((size_t)((cols + k4Block - 1) / k4Block) * (k4Block * 2) + 64); }
bool is_few4(int64_t tokens, int64_t cols) { return tokens <= k4Tokens && cols <= (1 << 20) && few4_x_bytes(tokens, cols) + k4Warps * k4Ring <= k4Smem; }

// Beyond, a bf16 copy of the weights and mm.cuh's products.
constexpr int64_t kC4Tokens = 256;

// Scratch: an aligned copy of X if it is not; many tokens need the weights in bf16 as well.
size_t workspace4(const Matrix& x, int64_t outputs, int matrices) {
    size_t need = x.tma_ok() ? 0 : x.padded_bytes();
    if (x.rows > kC4Tokens) need += (size_t)matrices * Matrix{nullptr, outputs, x.cols, x.cols}.padded_bytes();
    return need;
}

template <bool GATE> int launch_few4(Few4Args a, cudaStream_t st) {
    constexpr int kOutputs = GATE ? k4Rows / 2 : k4Rows;
    static DeviceCache opted;
    if (opted.get([]() -> int {
            if (cudaFuncSetAttribute(few4_kernel<GATE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k4Smem) == cudaSuccess) return 1;
            (void)cudaGetLastError();
            return -1;
        }) < 0)
        return MOSAIC_ERR_CUDA;
    a.tiles = (int)((a.outputs + kOutputs - 1) / kOutputs);
    const int most = k4Warps, ctas = a.tiles < sm_count() ? a.tiles : sm_count(), blocks = (int)((a.cols + k4Block - 1) / k4Block);
    // How many warps share a tile and how many tiles a CTA has in hand: the fewest blocks one after another, and a few
    // more where sums meet.
    const int each = (a.tiles + ctas - 1) / ctas;
    int groups = 1;
    int64_t best = 0;
    for (int parts = 1; parts <= most && parts <= blocks; ++parts) {
        const int g = most / parts < each ? most / parts : each, turns = (each + g - 1) / g;
        const int64_t cost = (int64_t)turns * ((blocks + parts - 1) / parts + (parts > 1 ? 3 : 1));
        if (parts == 1 || cost < best) {
            best = cost;
            a.parts = parts;
            groups = (each + turns - 1) / turns;
        }
    }
    const int warps = groups * a.parts;
    Launch l(dim3((unsigned)ctas), 32 * warps, few4_x_bytes(a.tokens, a.cols) + warps * k4Ring, st);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, few4_kernel<GATE>, a));
    return MOSAIC_OK;
}

// Nanoseconds of 256 columns of a tile by its tokens, and the rest as in mm.cuh.
constexpr int64_t k4Step = 590, k4WideStep = 1050;

template <int BN, int MODE>
int launch_mm4(const mosaic_weight4* W, const mosaic_weight4* W2, const Matrix& x, MmArgs a, const GateArgs& g, int split, cudaStream_t st) {
    static_assert(kC4Slots<BN> * kC4Slot<BN> >= (BN + kMMaxSplit) * kMI * 4, "the partial sums lie where the stages were");
    static DeviceCache opted;
    if (opted.get([]() -> int {
            if (cudaFuncSetAttribute(mm4_kernel<BN, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kC4Smem<BN>) == cudaSuccess) return 1;
            (void)cudaGetLastError();
            return -1;
        }) < 0)
        return MOSAIC_ERR_CUDA;
    const int64_t width = code_width(a.n_c);
    CUtensorMap code_map, x_map;
    Second<MODE> second;
    if (!encode_bytes(&code_map, W->codes, a.n_i, width, W->ldc, MODE == kGate ? kGateRows : kMI) || !encode_bf16(&x_map, x.p, x.rows, x.cols, x.ld, BN, kMC))
        return MOSAIC_ERR_CUDA;
    const auto wide = [](const mosaic_weight4* w) {
        const int64_t n = kC4Cols / w->group;
        return w->lds % n == 0 && (reinterpret_cast<uintptr_t>(w->scales) & (uintptr_t)(2 * n - 1)) == 0 ? 1 : 0;
    };
    const auto groups = [&](const mosaic_weight4* w) { return (int)((a.n_c + w->group - 1) / w->group); };
    Scales4 s = {static_cast<const uint16_t*>(W->scales), nullptr, W->lds, 0, group_shift(W->group), 0, groups(W), 0, wide(W), 0};
    if constexpr (MODE == kGate) {
        second.g = g;
        if (!encode_bytes(&second.a, W2->codes, a.n_i, width, W2->ldc, kGateRows)) return MOSAIC_ERR_CUDA;
        s.p2 = static_cast<const uint16_t*>(W2->scales); s.ld2 = W2->lds; s.shift2 = group_shift(W2->group); s.groups2 = groups(W2); s.wide2 = wide(W2);
    }
    a.tiles_i = (int)((a.n_i + kTileI<MODE> - 1) / kTileI<MODE>);
    a.tiles_j = (int)((a.n_j + BN - 1) / BN);
    a.split = split;
    Launch l(dim3((unsigned)((int64_t)a.tiles_i * a.tiles_j * split)), kC4Threads<BN>, kC4Smem<BN>, st, split);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, mm4_kernel<BN, MODE>, code_map, x_map, a, second, s));
    return MOSAIC_OK;
}

template <int MODE> int run_mm4(const mosaic_weight4* W, const mosaic_weight4* W2, const Matrix& x, MmArgs a, const GateArgs& g, cudaStream_t st) {
    const auto even = [](const void* p, int64_t ld) { return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 3u) == 0 && ld % 2 == 0); };
    a.pairs = even(a.out, a.ld_out) && even(a.resid, a.ld_resid) ? 1 : 0;
    a.first_pair = -1;
    const int64_t ti = (a.n_i + kTileI<MODE> - 1) / kTileI<MODE>, steps = (a.n_c + kC4Cols - 1) / kC4Cols;
    int64_t best = 0;
    int bn = 16, split = 1;
    for (int w = 16; w <= 128; w *= 2) {
        const int64_t tiles = ti * ((a.n_j + w - 1) / w);
        for (int p = 1; p <= kMMaxSplit && (p == 1 || steps >= 2 * p); ++p) {
            const int64_t held = resident_clusters(p), waves = (tiles + held - 1) / held;
            const int64_t c = waves * ((steps + p - 1) / p * (w > 64 ? k4WideStep : k4Step) + w * kTileColumn + kFixed + (p > 1 ? kSplitFixed + w * kSplitColumn : 0));
            if (best == 0 || c < best) {
                best = c;
                bn = w;
                split = p;
            }
        }
        if (w >= a.n_j) break;
    }
    if (ti * ((a.n_j + bn - 1) / bn) * split > 0x7FFFFFFF) return MOSAIC_ERR_INVALID_ARG;
    switch (bn) {
        case 16: return launch_mm4<16, MODE>(W, W2, x, a, g, split, st);
        case 32: return launch_mm4<32, MODE>(W, W2, x, a, g, split, st);
        case 64: return launch_mm4<64, MODE>(W, W2, x, a, g, split, st);
        default: return launch_mm4<128, MODE>(W, W2, x, a, g, split, st);
    }
}
// The weights in bf16, in scratch.
int widen4(const mosaic_weight4* w, int64_t rows, int64_t cols, char** ws, Matrix* out, cudaStream_t st) {
    *out = {nullptr, rows, cols, cols};
    out->ld = out->padded_ld();
    out->p = *ws;
    *ws += out->padded_bytes();
    return run_dequantize4(as_weight4(w), rows, cols, const_cast<void*>(out->p), out->ld, st);
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" int mosaic_quantize4(const void* W, int64_t rows, int64_t cols, int64_t ldw, int dtype, const mosaic_weight4* out, void* stream) {
    const int rc = check_pack(W, rows, cols, ldw, dtype, out);
    if (rc != MOSAIC_OK || rows == 0) return rc;
    PackLaunch l(rows, cols, static_cast<cudaStream_t>(stream));
    using Kernel = void (*)(const uint16_t*, int64_t, int64_t, int64_t, Weight4, unsigned);
    static const Kernel kernels[2][3] = {{quantize4_kernel<false, 5>, quantize4_kernel<false, 6>, quantize4_kernel<false, 7>},
                                         {quantize4_kernel<true, 5>, quantize4_kernel<true, 6>, quantize4_kernel<true, 7>}};
    const Kernel kernel = kernels[Matrix{W, rows, cols, ldw}.tma_ok() ? 1 : 0][group_shift(out->group) - 5];
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, kernel, static_cast<const uint16_t*>(W), ldw, rows, cols, as_weight4(out), l.chunks));
    return MOSAIC_OK;
}

extern "C" int mosaic_dequantize4(const mosaic_weight4* in, int64_t rows, int64_t cols, void* W, int64_t ldw, int dtype, void* stream) {
    const int rc = check_pack(W, rows, cols, ldw, dtype, in);
    if (rc != MOSAIC_OK || rows == 0) return rc;
    return run_dequantize4(as_weight4(in), rows, cols, W, ldw, static_cast<cudaStream_t>(stream));
}

extern "C" size_t mosaic_linear4_workspace_bytes(const void* X, int64_t ldx, int64_t tokens, int64_t out_features, int64_t in_features) {
    if (!extents_ok(tokens, out_features, in_features)) return 0;
    return workspace4({X, tokens, in_features, ldx}, out_features, 1);
}

extern "C" size_t mosaic_gated_linear4_workspace_bytes(const void* X, int64_t ldx, int64_t tokens, int64_t channels, int64_t in_features) {
    if (!extents_ok(tokens, channels, in_features)) return 0;
    return workspace4({X, tokens, in_features, ldx}, channels, 2);
}

extern "C" int mosaic_linear4(const void* X, int64_t ldx, const mosaic_weight4* W, int64_t tokens, int64_t out_features, int64_t in_features, int dtype,
                              const void* bias, const void* residual, int64_t ldr, int act, void* Y, int64_t ldy, int* status_dev, void* ws,
                              size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (!extents_ok(tokens, out_features, in_features) || !act_ok(act)) return MOSAIC_ERR_INVALID_ARG;
    Matrix x{X, tokens, in_features, ldx};
    const Matrix y{Y, tokens, out_features, ldy}, r{residual, tokens, out_features, ldr}, b{bias, 1, out_features, out_features};
    int rc;
    if ((rc = check_bf16(x)) != MOSAIC_OK || (rc = check_bf16(y)) != MOSAIC_OK || (rc = check_weight4(W, out_features, in_features)) != MOSAIC_OK) return rc;
    if ((residual != nullptr && (rc = check_bf16(r)) != MOSAIC_OK) || (bias != nullptr && (rc = check_bf16(b)) != MOSAIC_OK)) return rc;
    if ((reinterpret_cast<uintptr_t>(status_dev) & 3u) != 0) return MOSAIC_ERR_MISALIGNED;
    if (overlap(y, x) || overlap(y, b) || Spans4(W, out_features, in_features).meets(y)) return MOSAIC_ERR_ALIASING;
    if (overlap(y, r) && !(residual == Y && ldr == ldy)) return MOSAIC_ERR_ALIASING;
    if ((rc = check_workspace(ws, ws_bytes, tokens > 0 ? workspace4(x, out_features, 1) : 0)) != MOSAIC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (status_dev != nullptr) MOSAIC_CUDA_TRY(cudaMemsetAsync(status_dev, 0, sizeof(int), st));
    if (tokens == 0) return MOSAIC_OK;
    char* scratch = static_cast<char*>(ws);
    if ((rc = readable(x, &scratch, st)) != MOSAIC_OK) return rc;
    if (is_few4(tokens, in_features)) {
        Few4Args a = {};
        a.x = static_cast<const uint16_t*>(x.p); a.ldx = x.ld;
        a.tokens = (int)tokens; a.outputs = out_features; a.cols = in_features;
        a.w = as_weight4(W);
        a.bias = static_cast<const uint16_t*>(bias);
        a.resid = static_cast<const uint16_t*>(residual); a.ld_resid = ldr;
        a.act = act;
        a.y = static_cast<uint16_t*>(Y); a.ldy = ldy;
        return launch_few4<false>(a, st);
    }
    MmArgs a = {};
    a.n_i = out_features; a.n_j = tokens; a.n_c = in_features;
    a.out = static_cast<uint16_t*>(Y); a.ld_out = ldy;
    a.bias = static_cast<const uint16_t*>(bias);
    a.resid = static_cast<const uint16_t*>(residual); a.ld_resid = ldr;
    a.act = act; a.status = status_dev;
    if (tokens <= kC4Tokens) return run_mm4<kPlain>(W, nullptr, x, a, GateArgs{}, st);
    Matrix w;
    if ((rc = widen4(W, out_features, in_features, &scratch, &w, st)) != MOSAIC_OK) return rc;
    return run_mm<false, false>(w, x, a, st);
}

extern "C" int mosaic_gated_linear4(const void* X, int64_t ldx, const mosaic_weight4* W_gate, const mosaic_weight4* W_up, int64_t tokens, int64_t channels,
                                    int64_t in_features, int dtype, const void* bias_gate, const void* bias_up, int act, void* H, int64_t ldh,
                                    int* status_dev, void* ws, size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (!extents_ok(tokens, channels, in_features) || !act_ok(act)) return MOSAIC_ERR_INVALID_ARG;
    Matrix x{X, tokens, in_features, ldx};
    const Matrix h{H, tokens, channels, ldh}, bg{bias_gate, 1, channels, channels}, bu{bias_up, 1, channels, channels};
    int rc;
    if ((rc = check_bf16(x)) != MOSAIC_OK || (rc = check_bf16(h)) != MOSAIC_OK) return rc;
    if ((rc = check_weight4(W_gate, channels, in_features)) != MOSAIC_OK || (rc = check_weight4(W_up, channels, in_features)) != MOSAIC_OK) return rc;
    if ((bias_gate != nullptr && (rc = check_bf16(bg)) != MOSAIC_OK) || (bias_up != nullptr && (rc = check_bf16(bu)) != MOSAIC_OK)) return rc;
    if ((reinterpret_cast<uintptr_t>(status_dev) & 3u) != 0) return MOSAIC_ERR_MISALIGNED;
    if (overlap(h, x) || overlap(h, bg) || overlap(h, bu) || Spans4(W_gate, channels, in_features).meets(h) || Spans4(W_up, channels, in_features).meets(h))
        return MOSAIC_ERR_ALIASING;
    if ((rc = check_workspace(ws, ws_bytes, tokens > 0 ? workspace4(x, channels, 2) : 0)) != MOSAIC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (status_dev != nullptr) MOSAIC_CUDA_TRY(cudaMemsetAsync(status_dev, 0, sizeof(int), st));
    if (tokens == 0) return MOSAIC_OK;
    char* scratch = static_cast<char*>(ws);
    if ((rc = readable(x, &scratch, st)) != MOSAIC_OK) return rc;
    if (is_few4(tokens, in_features)) {
        Few4Args a = {};
        a.x = static_cast<const uint16_t*>(x.p); a.ldx = x.ld;
        a.tokens = (int)tokens; a.outputs = channels; a.cols = in_features;
        a.w = as_weight4(W_gate);
        a.w2 = as_weight4(W_up);
        a.bias = static_cast<const uint16_t*>(bias_gate);
        a.bias2 = static_cast<const uint16_t*>(bias_up);
        a.act = act;
        a.y = static_cast<uint16_t*>(H); a.ldy = ldh;
        return launch_few4<true>(a, st);
    }
    MmArgs a = {};
    a.n_i = channels; a.n_j = tokens; a.n_c = in_features;
    a.out = static_cast<uint16_t*>(H); a.ld_out = ldh;
    a.bias = static_cast<const uint16_t*>(bias_gate);
    a.act = act; a.status = status_dev;
    Also also = {};
    also.gate.bias = static_cast<const uint16_t*>(bias_up);
    if (tokens <= kC4Tokens) return run_mm4<kGate>(W_gate, W_up, x, a, also.gate, st);
    Matrix wg, wu;
    if ((rc = widen4(W_gate, channels, in_features, &scratch, &wg, st)) != MOSAIC_OK || (rc = widen4(W_up, channels, in_features, &scratch, &wu, st)) != MOSAIC_OK) return rc;
    also.A = wu;
    return run_mm<false, false, kGate>(wg, x, a, st, also);
}
