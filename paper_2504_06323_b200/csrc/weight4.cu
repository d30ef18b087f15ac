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
// A warp takes 256 columns, a lane eight of them, 4 to 16 lanes a group; kPackRows rows in flight.
constexpr int kPackWarps = 8, kPackRows = 4;

__device__ __forceinline__ float scale_of(float largest) {
    const float ideal = __fdiv_rn(largest, 7.0f);
    if (!(ideal <= 1.0633824e37f)) return ideal != ideal ? ideal : 1.0633824e37f;   // 2^123: 24 s below stays finite
    if (ideal < 1.17549435e-38f) return 0.0f;                                       // below bf16's normal numbers
    uint32_t u = __float_as_uint(ideal);
    u += 0x3FFFFu + ((u >> 19) & 1u);
    return __uint_as_float(u & 0xFFF80000u);
}

template <bool VEC>
__global__ void __launch_bounds__(32 * kPackWarps) quantize4_kernel(const uint16_t* W, int64_t ldw, int64_t rows, int64_t cols, const __grid_constant__ Weight4 out,
                                                                    unsigned chunks) {
    __shared__ uint4 turns[VEC ? 1 : kPackWarps][32];
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
        uint32_t bits = 0;   // of the largest magnitude: infinities and NaN are above all numbers
#pragma unroll
        for (int e = 0; e < 4; ++e) bits = max(bits, max(w[r][e] & 0x7FFFu, (w[r][e] >> 16) & 0x7FFFu));
        for (int o = 1; o < 1 << (out.shift - 3); o <<= 1) bits = max(bits, __shfl_xor_sync(0xFFFFFFFFu, bits, o));
        const float s = bits >= 0x7F80u ? __uint_as_float(0x7FC00000u) : scale_of(bf16_to_f32((uint16_t)bits));
        if (r0 + r >= rows || c >= (cols + 31) / 32 * 32) continue;
        uint32_t packed = 0x88888888u;
        if (s > 0.0f) {
            packed = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int q = min(7, max(-7, __float2int_rn(__fdiv_rn(half_of(w[r], e), s))));
                packed |= (uint32_t)(q + 8) << (4 * e);
            }
        }
        *reinterpret_cast<uint32_t*>(out.codes + (r0 + r) * out.ldc + c / 2) = packed;
        if ((c & ((1 << out.shift) - 1)) == 0 && c < cols) out.scales[(r0 + r) * out.lds + (c >> out.shift)] = (uint16_t)(__float_as_uint(s) >> 16);
    }
}

template <bool VEC>
__global__ void __launch_bounds__(32 * kPackWarps) dequantize4_kernel(const __grid_constant__ Weight4 in, int64_t rows, int64_t cols, uint16_t* W, int64_t ldw,
                                                                      unsigned chunks) {
    __shared__ uint4 turns[VEC ? 1 : kPackWarps][32];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* turn = turns[VEC ? 0 : warp];
    const int64_t c0 = ((int64_t)(blockIdx.x % chunks) * kPackWarps + warp) * kWarpCols, c = c0 + lane * kLaneCols;
    const int64_t r0 = (int64_t)(blockIdx.x / chunks) * kPackRows;
    if (c0 >= cols) return;
    await_previous_kernel();
    uint32_t q[kPackRows];
    float s[kPackRows];
#pragma unroll
    for (int r = 0; r < kPackRows; ++r) {
        const int64_t row = r0 + r < rows ? r0 + r : rows - 1;
        q[r] = 0x88888888u;
        s[r] = 0.0f;
        if (c < cols) {
            q[r] = *reinterpret_cast<const uint32_t*>(in.codes + row * in.ldc + c / 2);
            s[r] = bf16_to_f32(in.scales[row * in.lds + (c >> in.shift)]);
        }
    }
#pragma unroll
    for (int r = 0; r < kPackRows; ++r) {
        if (r0 + r >= rows) break;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = __fmul_rn((float)((int)((q[r] >> (4 * e)) & 15u) - 8), s[r]);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_bf16(v[2 * e], v[2 * e + 1]);   // exact
        lane_store8<VEC>(W + (r0 + r) * ldw, c0, cols, turn, w);
    }
}

// ---------------------------------------------------------------- few tokens
// The next tokens of up to k4Tokens sequences: the weights are read once, and what counts is that they stream.  A CTA takes 16
// weight rows - with GATE eight of each matrix, so that one lane has both sums of a channel - and its warps deal out blocks of
// 128 columns.  A lane loads 16 bytes, 32 codes, of two rows; each pair of codes becomes two bf16 weights in three
// instructions: shifted to bits 3..6 of its half, put under the exponent of 16, which makes it 16 + (code + 8), and one fma,
// (16 + n) s - 24 s, exact because s has five bits and 24 two.  The matrix instruction (16 rows, 8 tokens, 16 columns) does
// not mind which columns it is given as long as both operands agree: a lane's own 32 columns, in the order that the
// shifts yield, so neither operand moves between lanes.  Sums in fp32; over the warps in their order.
constexpr int k4Warps = 8, k4Tokens = 32, k4Rows = 16, k4Block = 128;

struct Few4Args {
    const uint16_t* x;                 // rows on 16-byte boundaries
    int64_t ldx, tokens, outputs, cols;
    Weight4 w, w2;                     // w2: GATE
    const uint16_t *bias, *bias2, *resid;
    int64_t ld_resid;
    int act;
    uint16_t* y;
    int64_t ldy;
};

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
// Codes i and i + 4 of a word (i = 0..3) as two bf16 weights; s2 and c2 hold s and -24 s twice.
__device__ __forceinline__ uint32_t weights4(uint32_t word, int i, uint32_t s2, uint32_t c2) {
    const uint32_t at = i == 0 ? word << 3 : word >> (4 * i - 3);
    return fma_bf16x2((at & 0x00780078u) | 0x41804180u, s2, c2);
}
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int NT, bool GATE>
__global__ void __launch_bounds__(32 * k4Warps) few4_kernel(const __grid_constant__ Few4Args a) {
    constexpr int kOutputs = GATE ? k4Rows / 2 : k4Rows, kCells = k4Rows * 8 * NT, kAhead = NT == 1 ? 4 : 2;
    __shared__ float part[k4Warps][kCells];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t o0 = (int64_t)blockIdx.x * kOutputs;
    // the lane's two rows: past the end the first again, not stored
    const int64_t lo = o0 + g < a.outputs ? o0 + g : o0, hi = GATE ? lo : (o0 + g + 8 < a.outputs ? o0 + g + 8 : o0);
    const Weight4& second = GATE ? a.w2 : a.w;
    const uint8_t *code0 = a.w.codes + lo * a.w.ldc, *code1 = second.codes + hi * second.ldc;
    const uint16_t *scale0 = a.w.scales + lo * a.w.lds, *scale1 = second.scales + hi * second.lds;
    float acc[NT][4] = {};
    await_previous_kernel();
    const int blocks = (int)((a.cols + k4Block - 1) / k4Block);
#pragma unroll 1
    for (int b0 = warp; b0 < blocks; b0 += k4Warps * kAhead) {
        uint4 q0[kAhead], q1[kAhead];
        uint32_t s0[kAhead], s1[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t k = (int64_t)(b0 + u * k4Warps) * k4Block + t * 32;
            q0[u] = q1[u] = make_uint4(0u, 0u, 0u, 0u);
            s0[u] = s1[u] = 0u;
            if (k < a.cols) {
                q0[u] = ld_stream16(code0 + (k >> 1));
                q1[u] = ld_stream16(code1 + (k >> 1));
                s0[u] = scale0[k >> a.w.shift];
                s1[u] = scale1[k >> second.shift];
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (b0 + u * k4Warps >= blocks) break;
            const int64_t k = (int64_t)(b0 + u * k4Warps) * k4Block + t * 32;
            const uint32_t sa = s0[u] | (s0[u] << 16), sb = s1[u] | (s1[u] << 16);
            const uint32_t ca = fma_bf16x2(sa, 0xC1C0C1C0u, 0x80008000u), cb = fma_bf16x2(sb, 0xC1C0C1C0u, 0x80008000u);   // -24 s
#pragma unroll
            for (int wd = 0; wd < 4; ++wd) {
                const uint32_t wa = wd == 0 ? q0[u].x : wd == 1 ? q0[u].y : wd == 2 ? q0[u].z : q0[u].w;
                const uint32_t wb = wd == 0 ? q1[u].x : wd == 1 ? q1[u].y : wd == 2 ? q1[u].z : q1[u].w;
                uint32_t fa[4], fb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    fa[i] = weights4(wa, i, sa, ca);
                    fb[i] = weights4(wb, i, sb, cb);
                }
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    uint32_t x[4] = {0u, 0u, 0u, 0u};
                    const int64_t token = n * 8 + g, c = k + wd * 8;
                    if (token < a.tokens) load8<true>(a.x + token * a.ldx, c, a.cols, x);
                    // elements (0, 4), (1, 5), (2, 6), (3, 7), as the codes come
                    mma_16816(acc[n], fa[0], fb[0], fa[1], fb[1], __byte_perm(x[0], x[2], 0x5410), __byte_perm(x[0], x[2], 0x7632));
                    mma_16816(acc[n], fa[2], fb[2], fa[3], fb[3], __byte_perm(x[1], x[3], 0x5410), __byte_perm(x[1], x[3], 0x7632));
                }
            }
        }
    }
    // a lane holds rows g and g + 8 of tokens 2 t and 2 t + 1
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[warp][(n * 8 + 2 * t + (e & 1)) * k4Rows + g + (e >> 1) * 8] = acc[n][e];
    __syncthreads();
    for (int at = threadIdx.x; at < kOutputs * 8 * NT; at += 32 * k4Warps) {
        const int token = at / kOutputs, r = at % kOutputs;
        const int64_t o = o0 + r;
        if (token >= a.tokens || o >= a.outputs) continue;
        float v = 0.0f, u = 0.0f;
        for (int w = 0; w < k4Warps; ++w) v = __fadd_rn(v, part[w][token * k4Rows + r]);
        v = __fadd_rn(v, a.bias != nullptr ? bf16_to_f32(a.bias[o]) : 0.0f);
        v = activate(v, a.act);
        if (GATE) {
            for (int w = 0; w < k4Warps; ++w) u = __fadd_rn(u, part[w][token * k4Rows + r + 8]);
            v = __fmul_rn(v, __fadd_rn(u, a.bias2 != nullptr ? bf16_to_f32(a.bias2[o]) : 0.0f));
        }
        if (a.resid != nullptr) v = __fadd_rn(v, bf16_to_f32(a.resid[token * a.ld_resid + o]));
        a.y[token * a.ldy + o] = f32_to_bf16(v);
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

// Scratch: few tokens need an aligned copy of X if it is not; many need the weights in bf16 as well.
size_t workspace4(const Matrix& x, int64_t outputs, int matrices) {
    size_t need = x.tma_ok() ? 0 : x.padded_bytes();
    if (x.rows > k4Tokens) need += (size_t)matrices * Matrix{nullptr, outputs, x.cols, x.cols}.padded_bytes();
    return need;
}

template <bool GATE> int launch_few4(const Few4Args& a, cudaStream_t st) {
    constexpr int kOutputs = GATE ? k4Rows / 2 : k4Rows;
    Launch l(dim3((unsigned)((a.outputs + kOutputs - 1) / kOutputs)), 32 * k4Warps, 0, st);
    const auto kernel = a.tokens <= 8 ? few4_kernel<1, GATE> : a.tokens <= 16 ? few4_kernel<2, GATE> : few4_kernel<4, GATE>;
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, kernel, a));
    return MOSAIC_OK;
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
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, Matrix{W, rows, cols, ldw}.tma_ok() ? quantize4_kernel<true> : quantize4_kernel<false>,
                                       static_cast<const uint16_t*>(W), ldw, rows, cols, as_weight4(out), l.chunks));
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
    if (tokens <= k4Tokens) {
        Few4Args a = {};
        a.x = static_cast<const uint16_t*>(x.p); a.ldx = x.ld;
        a.tokens = tokens; a.outputs = out_features; a.cols = in_features;
        a.w = as_weight4(W);
        a.bias = static_cast<const uint16_t*>(bias);
        a.resid = static_cast<const uint16_t*>(residual); a.ld_resid = ldr;
        a.act = act;
        a.y = static_cast<uint16_t*>(Y); a.ldy = ldy;
        return launch_few4<false>(a, st);
    }
    Matrix w;
    if ((rc = widen4(W, out_features, in_features, &scratch, &w, st)) != MOSAIC_OK) return rc;
    MmArgs a = {};
    a.n_i = out_features; a.n_j = tokens; a.n_c = in_features;
    a.out = static_cast<uint16_t*>(Y); a.ld_out = ldy;
    a.bias = static_cast<const uint16_t*>(bias);
    a.resid = static_cast<const uint16_t*>(residual); a.ld_resid = ldr;
    a.act = act; a.status = status_dev;
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
    if (tokens <= k4Tokens) {
        Few4Args a = {};
        a.x = static_cast<const uint16_t*>(x.p); a.ldx = x.ld;
        a.tokens = tokens; a.outputs = channels; a.cols = in_features;
        a.w = as_weight4(W_gate);
        a.w2 = as_weight4(W_up);
        a.bias = static_cast<const uint16_t*>(bias_gate);
        a.bias2 = static_cast<const uint16_t*>(bias_up);
        a.act = act;
        a.y = static_cast<uint16_t*>(H); a.ldy = ldh;
        return launch_few4<true>(a, st);
    }
    Matrix wg, wu;
    if ((rc = widen4(W_gate, channels, in_features, &scratch, &wg, st)) != MOSAIC_OK || (rc = widen4(W_up, channels, in_features, &scratch, &wu, st)) != MOSAIC_OK) return rc;
    MmArgs a = {};
    a.n_i = channels; a.n_j = tokens; a.n_c = in_features;
    a.out = static_cast<uint16_t*>(H); a.ld_out = ldh;
    a.bias = static_cast<const uint16_t*>(bias_gate);
    a.act = act; a.status = status_dev;
    Also also = {};
    also.A = wu;
    also.gate.bias = static_cast<const uint16_t*>(bias_up);
    return run_mm<false, false, kGate>(wg, x, a, st, also);
}
