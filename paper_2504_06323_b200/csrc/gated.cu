// mosaic_gated_linear / mosaic_gated_linear_backward: the gated pair of projections of a LLaMA-shaped MLP as one product, and its
// gradients.
//
//     forward    Z = X Wg^T + bg,  U = X Wu^T + bu,  H = act(Z) * U                    [tokens, channels]
//     backward   dZ = dH * U * act'(Z),  dU = dH * act(Z);   dX = dZ Wg + dU Wu
//                dWg = dZ^T X,  dWu = dU^T X,  db = sums over tokens of dZ and dU
//
// Forward: one launch of mm.cuh's kernels over both weight matrices, half of a tile's rows of either, so that the accumulators of
// both are in the same CTA and neither Z nor U needs to reach memory.  Backward: one elementwise pass makes dZ and dU (and H
// again), dX is one product over both contractions, dWg and dWu are one launch over both outputs.
#include "checkpoint.cuh"
#include "mm.cuh"

namespace mosaic {
namespace {

// act(z) and its slope.
__device__ __forceinline__ void activate_both(float z, int act, float& value, float& slope) {
    if (act == MOSAIC_ACT_SILU) {
        const float s = logistic(z);
        value = z * s;
        slope = s * (1.0f + z * (1.0f - s));
    } else if (act == MOSAIC_ACT_GELU) {
        const float bell = __expf(-0.5f * z * z), cdf = normal_cdf(z, bell);
        value = z * cdf;
        slope = cdf + z * bell * 0.39894228040143268f;
    } else {
        value = activate(z, act);
        slope = activate_slope(z, act);
    }
}

struct GatedSlope {
    const uint16_t *dh, *z, *u;        // z, u: bf16, or null where the checkpoints hold them
    int64_t ld_dh, ld_z, ld_u;
    Saved z8, u8;
    uint16_t *dz, *du;                 // rows on 16-byte boundaries, padded to whole vectors; or null
    int64_t ld_d;
    uint16_t* h;                       // act(z) u once more, or null
    int64_t ld_h;
    int64_t rows, cols, band;
    int act;
    float *z_sums, *u_sums;            // [bands, cols] column sums of the unrounded dz and du, with SUMS
};

// What a lane reads of a row.
template <bool VEC, bool SAVED> struct SlopeRow {
    uint32_t dh[4], z[SAVED ? 2 : 4], u[SAVED ? 2 : 4], ze, ue;
    __device__ __forceinline__ void load(const GatedSlope& a, int64_t r, int64_t c0, uint4* turn) {
        const int64_t c = c0 + ((int)threadIdx.x & 31) * kLaneCols;
        lane_load8<VEC, true>(a.dh + r * a.ld_dh, c0, a.cols, turn, dh);
        if constexpr (SAVED) {
            z[0] = z[1] = u[0] = u[1] = 0u;
            ze = ue = 1u;
            if (c < a.cols) {
                const uint2 zq = *reinterpret_cast<const uint2*>(a.z8.codes + r * a.z8.ldc + c), uq = *reinterpret_cast<const uint2*>(a.u8.codes + r * a.u8.ldc + c);
                z[0] = zq.x; z[1] = zq.y;
                u[0] = uq.x; u[1] = uq.y;
                ze = a.z8.exponents[r * a.z8.lde + c / kSavedGroup];
                ue = a.u8.exponents[r * a.u8.lde + c / kSavedGroup];
            }
        } else {
            lane_load8<VEC, true>(a.z + r * a.ld_z, c0, a.cols, turn, z);
            lane_load8<VEC, true>(a.u + r * a.ld_u, c0, a.cols, turn, u);
        }
    }
    __device__ __forceinline__ void values(float (&d)[8], float (&zv)[8], float (&uv)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) d[e] = half_of(dh, e);
        if constexpr (SAVED) {
            saved_values8(make_uint2(z[0], z[1]), ze, zv);
            saved_values8(make_uint2(u[0], u[1]), ue, uv);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                zv[e] = half_of(z, e);
                uv[e] = half_of(u, e);
            }
        }
    }
};

// A warp takes 256 columns, a lane eight of them, the CTA's eight warps every eighth row of its band, the next row on its way
// while one is computed; with SUMS the warps' column sums meet in shared memory in their order.  Bound by instructions (53 an
// element, issue 79 %) next to memory (48 %): 2048 x 13824 from 8 bits with H 57 us, of which 44 are the bytes; of odd rows by the
// loads' latency: 1001 x 8807 with sums 33 us (14).  Four CTAs an SM, but where sums take the
// registers of aligned rows: two there (44.7 with its product, 50.4 with four).
template <bool VEC, bool SAVED, bool SUMS>
__global__ void __launch_bounds__(32 * 8, VEC && SUMS ? 2 : 4) gated_slope_kernel(const __grid_constant__ GatedSlope a) {
    constexpr int kWarps = 8;
    __shared__ float sums[SUMS ? kWarps : 1][kWarpCols];
    __shared__ uint4 turns[VEC ? 1 : kWarps][kTurn];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* turn = turns[VEC ? 0 : warp];
    const int64_t c0 = (int64_t)blockIdx.x * kWarpCols, c = c0 + lane * kLaneCols;
    const int64_t r0 = (int64_t)blockIdx.y * a.band, r1 = r0 + a.band < a.rows ? r0 + a.band : a.rows;
    await_previous_kernel();
    float zs[8] = {}, us[8] = {};
    SlopeRow<VEC, SAVED> next;
    if (r0 + warp < r1) next.load(a, r0 + warp, c0, turn);
#pragma unroll 1
    for (int64_t r = r0 + warp; r < r1; r += kWarps) {
        float dh[8], z[8], u[8];
        next.values(dh, z, u);
        if (r + kWarps < r1) next.load(a, r + kWarps, c0, turn);
        // dz and du are rounded to bf16 here because the tensor cores take bf16; the column sums are not
        uint32_t pz[4], pu[4], ph[4];
        const auto pass = [&](int act) {
            float h[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float slope;
                activate_both(z[e], act, h[e], slope);
                z[e] = __fmul_rn(__fmul_rn(dh[e], u[e]), slope);
                dh[e] = __fmul_rn(dh[e], h[e]);
                h[e] = __fmul_rn(h[e], u[e]);
                if (SUMS) {
                    zs[e] = __fadd_rn(zs[e], z[e]);
                    us[e] = __fadd_rn(us[e], dh[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                pz[e] = pack2(z[2 * e], z[2 * e + 1]);
                pu[e] = pack2(dh[2 * e], dh[2 * e + 1]);
                ph[e] = pack2(h[2 * e], h[2 * e + 1]);
            }
        };
        switch (a.act) {   // one branch a row, then straight code
            case MOSAIC_ACT_SILU: pass(MOSAIC_ACT_SILU); break;
            case MOSAIC_ACT_GELU: pass(MOSAIC_ACT_GELU); break;
            case MOSAIC_ACT_RELU: pass(MOSAIC_ACT_RELU); break;
            default: pass(MOSAIC_ACT_NONE); break;
        }
        if (a.dz != nullptr && c < a.cols) {
            *reinterpret_cast<uint4*>(a.dz + r * a.ld_d + c) = make_uint4(pz[0], pz[1], pz[2], pz[3]);
            *reinterpret_cast<uint4*>(a.du + r * a.ld_d + c) = make_uint4(pu[0], pu[1], pu[2], pu[3]);
        }
        if (a.h != nullptr) lane_store8<VEC, true>(a.h + r * a.ld_h, c0, a.cols, turn, ph);
    }
    if constexpr (SUMS) {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[warp][lane * 8 + e] = which == 0 ? zs[e] : us[e];
            __syncthreads();
            const int64_t col = c0 + threadIdx.x;
            if (col >= a.cols) continue;
            float total = 0.0f;
            for (int w = 0; w < kWarps; ++w) total = __fadd_rn(total, sums[w][threadIdx.x]);
            (which == 0 ? a.z_sums : a.u_sums)[(int64_t)blockIdx.y * a.cols + col] = total;
        }
    }
}

// Sums over the bands: of dz and, in the grid's second half, of du.
__global__ void __launch_bounds__(kSumCols) gated_sums_kernel(const float* z_sums, const float* u_sums, int64_t bands, int64_t cols, uint16_t* z_out, uint16_t* u_out) {
    allow_next_kernel();
    await_previous_kernel();
    const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x;
    const float* from = blockIdx.y == 0 ? z_sums : u_sums;
    uint16_t* out = blockIdx.y == 0 ? z_out : u_out;
    if (c >= cols || out == nullptr) return;
    float sum = 0.0f;
#pragma unroll 8
    for (int64_t b = 0; b < bands; ++b) sum = __fadd_rn(sum, from[b * cols + c]);
    out[c] = f32_to_bf16(sum);
}

int run_gated_slope(const GatedSlope& a, bool vec, bool saved, void* dbias_gate, void* dbias_up, cudaStream_t st) {
    const bool sums = dbias_gate != nullptr || dbias_up != nullptr;
    const int64_t bands = bands_of(a.rows);
    if (bands > 0) {
        using Kernel = void (*)(GatedSlope);
        static const Kernel kernels[2][2][2] = {{{gated_slope_kernel<false, false, false>, gated_slope_kernel<false, false, true>},
                                                 {gated_slope_kernel<false, true, false>, gated_slope_kernel<false, true, true>}},
                                                {{gated_slope_kernel<true, false, false>, gated_slope_kernel<true, false, true>},
                                                 {gated_slope_kernel<true, true, false>, gated_slope_kernel<true, true, true>}}};
        Launch l(dim3((unsigned)((a.cols + kWarpCols - 1) / kWarpCols), (unsigned)bands), 32 * 8, 0, st);
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, kernels[vec ? 1 : 0][saved ? 1 : 0][sums ? 1 : 0], a));
    }
    if (sums) {
        Launch l(dim3((unsigned)((a.cols + kSumCols - 1) / kSumCols), 2), kSumCols, 0, st);
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, gated_sums_kernel, static_cast<const float*>(a.z_sums), static_cast<const float*>(a.u_sums), bands, a.cols,
                                           static_cast<uint16_t*>(dbias_gate), static_cast<uint16_t*>(dbias_up)));
    }
    return MOSAIC_OK;
}

size_t copy_bytes(const Matrix& m) { return m.tma_ok() ? 0 : m.padded_bytes(); }
Matrix plain(const Matrix& m) { return {nullptr, m.rows, m.cols, m.padded_ld()}; }   // where a call keeps one of its own

// Whether the kernel for few tokens takes a call.
bool few_tokens(const Matrix& x, const Matrix& wg, const Matrix& wu) { return x.rows <= (x.tma_ok() && wg.tma_ok() && wu.tma_ok() ? kFewVector : kFewTokens); }

size_t forward_workspace(const Matrix& x, const Matrix& wg, const Matrix& wu, bool saved) {
    size_t need = 0;
    const bool few = few_tokens(x, wg, wu);
    if (!few) need += copy_bytes(x) + copy_bytes(wg) + copy_bytes(wu);
    if (few && saved) need += 2 * Matrix{nullptr, x.rows, wg.rows, wg.rows}.padded_bytes();
    return need;
}
size_t backward_workspace(const Matrix& dh, const Matrix& x, bool x_saved, const Matrix& wg, const Matrix& wu, bool want_dx, bool want_dw, bool want_db) {
    size_t need = 0;
    if (want_dx || want_dw) need += 2 * dh.padded_bytes();
    if (want_dw) need += x_saved ? x.padded_bytes() : copy_bytes(x);
    if (want_dx) need += copy_bytes(wg) + copy_bytes(wu);
    if (want_db) need += 2 * align_up((size_t)bands_of(dh.rows) * (size_t)dh.cols * 4u, 256);
    return need;
}

struct Span {
    const void* p;
    size_t n;
};
Span span(const Matrix& m) { return {m.p, m.bytes()}; }
bool meet(const Span& a, const Span& b) { return spans_meet(a.p, a.n, b.p, b.n); }

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" size_t mosaic_gated_linear_workspace_bytes(const void* X, int64_t ldx, const void* W_gate, int64_t ld_gate, const void* W_up, int64_t ld_up,
                                                      int64_t tokens, int64_t channels, int64_t in_features, int saved) {
    if (!extents_ok(tokens, channels, in_features)) return 0;
    return forward_workspace({X, tokens, in_features, ldx}, {W_gate, channels, in_features, ld_gate}, {W_up, channels, in_features, ld_up}, saved != 0);
}

extern "C" int mosaic_gated_linear(const void* X, int64_t ldx, const void* W_gate, int64_t ld_gate, const void* W_up, int64_t ld_up, int64_t tokens,
                                   int64_t channels, int64_t in_features, int dtype, const void* bias_gate, const void* bias_up, int act, void* H,
                                   int64_t ldh, void* Z, int64_t ldz, void* U, int64_t ldu, const mosaic_checkpoint* z_saved,
                                   const mosaic_checkpoint* u_saved, int* status_dev, void* ws, size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (!extents_ok(tokens, channels, in_features) || !act_ok(act)) return MOSAIC_ERR_INVALID_ARG;
    const bool saved = z_saved != nullptr || u_saved != nullptr;
    if (saved && (z_saved == nullptr || u_saved == nullptr || Z != nullptr || U != nullptr)) return MOSAIC_ERR_INVALID_ARG;
    Matrix x{X, tokens, in_features, ldx}, wg{W_gate, channels, in_features, ld_gate}, wu{W_up, channels, in_features, ld_up};
    Matrix h{H, tokens, channels, ldh}, z{Z, tokens, channels, ldz}, u{U, tokens, channels, ldu};
    const Matrix bg{bias_gate, 1, channels, channels}, bu{bias_up, 1, channels, channels};
    int rc;
    if ((rc = check_bf16(x)) != MOSAIC_OK || (rc = check_bf16(wg)) != MOSAIC_OK || (rc = check_bf16(wu)) != MOSAIC_OK || (rc = check_bf16(h)) != MOSAIC_OK) return rc;
    if ((Z != nullptr && (rc = check_bf16(z)) != MOSAIC_OK) || (U != nullptr && (rc = check_bf16(u)) != MOSAIC_OK)) return rc;
    if ((bias_gate != nullptr && (rc = check_bf16(bg)) != MOSAIC_OK) || (bias_up != nullptr && (rc = check_bf16(bu)) != MOSAIC_OK)) return rc;
    if (saved && ((rc = check_saved(z_saved, tokens, channels)) != MOSAIC_OK || (rc = check_saved(u_saved, tokens, channels)) != MOSAIC_OK)) return rc;
    if ((reinterpret_cast<uintptr_t>(status_dev) & 3u) != 0) return MOSAIC_ERR_MISALIGNED;
    {   // outputs overlap neither inputs nor one another
        const Span in[5] = {span(x), span(wg), span(wu), span(bg), span(bu)};
        Span out[7] = {span(h), span(z), span(u), {}, {}, {}, {}};
        if (saved) {
            const Saved s[2] = {as_saved(z_saved), as_saved(u_saved)};
            for (int k = 0; k < 2; ++k) {
                out[3 + 2 * k] = {s[k].codes, saved_code_bytes(s[k], tokens, channels)};
                out[4 + 2 * k] = {s[k].exponents, saved_exponent_bytes(s[k], tokens, channels)};
            }
        }
        for (int o = 0; o < 7; ++o) {
            for (const Span& i : in)
                if (meet(out[o], i)) return MOSAIC_ERR_ALIASING;
            for (int i = o + 1; i < 7; ++i)
                if (meet(out[o], out[i])) return MOSAIC_ERR_ALIASING;
        }
    }
    if ((rc = check_workspace(ws, ws_bytes, tokens > 0 ? forward_workspace(x, wg, wu, saved) : 0)) != MOSAIC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (status_dev != nullptr) MOSAIC_CUDA_TRY(cudaMemsetAsync(status_dev, 0, sizeof(int), st));
    if (tokens == 0) return MOSAIC_OK;
    char* scratch = static_cast<char*>(ws);
    const bool few = few_tokens(x, wg, wu), two_steps = few && saved;   // few tokens: through bf16, whose groups are other warps' too
    if (two_steps) {
        z = u = plain(h);
        z.p = scratch;
        u.p = scratch + z.padded_bytes();
        scratch += 2 * z.padded_bytes();
    }
    MmArgs a = {};
    a.n_i = channels; a.n_j = tokens; a.n_c = in_features;
    a.out = static_cast<uint16_t*>(H); a.ld_out = ldh;
    a.bias = static_cast<const uint16_t*>(bias_gate);
    a.z = static_cast<uint16_t*>(const_cast<void*>(z.p)); a.ld_z = z.ld;
    a.act = act; a.status = status_dev;
    GateArgs g = {};
    g.w = static_cast<const uint16_t*>(W_up); g.ld_w = ld_up;
    g.bias = static_cast<const uint16_t*>(bias_up);
    g.u = static_cast<uint16_t*>(const_cast<void*>(u.p)); g.ld_u = u.ld;
    if (saved && !few) {
        g.z8 = as_saved(z_saved);
        g.u8 = as_saved(u_saved);
    }
    if (few) {
        if ((rc = launch_few<true>(x, wg, a, st, g)) != MOSAIC_OK) return rc;
    } else {
        if ((rc = readable(x, &scratch, st)) != MOSAIC_OK || (rc = readable(wg, &scratch, st)) != MOSAIC_OK || (rc = readable(wu, &scratch, st)) != MOSAIC_OK) return rc;
        Also also = {};
        also.A = wu;
        also.gate = g;
        if ((rc = run_mm<false, false, kGate>(wg, x, a, st, also)) != MOSAIC_OK) return rc;
    }
    if (two_steps) {
        if ((rc = store_saved(z.p, z.ld, tokens, channels, as_saved(z_saved), st)) != MOSAIC_OK) return rc;
        if ((rc = store_saved(u.p, u.ld, tokens, channels, as_saved(u_saved), st)) != MOSAIC_OK) return rc;
    }
    return MOSAIC_OK;
}

extern "C" size_t mosaic_gated_linear_backward_workspace_bytes(const void* X, int64_t ldx, int x_saved, const void* W_gate, int64_t ld_gate,
                                                               const void* W_up, int64_t ld_up, int64_t tokens, int64_t channels, int64_t in_features,
                                                               int want_dx, int want_dw, int want_dbias) {
    if (!extents_ok(tokens, channels, in_features)) return 0;
    return backward_workspace({nullptr, tokens, channels, channels}, {X, tokens, in_features, ldx}, x_saved != 0, {W_gate, channels, in_features, ld_gate},
                              {W_up, channels, in_features, ld_up}, want_dx != 0, want_dw != 0, want_dbias != 0);
}

extern "C" int mosaic_gated_linear_backward(const void* dH, int64_t lddh, const void* X, int64_t ldx, const mosaic_checkpoint* x_saved, const void* W_gate,
                                            int64_t ld_gate, const void* W_up, int64_t ld_up, const void* Z, int64_t ldz, const void* U, int64_t ldu,
                                            const mosaic_checkpoint* z_saved, const mosaic_checkpoint* u_saved, int64_t tokens, int64_t channels,
                                            int64_t in_features, int dtype, int act, void* dX, int64_t lddx, void* dW_gate, int64_t lddwg, void* dW_up,
                                            int64_t lddwu, void* dbias_gate, void* dbias_up, void* H, int64_t ldh, int* status_dev, void* ws,
                                            size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (!extents_ok(tokens, channels, in_features) || !act_ok(act)) return MOSAIC_ERR_INVALID_ARG;
    const bool saved = z_saved != nullptr || u_saved != nullptr, want_dw = dW_gate != nullptr || dW_up != nullptr, want_db = dbias_gate != nullptr || dbias_up != nullptr;
    if (saved && (z_saved == nullptr || u_saved == nullptr || Z != nullptr || U != nullptr)) return MOSAIC_ERR_INVALID_ARG;
    if (x_saved != nullptr && X != nullptr) return MOSAIC_ERR_INVALID_ARG;
    const Matrix dh{dH, tokens, channels, lddh}, z{Z, tokens, channels, ldz}, u{U, tokens, channels, ldu}, h{H, tokens, channels, ldh};
    Matrix x{X, tokens, in_features, ldx}, wg{W_gate, channels, in_features, ld_gate}, wu{W_up, channels, in_features, ld_up};
    const Matrix dx{dX, tokens, in_features, lddx}, dwg{dW_gate, channels, in_features, lddwg}, dwu{dW_up, channels, in_features, lddwu};
    const Matrix dbg{dbias_gate, 1, channels, channels}, dbu{dbias_up, 1, channels, channels};
    int rc;
    if ((rc = check_bf16(dh)) != MOSAIC_OK) return rc;
    if (!saved && ((rc = check_bf16(z)) != MOSAIC_OK || (rc = check_bf16(u)) != MOSAIC_OK)) return rc;
    if (saved && ((rc = check_saved(z_saved, tokens, channels)) != MOSAIC_OK || (rc = check_saved(u_saved, tokens, channels)) != MOSAIC_OK)) return rc;
    if (want_dw && (rc = x_saved != nullptr ? check_saved(x_saved, tokens, in_features) : check_bf16(x)) != MOSAIC_OK) return rc;
    if (dX != nullptr && ((rc = check_bf16(wg)) != MOSAIC_OK || (rc = check_bf16(wu)) != MOSAIC_OK || (rc = check_bf16(dx)) != MOSAIC_OK)) return rc;
    if ((dW_gate != nullptr && (rc = check_bf16(dwg)) != MOSAIC_OK) || (dW_up != nullptr && (rc = check_bf16(dwu)) != MOSAIC_OK)) return rc;
    if ((dbias_gate != nullptr && (rc = check_bf16(dbg)) != MOSAIC_OK) || (dbias_up != nullptr && (rc = check_bf16(dbu)) != MOSAIC_OK)) return rc;
    if (H != nullptr && (rc = check_bf16(h)) != MOSAIC_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(status_dev) & 3u) != 0) return MOSAIC_ERR_MISALIGNED;
    {
        Span in[12] = {span(dh)};
        int n = 1;
        const auto codes = [&](const mosaic_checkpoint* c, int64_t cols) {
            const Saved s = as_saved(c);
            in[n++] = {s.codes, saved_code_bytes(s, tokens, cols)};
            in[n++] = {s.exponents, saved_exponent_bytes(s, tokens, cols)};
        };
        if (saved) {
            codes(z_saved, channels);
            codes(u_saved, channels);
        } else {
            in[n++] = span(z);
            in[n++] = span(u);
        }
        if (want_dw && x_saved != nullptr) codes(x_saved, in_features);
        else if (want_dw) in[n++] = span(x);
        if (dX != nullptr) {
            in[n++] = span(wg);
            in[n++] = span(wu);
        }
        const Span out[6] = {span(dx), span(dwg), span(dwu), span(dbg), span(dbu), span(h)};
        for (int o = 0; o < 6; ++o) {
            for (int i = 0; i < n; ++i)
                if (meet(out[o], in[i])) return MOSAIC_ERR_ALIASING;
            for (int i = o + 1; i < 6; ++i)
                if (meet(out[o], out[i])) return MOSAIC_ERR_ALIASING;
        }
    }
    if ((rc = check_workspace(ws, ws_bytes, backward_workspace(dh, x, x_saved != nullptr, wg, wu, dX != nullptr, want_dw, want_db))) != MOSAIC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (status_dev != nullptr) MOSAIC_CUDA_TRY(cudaMemsetAsync(status_dev, 0, sizeof(int), st));
    char* scratch = static_cast<char*>(ws);
    GatedSlope s = {};
    s.dh = static_cast<const uint16_t*>(dH); s.ld_dh = lddh;
    s.z = static_cast<const uint16_t*>(Z); s.ld_z = ldz;
    s.u = static_cast<const uint16_t*>(U); s.ld_u = ldu;
    if (saved) {
        s.z8 = as_saved(z_saved);
        s.u8 = as_saved(u_saved);
    }
    s.h = static_cast<uint16_t*>(H); s.ld_h = ldh;
    s.rows = tokens; s.cols = channels; s.band = band_rows(tokens); s.act = act;
    const int64_t bands = bands_of(tokens);
    if (want_db) {
        const size_t sums = align_up((size_t)bands * (size_t)channels * 4u, 256);
        s.z_sums = reinterpret_cast<float*>(scratch);
        s.u_sums = reinterpret_cast<float*>(scratch + sums);
        scratch += 2 * sums;
    }
    Matrix dz = plain(dh), du = plain(dh);
    if (dX != nullptr || want_dw) {
        dz.p = s.dz = reinterpret_cast<uint16_t*>(scratch);
        du.p = s.du = reinterpret_cast<uint16_t*>(scratch + dz.padded_bytes());
        s.ld_d = dz.ld;
        scratch += 2 * dz.padded_bytes();
    }
    const bool vec = dh.tma_ok() && (saved || (z.tma_ok() && u.tma_ok())) && (H == nullptr || h.tma_ok());
    if (dX != nullptr || want_dw || want_db || H != nullptr)
        if ((rc = run_gated_slope(s, vec, saved, dbias_gate, dbias_up, st)) != MOSAIC_OK) return rc;
    if (tokens == 0) {   // empty sums
        const size_t wide = (size_t)in_features * 2u;
        if (dW_gate != nullptr) MOSAIC_CUDA_TRY(cudaMemset2DAsync(dW_gate, (size_t)lddwg * 2u, 0, wide, (size_t)channels, st));
        if (dW_up != nullptr) MOSAIC_CUDA_TRY(cudaMemset2DAsync(dW_up, (size_t)lddwu * 2u, 0, wide, (size_t)channels, st));
        return MOSAIC_OK;
    }
    if (dX != nullptr) {
        if ((rc = readable(wg, &scratch, st)) != MOSAIC_OK || (rc = readable(wu, &scratch, st)) != MOSAIC_OK) return rc;
        MmArgs a = {};
        a.n_i = in_features; a.n_j = tokens; a.n_c = channels;
        a.out = static_cast<uint16_t*>(dX); a.ld_out = lddx; a.status = status_dev;
        Also also = {};
        also.A = wu;
        also.B = du;
        if ((rc = run_mm<true, false, kSum>(wg, dz, a, st, also)) != MOSAIC_OK) return rc;
    }
    if (want_dw) {
        if (x_saved != nullptr) {
            x.p = scratch;
            x.ld = x.padded_ld();
            if ((rc = load_saved(as_saved(x_saved), tokens, in_features, scratch, x.ld, st)) != MOSAIC_OK) return rc;
            scratch += x.padded_bytes();
        } else if ((rc = readable(x, &scratch, st)) != MOSAIC_OK) {
            return rc;
        }
        MmArgs a = {};
        a.n_i = in_features; a.n_j = channels; a.n_c = tokens; a.status = status_dev;
        a.out = static_cast<uint16_t*>(dW_gate != nullptr ? dW_gate : dW_up);
        a.ld_out = dW_gate != nullptr ? lddwg : lddwu;
        if (dW_gate != nullptr && dW_up != nullptr) {
            Also also = {};
            also.B = du;
            also.out = static_cast<uint16_t*>(dW_up);
            also.ld_out = lddwu;
            rc = run_mm<true, true, kTwin>(x, dz, a, st, also);
        } else {
            rc = run_mm<true, true>(x, dW_gate != nullptr ? dz : du, a, st);
        }
    }
    return rc;
}
