// mosaic_linear / mosaic_linear_backward: a projection's matrix product with its bias, activation and residual
// in the epilogue, and the three products of its gradient - all on the tensor cores (bf16 in, fp32 sums).
//
//     forward    Z = X W^T + b,  Y = act(Z) + R          [tokens, out]
//     backward   dZ = dY * act'(Z);  dX = dZ W  [tokens, in],  dW = dZ^T X  [out, in],  db = sum over tokens of dZ
//
// The kernels are in mm.cuh.
#include "mm.cuh"

namespace mosaic {
namespace {

size_t backward_workspace(const Matrix& dY, const Matrix& X, const Matrix& W, int act, bool want_dx, bool want_dw, bool want_db) {
    size_t need = 0;
    if (want_dx || want_dw) {
        if (act != MOSAIC_ACT_NONE || !dY.tma_ok()) need += dY.padded_bytes();
        if (want_dw && !X.tma_ok()) need += X.padded_bytes();
        if (want_dx && !W.tma_ok()) need += W.padded_bytes();
    }
    if (want_db) need += align_up((size_t)bands_of(dY.rows) * (size_t)dY.cols * 4u, 256);
    return need;
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" size_t mosaic_linear_workspace_bytes(const void* X, int64_t ldx, const void* W, int64_t ldw, int64_t tokens, int64_t out_features,
                                                int64_t in_features) {
    if (!extents_ok(tokens, out_features, in_features)) return 0;
    if (tokens <= kFewTokens) return 0;   // read as they are
    const Matrix x{X, tokens, in_features, ldx}, w{W, out_features, in_features, ldw};
    return (x.tma_ok() ? 0 : x.padded_bytes()) + (w.tma_ok() ? 0 : w.padded_bytes());
}

extern "C" int mosaic_linear(const void* X, int64_t ldx, const void* W, int64_t ldw, int64_t tokens, int64_t out_features, int64_t in_features,
                             int dtype, const void* bias, const void* residual, int64_t ldr, int act, void* Y, int64_t ldy, void* Z, int64_t ldz,
                             int* status_dev, void* ws, size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;   // bf16 products are exact in fp32; fp32 ones are not
    if (!extents_ok(tokens, out_features, in_features) || !act_ok(act)) return MOSAIC_ERR_INVALID_ARG;
    Matrix x{X, tokens, in_features, ldx}, w{W, out_features, in_features, ldw};
    const Matrix y{Y, tokens, out_features, ldy}, z{Z, tokens, out_features, ldz}, r{residual, tokens, out_features, ldr};
    const Matrix b{bias, 1, out_features, out_features};
    int rc;
    if ((rc = check_bf16(x)) != MOSAIC_OK || (rc = check_bf16(w)) != MOSAIC_OK || (rc = check_bf16(y)) != MOSAIC_OK) return rc;
    if (Z != nullptr && (rc = check_bf16(z)) != MOSAIC_OK) return rc;
    if (residual != nullptr && (rc = check_bf16(r)) != MOSAIC_OK) return rc;
    if (bias != nullptr && (rc = check_bf16(b)) != MOSAIC_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(status_dev) & 3u) != 0) return MOSAIC_ERR_MISALIGNED;
    // the residual may be the output itself (added in place), with the same leading dimension
    if (overlap(y, x) || overlap(y, w) || overlap(y, b) || overlap(y, z) || overlap(z, x) || overlap(z, w) || overlap(z, b) || overlap(z, r))
        return MOSAIC_ERR_ALIASING;
    if (overlap(y, r) && !(residual == Y && ldr == ldy)) return MOSAIC_ERR_ALIASING;
    if ((rc = check_workspace(ws, ws_bytes, mosaic_linear_workspace_bytes(X, ldx, W, ldw, tokens, out_features, in_features))) != MOSAIC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (status_dev != nullptr) MOSAIC_CUDA_TRY(cudaMemsetAsync(status_dev, 0, sizeof(int), st));
    if (tokens == 0) return MOSAIC_OK;
    MmArgs a = {};
    a.n_i = out_features; a.n_j = tokens; a.n_c = in_features;
    a.out = static_cast<uint16_t*>(Y); a.ld_out = ldy;
    a.bias = static_cast<const uint16_t*>(bias);
    a.resid = static_cast<const uint16_t*>(residual); a.ld_resid = ldr;
    a.z = static_cast<uint16_t*>(Z); a.ld_z = ldz;
    a.act = act; a.status = status_dev;
    if (tokens <= (x.tma_ok() && w.tma_ok() ? kFewVector : kFewTokens)) return launch_few<false>(x, w, a, st);
    char* scratch = static_cast<char*>(ws);
    if ((rc = readable(x, &scratch, st)) != MOSAIC_OK || (rc = readable(w, &scratch, st)) != MOSAIC_OK) return rc;
    return run_mm<false, false>(w, x, a, st);
}

extern "C" size_t mosaic_linear_backward_workspace_bytes(const void* dY, int64_t lddy, const void* X, int64_t ldx, const void* W, int64_t ldw,
                                                         int64_t tokens, int64_t out_features, int64_t in_features, int act, int want_dx,
                                                         int want_dw, int want_dbias) {
    if (!extents_ok(tokens, out_features, in_features)) return 0;
    return backward_workspace({dY, tokens, out_features, lddy}, {X, tokens, in_features, ldx}, {W, out_features, in_features, ldw}, act, want_dx != 0,
                              want_dw != 0, want_dbias != 0);
}

extern "C" int mosaic_linear_backward(const void* dY, int64_t lddy, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* Z, int64_t ldz,
                                      int64_t tokens, int64_t out_features, int64_t in_features, int dtype, int act, void* dX, int64_t lddx, void* dW,
                                      int64_t lddw, void* dbias, int* status_dev, void* ws, size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (!extents_ok(tokens, out_features, in_features) || !act_ok(act)) return MOSAIC_ERR_INVALID_ARG;
    Matrix dy{dY, tokens, out_features, lddy}, x{X, tokens, in_features, ldx}, w{W, out_features, in_features, ldw};
    const Matrix z{Z, tokens, out_features, ldz}, dx{dX, tokens, in_features, lddx}, dw{dW, out_features, in_features, lddw}, db{dbias, 1, out_features, out_features};
    int rc;
    if ((rc = check_bf16(dy)) != MOSAIC_OK) return rc;
    if (dW != nullptr && ((rc = check_bf16(x)) != MOSAIC_OK || (rc = check_bf16(dw)) != MOSAIC_OK)) return rc;
    if (dX != nullptr && ((rc = check_bf16(w)) != MOSAIC_OK || (rc = check_bf16(dx)) != MOSAIC_OK)) return rc;
    if (act != MOSAIC_ACT_NONE && (rc = check_bf16(z)) != MOSAIC_OK) return rc;
    if (dbias != nullptr && (rc = check_bf16(db)) != MOSAIC_OK) return rc;
    if ((reinterpret_cast<uintptr_t>(status_dev) & 3u) != 0) return MOSAIC_ERR_MISALIGNED;
    {   // outputs overlap neither inputs nor one another
        const Matrix in[4] = {dy, dW != nullptr ? x : Matrix{}, dX != nullptr ? w : Matrix{}, act != MOSAIC_ACT_NONE ? z : Matrix{}};
        const Matrix out[3] = {dx, dw, db};
        for (int o = 0; o < 3; ++o) {
            for (int i = 0; i < 4; ++i)
                if (overlap(out[o], in[i])) return MOSAIC_ERR_ALIASING;
            for (int i = o + 1; i < 3; ++i)
                if (overlap(out[o], out[i])) return MOSAIC_ERR_ALIASING;
        }
    }
    if ((rc = check_workspace(ws, ws_bytes, backward_workspace(dy, x, w, act, dX != nullptr, dW != nullptr, dbias != nullptr))) != MOSAIC_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (status_dev != nullptr) MOSAIC_CUDA_TRY(cudaMemsetAsync(status_dev, 0, sizeof(int), st));
    char* scratch = static_cast<char*>(ws);
    float* partial = nullptr;
    if (dbias != nullptr) {
        partial = reinterpret_cast<float*>(scratch);
        scratch += align_up((size_t)bands_of(tokens) * (size_t)out_features * 4u, 256);
    }
    const bool products = dX != nullptr || dW != nullptr;
    const bool copy = products && tokens > 0 && (act != MOSAIC_ACT_NONE || !dy.tma_ok());
    if (copy || dbias != nullptr) {
        if ((rc = run_slope(dy, act != MOSAIC_ACT_NONE ? Z : nullptr, ldz, act, copy ? scratch : nullptr, dy.padded_ld(), partial, dbias, st)) != MOSAIC_OK) return rc;
        if (copy) {
            dy.p = scratch;
            dy.ld = dy.padded_ld();
            scratch += dy.padded_bytes();
        }
    }
    if (tokens == 0) {   // an empty sum
        if (dW != nullptr) MOSAIC_CUDA_TRY(cudaMemset2DAsync(dW, (size_t)lddw * 2u, 0, (size_t)in_features * 2u, (size_t)out_features, st));
        return MOSAIC_OK;
    }
    if (dX != nullptr) {
        if ((rc = readable(w, &scratch, st)) != MOSAIC_OK) return rc;
        MmArgs a = {};
        a.n_i = in_features; a.n_j = tokens; a.n_c = out_features;
        a.out = static_cast<uint16_t*>(dX); a.ld_out = lddx; a.status = status_dev;
        if ((rc = run_mm<true, false>(w, dy, a, st)) != MOSAIC_OK) return rc;
    }
    if (dW != nullptr) {
        if ((rc = readable(x, &scratch, st)) != MOSAIC_OK) return rc;
        MmArgs a = {};
        a.n_i = in_features; a.n_j = out_features; a.n_c = tokens;
        a.out = static_cast<uint16_t*>(dW); a.ld_out = lddw; a.status = status_dev;
        if ((rc = run_mm<true, true>(x, dy, a, st)) != MOSAIC_OK) return rc;
    }
    return MOSAIC_OK;
}
