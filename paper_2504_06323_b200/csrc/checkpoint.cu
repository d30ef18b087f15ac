// mosaic_checkpoint_store / mosaic_checkpoint_load: activations in 8 bits between the forward and the backward pass.
#include "checkpoint.cuh"

namespace mosaic {
namespace {

// A warp takes 256 columns, a lane eight of them (two lanes a group), kSavedRows rows in flight.  A pass reads two bytes an
// element and writes 1 1/16, or the other way round.  Bound by memory with issue close behind (85 % storing, 69 % loading):
// 4096 x 13824 stored and loaded in a row 61 to 64 us, 5.4 to 5.6 TB/s, of which 53 are the bytes at the measured peak.
constexpr int kSavedWarps = 8, kSavedRows = 4;

template <bool VEC>
__global__ void __launch_bounds__(32 * kSavedWarps) store_kernel(const uint16_t* X, int64_t ldx, int64_t rows, int64_t cols, const __grid_constant__ Saved out,
                                                                 unsigned chunks) {
    __shared__ uint4 turns[VEC ? 1 : kSavedWarps][kTurn];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* turn = turns[VEC ? 0 : warp];
    const int64_t c0 = ((int64_t)(blockIdx.x % chunks) * kSavedWarps + warp) * kWarpCols, c = c0 + lane * kLaneCols;
    const int64_t r0 = (int64_t)(blockIdx.x / chunks) * kSavedRows;
    if (c0 >= cols) return;
    await_previous_kernel();
    uint32_t w[kSavedRows][4];
#pragma unroll
    for (int r = 0; r < kSavedRows; ++r) {
        const int64_t row = r0 + r < rows ? r0 + r : rows - 1;
        lane_load8<VEC>(X + row * ldx, c0, cols, turn, w[r]);
    }
#pragma unroll
    for (int r = 0; r < kSavedRows; ++r) {
        uint32_t largest = largest8(w[r]);
        const bool finite = largest < kNotFinite;
        if (!finite) largest = largest_finite8(w[r]);
        largest = max(largest, __shfl_xor_sync(0xFFFFFFFFu, largest, 1));
        if (r0 + r >= rows || c >= (cols + kSavedGroup - 1) / kSavedGroup * kSavedGroup) continue;
        const uint32_t E = saved_exponent(largest);
        *reinterpret_cast<uint2*>(out.codes + (r0 + r) * out.ldc + c) = saved_codes8(w[r], E, finite);
        if ((lane & 1) == 0) out.exponents[(r0 + r) * out.lde + c / kSavedGroup] = (uint8_t)E;
    }
}

template <bool VEC>
__global__ void __launch_bounds__(32 * kSavedWarps) load_kernel(const __grid_constant__ Saved in, int64_t rows, int64_t cols, uint16_t* X, int64_t ldx,
                                                                unsigned chunks) {
    __shared__ uint4 turns[VEC ? 1 : kSavedWarps][kTurn];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint4* turn = turns[VEC ? 0 : warp];
    const int64_t c0 = ((int64_t)(blockIdx.x % chunks) * kSavedWarps + warp) * kWarpCols, c = c0 + lane * kLaneCols;
    const int64_t r0 = (int64_t)(blockIdx.x / chunks) * kSavedRows;
    if (c0 >= cols) return;
    await_previous_kernel();
    uint2 q[kSavedRows];
    uint32_t E[kSavedRows];
#pragma unroll
    for (int r = 0; r < kSavedRows; ++r) {
        const int64_t row = r0 + r < rows ? r0 + r : rows - 1;
        q[r] = make_uint2(0u, 0u);
        E[r] = 0;
        if (c < cols) {
            q[r] = *reinterpret_cast<const uint2*>(in.codes + row * in.ldc + c);
            E[r] = in.exponents[row * in.lde + c / kSavedGroup];
        }
    }
#pragma unroll
    for (int r = 0; r < kSavedRows; ++r) {
        if (r0 + r >= rows) break;
        float v[8];
        saved_values8(q[r], E[r], v);
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = pack_exact(v[2 * e], v[2 * e + 1]);
        lane_store8<VEC>(X + (r0 + r) * ldx, c0, cols, turn, w);
    }
}

bool on_vectors(const void* p, int64_t ld, int64_t rows) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld % 8 == 0); }

// A CTA for kSavedRows rows of `chunks` parts each; their number fits a grid for any matrix that fits a memory.
struct RowLaunch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    unsigned chunks;
    RowLaunch(int64_t rows, int64_t cols, cudaStream_t st) {
        const int64_t wide = kSavedWarps * kWarpCols;
        attr = early_start();
        chunks = (unsigned)((cols + wide - 1) / wide);
        cfg.gridDim = dim3((unsigned)(chunks * ((rows + kSavedRows - 1) / kSavedRows)));
        cfg.blockDim = dim3(32 * kSavedWarps);
        cfg.stream = st;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
    }
};

constexpr int64_t kMostSide = 0x7FFFFFFF - 1024, kMostCells = (int64_t)1 << 41;

int check_pass(const void* X, int64_t rows, int64_t cols, int64_t ldx, int dtype, const mosaic_checkpoint* c) {
    if (dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (rows < 0 || cols <= 0 || rows > kMostSide || cols > kMostSide || ldx < cols || rows * (cols + 2048) > kMostCells) return MOSAIC_ERR_INVALID_ARG;
    if (c == nullptr || (rows > 0 && X == nullptr)) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(X) & 1u) != 0) return MOSAIC_ERR_MISALIGNED;
    int rc = check_saved(c, rows, cols);
    if (rc != MOSAIC_OK) return rc;
    if (rows > 0) {
        const Saved s = as_saved(c);
        const size_t x = ((size_t)(rows - 1) * (size_t)ldx + (size_t)cols) * 2u;
        if (spans_meet(X, x, s.codes, saved_code_bytes(s, rows, cols)) || spans_meet(X, x, s.exponents, saved_exponent_bytes(s, rows, cols)) ||
            spans_meet(s.codes, saved_code_bytes(s, rows, cols), s.exponents, saved_exponent_bytes(s, rows, cols)))
            return MOSAIC_ERR_ALIASING;
    }
    return MOSAIC_OK;
}

}  // namespace

int check_saved(const mosaic_checkpoint* c, int64_t rows, int64_t cols) {
    if (c->ldc < saved_groups(cols) * kSavedGroup || c->lde < saved_groups(cols)) return MOSAIC_ERR_INVALID_ARG;
    if (rows > 0 && (c->codes == nullptr || c->exponents == nullptr)) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(c->codes) & 15u) != 0 || c->ldc % kSavedGroup != 0) return MOSAIC_ERR_MISALIGNED;
    return MOSAIC_OK;
}

int store_saved(const void* X, int64_t ldx, int64_t rows, int64_t cols, const Saved& out, cudaStream_t st) {
    if (rows == 0) return MOSAIC_OK;
    RowLaunch l(rows, cols, st);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, on_vectors(X, ldx, rows) ? store_kernel<true> : store_kernel<false>, static_cast<const uint16_t*>(X), ldx, rows,
                                       cols, out, l.chunks));
    return MOSAIC_OK;
}

int load_saved(const Saved& in, int64_t rows, int64_t cols, void* X, int64_t ldx, cudaStream_t st) {
    if (rows == 0) return MOSAIC_OK;
    RowLaunch l(rows, cols, st);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, on_vectors(X, ldx, rows) ? load_kernel<true> : load_kernel<false>, in, rows, cols, static_cast<uint16_t*>(X), ldx,
                                       l.chunks));
    return MOSAIC_OK;
}

}  // namespace mosaic

using namespace mosaic;

extern "C" int mosaic_checkpoint_store(const void* X, int64_t rows, int64_t cols, int64_t ldx, int dtype, const mosaic_checkpoint* out, void* stream) {
    const int rc = check_pass(X, rows, cols, ldx, dtype, out);
    return rc != MOSAIC_OK ? rc : store_saved(X, ldx, rows, cols, as_saved(out), static_cast<cudaStream_t>(stream));
}

extern "C" int mosaic_checkpoint_load(const mosaic_checkpoint* in, int64_t rows, int64_t cols, void* X, int64_t ldx, int dtype, void* stream) {
    const int rc = check_pass(X, rows, cols, ldx, dtype, in);
    return rc != MOSAIC_OK ? rc : load_saved(as_saved(in), rows, cols, X, ldx, static_cast<cudaStream_t>(stream));
}
