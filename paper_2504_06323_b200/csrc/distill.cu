// mosaic_distill_loss / _grad / _loss_grad: how far a student's distribution is from the kept top logits
// of its teacher, per row, and the gradient with respect to the student's logits.
//
// With x = S / T, q = softmax(x) over the whole vocabulary and p_i the teacher's probabilities of the
// kept entries (P their sum),
//     loss  = w T^2 sum_i p_i (log p_i - log q_{idx_i}),          log q_j = x_j - lse
//     dS_j  = g w T (P q_j - sum_{i: idx_i = j} p_i).
// One pass over the row for the running maximum and sum of the softmax, one for the gradient; the kept
// entries (tens to hundreds) are a gather and a correction.  Bound by memory: the row is read once into
// registers (rows.cuh) and the gradient written once.
#include <math.h>

#include "rows.cuh"

namespace cg = cooperative_groups;

namespace mosaic {
namespace {

struct DistillArgs {
    const void* S;
    void* dS;
    int64_t rows, vocab, lds, ldd;
    const float* t_values;
    const int32_t* t_indices;
    int top;
    const float* t_lse;
    const float* row_weight;
    const float* grad_rows;
    float grad_scale;
    double inv_t, t;
    float c;          // log2(e) / T
    float* loss;
    float* lse;
};

constexpr int kWantLoss = 1, kWantGrad = 2;

__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmax(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

// One row by a cluster of CTAs.  MODE: what is wanted; with kWantGrad alone the saved log-sum-exp is an input.
template <int DT, int MODE>
__global__ void __launch_bounds__(kRowThreads, 2) distill_kernel(const __grid_constant__ DistillArgs a) {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    __shared__ SoftStat warp_stat[kRowWarps];
    __shared__ SoftStat cta_stat[kMaxCluster];   // written by the CTAs of the cluster
    __shared__ float mass_s;                     // P
    __shared__ int doubled;                      // some vocabulary entry is kept twice
    extern __shared__ unsigned char dyn[];
    int32_t* k_idx = reinterpret_cast<int32_t*>(dyn);          // [top] -1: absent
    float* k_p = reinterpret_cast<float*>(k_idx + a.top);      // [top]
    float* k_x = k_p + a.top;                                  // [top] the student's logit there
    uint32_t* table = reinterpret_cast<uint32_t*>(k_x + a.top);   // [slots] entries seen, to find doubled ones

    cg::cluster_group cluster = cg::this_cluster();
    const int n_ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x / n_ctas;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int vocab = (int)a.vocab;
    const RowPart<DT> part(a.S, r, a.lds, vocab, rank, n_ctas);
    const bool held = part.v_hi - part.v_lo <= kRowThreads * kRowVecs;   // the CTA's part stays in registers between the passes
    const float weight = a.row_weight != nullptr ? a.row_weight[r] : 1.0f;
    const bool reads = (MODE & kWantLoss) != 0 || weight != 0.0f;   // a dropped row's gradient is zero whatever it holds
    int slots = 64;
    while (slots < 2 * a.top) slots *= 2;

    uint4 raw[kRowVecs];
    if (reads) part.load_pass(part.v_lo, raw);

    cg::cluster_group::arrival_token started = cluster.barrier_arrive();   // waited for before the first write to another CTA

    // ---- the kept entries: one warp, while the row is on its way
    if (threadIdx.x == 32) doubled = 0;
    if (MODE & kWantGrad)
        for (int i = threadIdx.x; i < slots; i += kRowThreads) table[i] = 0xFFFFFFFFu;
    const float* tv = a.t_values + r * a.top;
    double norm = 0.0;   // warp 0: log of what the kept entries' exponentials are divided by
    if (warp == 0) {
        const int32_t* ti = a.t_indices + r * a.top;
        double top_u = -INFINITY;
        for (int i = lane; i < a.top; i += 32) {
            const int32_t j = ti[i];
            const bool there = j >= 0 && j < vocab;
            k_idx[i] = there ? j : -1;
            // gathered before any gradient is written (dS may be S); without the loss only the own part's are used
            k_x[i] = there && reads && ((MODE & kWantLoss) || part.owns(j)) ? part.at(j) : 0.0f;
            if (there) top_u = fmax(top_u, (double)tv[i] * a.inv_t);
        }
        if (a.t_lse != nullptr) {
            norm = (double)a.t_lse[r];
        } else {
            top_u = warp_max(top_u);
            if (!(fabs(top_u) <= 1.7e308)) top_u = 0.0;   // no finite entry
            double s = 0.0;
            for (int i = lane; i < a.top; i += 32)
                if (k_idx[i] >= 0) s += exp((double)tv[i] * a.inv_t - top_u);
            norm = top_u + log(warp_sum(s));
        }
        double mass = 0.0;
        for (int i = lane; i < a.top; i += 32) {
            double p = 0.0;
            const double u = (double)tv[i] * a.inv_t;
            if (k_idx[i] >= 0 && u != -INFINITY) p = exp(u - norm);
            k_p[i] = (float)p;
            mass += p;
        }
        mass = warp_sum(mass);
        if (lane == 0) mass_s = (float)mass;
    }

    // ---- softmax statistics of the row
    SoftStat st = {-INFINITY, 0.0f};
    if (MODE & kWantLoss) {
        soft_pass<DT>(raw, a.c, st);
        for (int b = part.v_lo + kRowThreads * kRowVecs; b < part.v_hi; b += kRowThreads * kRowVecs) {
            part.load_pass(b, raw);
            soft_pass<DT>(raw, a.c, st);
        }
        st = soft_warp(st, a.c);
        if (lane == 0) warp_stat[warp] = st;
    }
    cluster.barrier_wait(std::move(started));
    __syncthreads();
    if (MODE & kWantLoss) {
        st = soft_all(warp_stat, kRowWarps, a.c);
        if (n_ctas > 1) {
            if (threadIdx.x < n_ctas) *cluster.map_shared_rank(&cta_stat[rank], threadIdx.x) = st;
            cluster.sync();   // also: every CTA has gathered its kept entries' logits
            st = soft_all(cta_stat, n_ctas, a.c);
        }
        if (rank == 0 && warp == 0) {
            const double lse = soft_lse(st, a.inv_t);
            double sum = 0.0;
            for (int i = lane; i < a.top; i += 32) {
                const double p = (double)k_p[i];
                if (p != 0.0) sum += p * (((double)tv[i] * a.inv_t - norm) - ((double)k_x[i] * a.inv_t - lse));
            }
            sum = warp_sum(sum);
            if (lane == 0) {
                a.loss[r] = weight != 0.0f ? (float)((double)weight * a.t * a.t * sum) : 0.0f;
                if (a.lse != nullptr) a.lse[r] = (float)lse;
            }
        }
    }
    if (!(MODE & kWantGrad)) return;

    // ---- gradient
    const float mass = mass_s;
    const bool zero = weight == 0.0f || mass == 0.0f;
    const float coef = (float)((a.grad_rows != nullptr ? (double)a.grad_rows[r] : 1.0) * (double)a.grad_scale * (double)weight * a.t);
    // q_j = 2^((x_j - ref) c) * scale;  from a saved log-sum-exp L: ref = L T and scale = 1
    float ref, scale;
    if (MODE & kWantLoss) {
        ref = soft_ref(st.m);
        scale = (float)(1.0 / (double)st.s);
    } else {
        ref = 0.0f;
        scale = 1.0f;
    }
    const float inv_t = (float)a.inv_t;
    const float minus_lse = (MODE & kWantLoss) || zero ? 0.0f : -a.lse[r];
    const float dense = __fmul_rn(__fmul_rn(coef, mass), scale);
    auto q_of = [&](float x) -> float {   // without `scale`
        if (MODE & kWantLoss) return exp2_fast(__fmul_rn(__fsub_rn(x, ref), a.c));
        return exp2_fast(__fmul_rn(__fmaf_rn(x, inv_t, minus_lse), 1.4426950408889634f));
    };
    Elem* out = reinterpret_cast<Elem*>(a.dS) + r * a.ldd;
    const bool aligned = (((reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(part.row)) & 15u) == 0);
    for (int b = part.v_lo; b < part.v_hi; b += kRowThreads * kRowVecs) {
        if (!held && !zero) part.load_pass(b, raw);
        keep_packed(raw);
#pragma unroll
        for (int i = 0; i < kRowVecs; ++i) {
            const int v = b + (int)threadIdx.x + i * kRowThreads;
            if (v < part.v_hi) {
                float f[RV::kElems];
#pragma unroll
                for (int e = 0; e < RV::kElems; ++e) f[e] = zero ? 0.0f : __fmul_rn(q_of(RV::get(raw[i], e)), dense);
                const int j = part.first(v);
                if (aligned && part.whole(v)) {
                    st_stream16(out + j, RV::pack(f));
                } else {
#pragma unroll
                    for (int e = 0; e < RV::kElems; ++e)
                        if (j + e >= 0 && j + e < vocab) out[j + e] = RV::narrow(f[e]);
                }
            }
        }
    }
    if (zero) return;

    // ---- the kept entries' correction: their whole value, from the gathered logit
    for (int i = threadIdx.x; i < a.top; i += kRowThreads) {
        const int32_t j = k_idx[i];
        if (j >= 0) {   // open addressing; a second entry for the same place is noted
            uint32_t h = ((uint32_t)j * 2654435761u) & (uint32_t)(slots - 1);
            for (;;) {
                const uint32_t old = atomicCAS(&table[h], 0xFFFFFFFFu, (uint32_t)j);
                if (old == 0xFFFFFFFFu) break;
                if (old == (uint32_t)j) {
                    doubled = 1;
                    break;
                }
                h = (h + 1u) & (uint32_t)(slots - 1);
            }
        }
    }
    __syncthreads();   // the dense values of this CTA's part are written, the table is complete
    for (int i = threadIdx.x; i < a.top; i += kRowThreads) {
        const int32_t j = k_idx[i];
        if (j < 0 || !part.owns(j)) continue;
        float p = k_p[i];
        if (doubled) {   // every copy of the entry writes the same sum
            p = 0.0f;
            for (int o = 0; o < a.top; ++o)
                if (k_idx[o] == j) p = __fadd_rn(p, k_p[o]);
        }
        out[j] = RV::narrow(__fsub_rn(__fmul_rn(q_of(k_x[i]), dense), __fmul_rn(coef, p)));
    }
}

template <int DT, int MODE> int launch_distill(const DistillArgs& a, cudaStream_t st) {
    const int c = row_cluster(a.rows, row_vectors(a.vocab, DT));
    int slots = 64;
    while (slots < 2 * a.top) slots *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    cfg.blockDim = dim3(kRowThreads);
    cfg.dynamicSmemBytes = (size_t)a.top * 12u + (size_t)slots * 4u;   // at most 20 KB
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, distill_kernel<DT, MODE>, a));
    return MOSAIC_OK;
}

bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
    return x != nullptr && y != nullptr && an > 0 && bn > 0 && x < y + bn && y < x + an;
}
size_t span(int64_t rows, int64_t cols, int64_t ld, size_t elem) { return ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem; }

template <int MODE> int distill(DistillArgs a, int64_t top, float temperature, int dtype, void* stream) {
    if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (a.rows < 0 || a.rows > 0x7FFFFFFF / kMaxCluster || a.vocab <= 0 || a.vocab > kMaxRow || a.lds < a.vocab || top < 1 || top > kMaxTop)
        return MOSAIC_ERR_INVALID_ARG;
    if ((MODE & kWantGrad) && a.ldd < a.vocab) return MOSAIC_ERR_INVALID_ARG;
    if (!(temperature >= 1.17549435e-38f) || !(temperature <= 3.402823466e38f)) return MOSAIC_ERR_INVALID_ARG;
    if (a.rows == 0) return MOSAIC_OK;
    if (a.S == nullptr || a.t_values == nullptr || a.t_indices == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((MODE & kWantLoss) && a.loss == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((MODE & kWantGrad) && (a.dS == nullptr || (!(MODE & kWantLoss) && a.lse == nullptr))) return MOSAIC_ERR_NULL_PTR;
    const size_t es = elem_size(dtype);
    const uintptr_t words = reinterpret_cast<uintptr_t>(a.t_values) | reinterpret_cast<uintptr_t>(a.t_indices) |
                            reinterpret_cast<uintptr_t>(a.t_lse) | reinterpret_cast<uintptr_t>(a.row_weight) |
                            reinterpret_cast<uintptr_t>(a.grad_rows) | reinterpret_cast<uintptr_t>(a.loss) | reinterpret_cast<uintptr_t>(a.lse);
    if ((words & 3u) != 0 || ((reinterpret_cast<uintptr_t>(a.S) | reinterpret_cast<uintptr_t>(a.dS)) & (es - 1u)) != 0) return MOSAIC_ERR_MISALIGNED;
    a.top = (int)top;
    const size_t n = (size_t)a.rows, s_bytes = span(a.rows, a.vocab, a.lds, es);
    // what is written, against everything that is read or written beside it
    const void* in[6] = {a.S, a.t_values, a.t_indices, a.t_lse, a.row_weight, a.grad_rows};
    const size_t in_n[6] = {s_bytes, n * (size_t)top * 4u, n * (size_t)top * 4u, n * 4u, n * 4u, n * 4u};
    const void* out[3] = {(MODE & kWantGrad) ? a.dS : nullptr, (MODE & kWantLoss) ? a.loss : nullptr, a.lse};
    const size_t out_n[3] = {(MODE & kWantGrad) ? span(a.rows, a.vocab, a.ldd, es) : 0u, n * 4u, n * 4u};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 6; ++i) {
            if (o == 0 && i == 0 && a.dS == a.S && a.ldd == a.lds) continue;   // in place
            if (o == 2 && !(MODE & kWantLoss)) continue;                       // lse is an input
            if (overlap(out[o], out_n[o], in[i], in_n[i])) return MOSAIC_ERR_ALIASING;
        }
        for (int i = o + 1; i < 3; ++i)
            if (overlap(out[o], out_n[o], out[i], out_n[i])) return MOSAIC_ERR_ALIASING;
    }
    a.t = (double)temperature;
    a.inv_t = 1.0 / (double)temperature;
    a.c = (float)(1.4426950408889634 / (double)temperature);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == MOSAIC_BF16 ? launch_distill<MOSAIC_BF16, MODE>(a, st) : launch_distill<MOSAIC_F32, MODE>(a, st);
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" int mosaic_distill_loss(const void* S, int64_t rows, int64_t vocab, int64_t lds, int dtype, const float* t_values,
                                   const int32_t* t_indices, int64_t top, const float* t_lse, const float* row_weight, float temperature,
                                   float* loss, float* lse, void* stream) {
    DistillArgs a = {};
    a.S = S; a.rows = rows; a.vocab = vocab; a.lds = lds;
    a.t_values = t_values; a.t_indices = t_indices; a.t_lse = t_lse; a.row_weight = row_weight;
    a.loss = loss; a.lse = lse;
    return distill<kWantLoss>(a, top, temperature, dtype, stream);
}

extern "C" int mosaic_distill_grad(const void* S, int64_t rows, int64_t vocab, int64_t lds, int dtype, const float* t_values,
                                   const int32_t* t_indices, int64_t top, const float* t_lse, const float* row_weight, float temperature,
                                   const float* lse, const float* grad_rows, float grad_scale, void* dS, int64_t ldd, void* stream) {
    DistillArgs a = {};
    a.S = S; a.rows = rows; a.vocab = vocab; a.lds = lds; a.dS = dS; a.ldd = ldd;
    a.t_values = t_values; a.t_indices = t_indices; a.t_lse = t_lse; a.row_weight = row_weight;
    a.lse = const_cast<float*>(lse); a.grad_rows = grad_rows; a.grad_scale = grad_scale;
    return distill<kWantGrad>(a, top, temperature, dtype, stream);
}

extern "C" int mosaic_distill_loss_grad(const void* S, int64_t rows, int64_t vocab, int64_t lds, int dtype, const float* t_values,
                                        const int32_t* t_indices, int64_t top, const float* t_lse, const float* row_weight, float temperature,
                                        float* loss, float* lse, const float* grad_rows, float grad_scale, void* dS, int64_t ldd, void* stream) {
    DistillArgs a = {};
    a.S = S; a.rows = rows; a.vocab = vocab; a.lds = lds; a.dS = dS; a.ldd = ldd;
    a.t_values = t_values; a.t_indices = t_indices; a.t_lse = t_lse; a.row_weight = row_weight;
    a.loss = loss; a.lse = lse; a.grad_rows = grad_rows; a.grad_scale = grad_scale;
    return distill<kWantLoss | kWantGrad>(a, top, temperature, dtype, stream);
}
