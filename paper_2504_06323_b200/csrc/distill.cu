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

struct DistillArgs {   // (rows and leading dimensions in elements)
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
    double inv_t;
    float t, c;       // T, log2(e) / T
    int slots;        // of the table of kept places: a power of two, at least 2 * top
    float* loss;
    float* lse;
};

constexpr int kWantLoss = 1, kWantGrad = 2;

// A kept logit's probability under the teacher's own log-sum-exp.
__device__ __forceinline__ float teacher_p(float t, float t_lse, double inv_t) { return expf((float)((double)t * inv_t - (double)t_lse)); }

// One row by a cluster of CTAs.  MODE: what is wanted; with kWantGrad alone the saved log-sum-exp is an input.
// Every thread takes its share of the kept entries (loads in flight beside the row's), so that the row's and the
// teacher's statistics meet in one barrier.
template <int DT, int MODE>
__global__ void __launch_bounds__(kRowThreads, kRowCtasPerSm) distill_kernel(const __grid_constant__ DistillArgs a) {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    __shared__ SoftStat warp_stat[kRowWarps];
    __shared__ SoftStat cta_stat[kMaxCluster];   // written by the CTAs of the cluster
    __shared__ SoftStat kept_stat[kRowWarps];    // renormalised: softmax statistics of the kept entries; else the sum of their p in .s
    __shared__ double warp_loss[kRowWarps];
    __shared__ int doubled;                      // some vocabulary entry is kept twice
    extern __shared__ unsigned char dyn[];
    int32_t* k_idx = reinterpret_cast<int32_t*>(dyn);             // [top] -1: absent
    float* k_t = reinterpret_cast<float*>(k_idx + a.top);         // [top] the teacher's logit, later its probability
    float* k_x = k_t + a.top;                                     // [top] the student's logit there
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
    const bool given = a.t_lse != nullptr;
    const int lone = part.single();

    uint4 raw[kRowVecs];
    if (reads) part.load_pass(part.v_lo, raw);
    const float lone_x = reads && lone >= 0 ? part.at(lone) : -INFINITY;
    cg::cluster_group::arrival_token started = cluster.barrier_arrive();   // waited for before the first write to another CTA

    // ---- the kept entries, while the row is on its way
    const float t_lse = given ? a.t_lse[r] : 0.0f;
    {
        const float* tv = a.t_values + r * a.top;
        const int32_t* ti = a.t_indices + r * a.top;
        SoftStat kst = {-INFINITY, 0.0f};
        for (int i = threadIdx.x; i < a.top; i += kRowThreads) {
            const int32_t j = ti[i];
            const bool there = j >= 0 && j < vocab;
            const float t = there ? tv[i] : -INFINITY;
            k_idx[i] = there ? j : -1;
            // gathered before any gradient is written (dS may be S); without the loss only the own part's are used
            k_x[i] = there && reads && ((MODE & kWantLoss) || part.owns(j)) ? part.at(j) : 0.0f;
            k_t[i] = t;
            if (given) kst.s = __fadd_rn(kst.s, teacher_p(t, t_lse, a.inv_t));
            else kst = soft_merge(kst, soft_one(t, a.c), a.c);
        }
        if (given) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) kst.s = __fadd_rn(kst.s, __shfl_xor_sync(0xFFFFFFFFu, kst.s, o));
        } else {
            kst = soft_warp(kst, a.c);
        }
        if (lane == 0) kept_stat[warp] = kst;
        if (MODE & kWantGrad) {
            if (threadIdx.x == 0) doubled = 0;
            for (int i = threadIdx.x; i < a.slots; i += kRowThreads) table[i] = 0xFFFFFFFFu;
        }
    }

    // ---- softmax statistics of the row
    SoftStat st = {-INFINITY, 0.0f};
    if (MODE & kWantLoss) {
        st = soft_warp(soft_part<DT>(part, raw, lone_x, a.c), a.c);
        if (lane == 0) warp_stat[warp] = st;
    }
    cluster.barrier_wait(std::move(started));
    __syncthreads();
    SoftStat kst = {0.0f, 0.0f};
    float mass;   // P
    if (given) {
        mass = lane < kRowWarps ? kept_stat[lane].s : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mass = __fadd_rn(mass, __shfl_xor_sync(0xFFFFFFFFu, mass, o));
    } else {
        kst = soft_all(kept_stat, kRowWarps, a.c);
        mass = kst.s == 0.0f ? 0.0f : __fdiv_rn(kst.s, kst.s);   // 1; NaN stays NaN
    }
    if (MODE & kWantLoss) {
        st = soft_all(warp_stat, kRowWarps, a.c);
        if (n_ctas > 1) {
            if (threadIdx.x < n_ctas) *cluster.map_shared_rank(&cta_stat[rank], threadIdx.x) = st;
            cluster.sync();   // also: every CTA has gathered its kept entries' logits
            st = soft_all(cta_stat, n_ctas, a.c);
        }
    }

    // ---- the kept entries' probabilities, and the loss in fp64: differences of logarithms that nearly cancel
    const float kept_inv = __frcp_rn(kst.s), kept_ref = soft_ref(kst.m);
    double sum = 0.0;
    if ((int)threadIdx.x < a.top) {
        double lse = 0.0, norm = 0.0;
        if ((MODE & kWantLoss) && rank == 0) {
            lse = soft_lse(st, a.inv_t);
            norm = given ? (double)t_lse : soft_lse(kst, a.inv_t);
            if (threadIdx.x == 0 && a.lse != nullptr) a.lse[r] = (float)lse;
        }
        for (int i = threadIdx.x; i < a.top; i += kRowThreads) {
            const float t = k_t[i];
            float p = given ? teacher_p(t, t_lse, a.inv_t) : __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(t, kept_ref), a.c)), kept_inv);
            if (t == -INFINITY) p = 0.0f;
            k_t[i] = p;
            if ((MODE & kWantLoss) && rank == 0 && p != 0.0f)
                sum += (double)p * (((double)t * a.inv_t - norm) - ((double)k_x[i] * a.inv_t - lse));
        }
    }
    if ((MODE & kWantLoss) && rank == 0) {
        if (warp * 32 < a.top) sum = warp_sum(sum);
        if (lane == 0) warp_loss[warp] = sum;
    }
    const bool zero = weight == 0.0f || mass == 0.0f;

    if (MODE & kWantGrad) {
        const float coef = __fmul_rn(__fmul_rn(__fmul_rn(a.grad_rows != nullptr ? a.grad_rows[r] : 1.0f, a.grad_scale), weight), a.t);
        // P q_j coef = 2^((x_j - ref) c) * dense;  from a saved log-sum-exp L: 2^((x_j / T - L) log2 e) * dense
        const float ref = soft_ref(st.m), inv_t = (float)a.inv_t;
        const float minus_lse = (MODE & kWantLoss) || zero ? 0.0f : -a.lse[r];
        const float dense = (MODE & kWantLoss) ? __fmul_rn(__fmul_rn(coef, mass), __frcp_rn(st.s)) : __fmul_rn(coef, mass);
        auto dense_of = [&](float x) -> float {
            if (MODE & kWantLoss) return __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(x, ref), a.c)), dense);
            return __fmul_rn(exp2_fast(__fmul_rn(__fmaf_rn(x, inv_t, minus_lse), 1.4426950408889634f)), dense);
        };
        Elem* out = reinterpret_cast<Elem*>(a.dS) + r * a.ldd;
        const bool aligned = (reinterpret_cast<uintptr_t>(out + part.head) & 15u) == 0;
        if (lone >= 0) out[lone] = RV::narrow(zero ? 0.0f : dense_of(lone_x));
        for (int b = part.v_lo; b < part.v_hi; b += kRowThreads * kRowVecs) {
            if (!held && !zero) part.load_pass(b, raw);
            keep_packed(raw);
#pragma unroll
            for (int i = 0; i < kRowVecs; ++i) {
                const int v = b + (int)threadIdx.x + i * kRowThreads;
                if (v < part.v_hi) {
                    float f[RV::kElems];
#pragma unroll
                    for (int e = 0; e < RV::kElems; ++e) f[e] = zero ? 0.0f : dense_of(RV::get(raw[i], e));
                    Elem* o = out + part.first(v);
                    if (aligned) {
                        st_stream16(o, RV::pack(f));
                    } else {
#pragma unroll
                        for (int e = 0; e < RV::kElems; ++e) o[e] = RV::narrow(f[e]);
                    }
                }
            }
        }
        if (!zero) {
            for (int i = threadIdx.x; i < a.top; i += kRowThreads) {
                const int32_t j = k_idx[i];
                if (j >= 0) {   // open addressing; a second entry for the same place is noted
                    uint32_t h = ((uint32_t)j * 2654435761u) & (uint32_t)(a.slots - 1);
                    for (;;) {
                        const uint32_t old = atomicCAS(&table[h], 0xFFFFFFFFu, (uint32_t)j);
                        if (old == 0xFFFFFFFFu) break;
                        if (old == (uint32_t)j) {
                            doubled = 1;
                            break;
                        }
                        h = (h + 1u) & (uint32_t)(a.slots - 1);
                    }
                }
            }
        }
        __syncthreads();   // the dense values of this CTA's part are written, the table and the losses are complete
        // the kept entries' places: their whole value, from the gathered logit
        if (!zero) {
            for (int i = threadIdx.x; i < a.top; i += kRowThreads) {
                const int32_t j = k_idx[i];
                if (j < 0 || !part.owns(j)) continue;
                float p = k_t[i];
                if (doubled) {   // every copy of the entry writes the same sum
                    p = 0.0f;
                    for (int o = 0; o < a.top; ++o)
                        if (k_idx[o] == j) p = __fadd_rn(p, k_t[o]);
                }
                out[j] = RV::narrow(__fsub_rn(dense_of(k_x[i]), __fmul_rn(coef, p)));
            }
        }
    } else {
        __syncthreads();
    }
    if ((MODE & kWantLoss) && rank == 0 && threadIdx.x == 0) {
        double total = 0.0;
        for (int w = 0; w < kRowWarps; ++w) total += warp_loss[w];
        a.loss[r] = zero ? 0.0f : (float)((double)weight * (double)a.t * (double)a.t * total);
    }
}

template <int DT, int MODE> int launch_distill(const DistillArgs& a, cudaStream_t st) {
    const int c = row_cluster(a.rows, row_vectors(a.vocab, DT));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    cfg.blockDim = dim3(kRowThreads);
    cfg.dynamicSmemBytes = (size_t)a.top * 12u + (size_t)a.slots * 4u;   // at most 20 KB
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
    a.t = temperature;
    a.slots = 64;
    while (a.slots < 2 * a.top) a.slots *= 2;
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
