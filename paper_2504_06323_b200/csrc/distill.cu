// mosaic_distill_loss / _grad / _loss_grad: how far a student's distribution is from the kept top logits
// of its teacher, per row, and the gradient with respect to the student's logits.
//
// With x = S / T, q = softmax(x) over the whole vocabulary and p_i the teacher's probabilities of the
// kept entries (P their sum),
//     loss  = w T^2 sum_i p_i (log p_i - log q_{idx_i}),          log q_j = x_j - lse
//     dS_j  = g w T (P q_j - sum_{i: idx_i = j} p_i).
// One pass over the row for the running maximum and sum of the softmax, one for the gradient; the kept
// entries (tens to hundreds) are a gather and a correction.  Bound by memory: the row is read once (rows.cuh)
// and the gradient written once.
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
    int copy_vecs;    // vectors of the copy in shared memory (0: none)
    int ahead;        // rows between a row and the one it prefetches
    int slots;        // of the table of kept places: a power of two, at least 2 * top
    float* loss;
    float* lse;
};

constexpr int kWantLoss = 1, kWantGrad = 2;

// A kept logit's probability under the teacher's own log-sum-exp.
__device__ __forceinline__ float teacher_p(float t, float t_lse, double inv_t) { return expf((float)((double)t * inv_t - (double)t_lse)); }

// One kept entry in a thread's hands.
struct Kept {
    int j;       // its place, -1: absent
    float t;     // the teacher's logit
    float x;     // the student's logit there
};

// One row by a cluster of CTAs.  MODE: what is wanted; with kWantGrad alone the saved log-sum-exp is an input.
//   loss alone   one pass over the row for its softmax statistics
//   gradient     one pass that reads and writes
//   both         the first pass leaves the CTA's part of the row in shared memory, the second reads it there
// Every thread takes its share of the kept entries; their statistics meet the row's in one barrier.
template <int DT, int MODE>
__global__ void __launch_bounds__(kThreads, kRowCtas) distill_kernel(const __grid_constant__ DistillArgs a) {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    __shared__ SoftStat warp_stat[kWarps];
    __shared__ SoftStat cta_stat[kMaxCluster];   // written by the CTAs of the cluster
    __shared__ SoftStat kept_stat[kWarps];       // renormalised: softmax statistics of the kept entries; else the sum of their p in .s
    __shared__ double warp_loss[kWarps];
    __shared__ int doubled;                      // some vocabulary entry is kept twice
    extern __shared__ __align__(16) unsigned char dyn[];
    uint4* copy = reinterpret_cast<uint4*>(dyn);                                    // the CTA's part of the row (both wanted)
    Kept* kept = reinterpret_cast<Kept*>(dyn + (size_t)a.copy_vecs * 16u);          // [top]
    float* kept_prob = reinterpret_cast<float*>(kept + a.top);                      // [top] the teacher's probabilities (gradient)
    uint32_t* table = reinterpret_cast<uint32_t*>(kept_prob + a.top);               // [slots] places seen, to find doubled ones

    cg::cluster_group cluster = cg::this_cluster();
    const int n_ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x >> (__ffs(n_ctas) - 1);   // a power of two
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int vocab = (int)a.vocab;
    const RowPart<DT> part(a.S, r, a.lds, vocab, rank, n_ctas);
    const float weight = a.row_weight != nullptr ? a.row_weight[r] : 1.0f;
    const bool reads = (MODE & kWantLoss) != 0 || weight != 0.0f;   // a dropped row's gradient is zero whatever it holds
    const bool given = a.t_lse != nullptr;
    const float t_lse = given ? a.t_lse[r] : 0.0f;
    const bool held = (MODE & kWantGrad) && (MODE & kWantLoss) && part.v_hi - part.v_lo <= a.copy_vecs;
    const int lone = part.single();
    const float lone_x = reads && lone >= 0 ? part.at(lone) : -INFINITY;
    if (threadIdx.x == 0 && r + a.ahead < a.rows) part.prefetch((int64_t)a.ahead * a.lds);
    if (n_ctas > 1) cluster_arrive();   // waited for before the first write to another CTA

    // ---- the kept entries: places and teacher's logits (the first of a thread's stays in registers)
    const float* tv = a.t_values + r * a.top;
    const int32_t* ti = a.t_indices + r * a.top;
    SoftStat kst = {-INFINITY, 0.0f};
    auto fetch = [&](int i) -> Kept {
        Kept k = {ti[i], tv[i], 0.0f};
        if (k.j < 0 || k.j >= vocab) k = {-1, -INFINITY, 0.0f};
        return k;
    };
    auto count_in = [&](const Kept& k) {
        if (given) kst.s = __fadd_rn(kst.s, teacher_p(k.t, t_lse, a.inv_t));
        else kst = soft_merge(kst, soft_one(k.t, a.c), a.c);
    };
    // the student's logit, before any gradient is written (dS may be S); without the loss only the own part's is used
    auto gather = [&](Kept& k) {
        if (k.j >= 0 && reads && ((MODE & kWantLoss) || part.owns(k.j))) k.x = part.at(k.j);
    };
    const bool has = (int)threadIdx.x < a.top;
    Kept mine = {-1, -INFINITY, 0.0f};
    if (has) mine = fetch((int)threadIdx.x);

    // ---- first pass: softmax statistics of the row
    SoftStat st = {-INFINITY, 0.0f};
    if (MODE & kWantLoss) {
        bool gathered = false;
        for (int v = part.v_lo + (int)threadIdx.x; v < part.v_hi; v += kBatch * kThreads) {
            uint4 raw[kBatch];
            part.load(v, raw);
            if (held) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (v + i * kThreads < part.v_hi) copy[v + i * kThreads - part.v_lo] = raw[i];
            }
            soft_batch<DT>(raw, a.c, st);
            if (!gathered) gather(mine);   // on its way while the next batch is
            gathered = true;
        }
        if (!gathered) gather(mine);
        if (lone >= 0) st = soft_merge(st, soft_one(lone_x, a.c), a.c);
        st = soft_warp(st, a.c);
        if (lane == 0) warp_stat[warp] = st;
    } else {
        gather(mine);
    }
    if (has) {
        count_in(mine);
        kept[threadIdx.x] = mine;
        for (int i = (int)threadIdx.x + kThreads; i < a.top; i += kThreads) {
            Kept k = fetch(i);
            gather(k);
            count_in(k);
            kept[i] = k;
        }
    }
    if (warp * 32 < a.top) {
        if (given) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) kst.s = __fadd_rn(kst.s, __shfl_xor_sync(0xFFFFFFFFu, kst.s, o));
        } else {
            kst = soft_warp(kst, a.c);
        }
        if (lane == 0) kept_stat[warp] = kst;
    }
    if (MODE & kWantGrad) {
        if (threadIdx.x == 0) doubled = 0;
        for (int i = threadIdx.x; i < a.slots; i += kThreads) table[i] = 0xFFFFFFFFu;
    }
    if (n_ctas > 1) cluster_wait();
    __syncthreads();
    const int kept_warps = a.top < kThreads ? (a.top + 31) / 32 : kWarps;
    float mass;   // P
    if (given) {
        mass = lane < kept_warps ? kept_stat[lane].s : 0.0f;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) mass = __fadd_rn(mass, __shfl_xor_sync(0xFFFFFFFFu, mass, o));
    } else {
        kst = soft_all(kept_stat, kept_warps, a.c);
        mass = kst.s == 0.0f ? 0.0f : (kst.s < INFINITY ? 1.0f : NAN);   // NaN and +inf among the kept logits: NaN
    }
    if (MODE & kWantLoss) {
        st = soft_all(warp_stat, kWarps, a.c);
        if (n_ctas > 1) {
            if (threadIdx.x < n_ctas) *cluster.map_shared_rank(&cta_stat[rank], threadIdx.x) = st;
            cluster.sync();   // also: every CTA has gathered its kept entries' logits
            st = soft_all(cta_stat, n_ctas, a.c);
        }
    }
    const bool zero = weight == 0.0f || mass == 0.0f;
    const float kept_inv = __fdividef(1.0f, kst.s), kept_ref = soft_ref(kst.m);
    auto prob = [&](float t) -> float {
        if (t == -INFINITY) return 0.0f;
        return given ? teacher_p(t, t_lse, a.inv_t) : __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(t, kept_ref), a.c)), kept_inv);
    };

    // ---- gradient
    if (MODE & kWantGrad) {
        const float coef = __fmul_rn(__fmul_rn(__fmul_rn(a.grad_rows != nullptr ? a.grad_rows[r] : 1.0f, a.grad_scale), weight), a.t);
        // coef P q_j = 2^((x_j - ref) c) * dense:  the row's maximum and 1 / sum, or T times the saved log-sum-exp
        // (rounded, and what the rounding left out as a factor)
        float ref = soft_ref(st.m), dense = __fmul_rn(coef, mass);
        if (MODE & kWantLoss) {
            dense = __fdiv_rn(dense, st.s);
        } else if (!zero) {
            const double at = (double)a.lse[r] * (double)a.t;
            ref = (float)at;
            if (fabsf(ref) <= 3.402823466e38f) dense = __fmul_rn(dense, exp2_fast(__fmul_rn((float)((double)ref - at), a.c)));
        }
        const Pair minus_ref = pair_of(-ref, -ref), cc = pair_of(a.c, a.c), dd = pair_of(dense, dense);
        auto dense_of = [&](float x) -> float { return __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(x, ref), a.c)), dense); };
        auto dense_vec = [&](const uint4& w) -> uint4 {
            float f[RV::kElems];
#pragma unroll
            for (int e = 0; e < RV::kElems; e += 2) split(mul2(soft_pair(RV::get(w, e), RV::get(w, e + 1), minus_ref, cc), dd), f[e], f[e + 1]);
            return RV::pack(f);
        };
        Elem* out = reinterpret_cast<Elem*>(a.dS) + r * a.ldd;
        const bool aligned = (reinterpret_cast<uintptr_t>(out + part.head) & 15u) == 0;
        auto store = [&](int v, const uint4& w) {
            Elem* o = out + part.first(v);
            if (aligned) {
                st_stream16(o, w);
            } else {
#pragma unroll
                for (int e = 0; e < RV::kElems; ++e) o[e] = RV::bits(w, e);
            }
        };
        if (lone >= 0) out[lone] = zero ? (Elem)0 : RV::narrow(dense_of(lone_x));
        if (zero) {
            for (int v = part.v_lo + (int)threadIdx.x; v < part.v_hi; v += kThreads) store(v, make_uint4(0u, 0u, 0u, 0u));
        } else if (held) {
            for (int v = part.v_lo + (int)threadIdx.x; v < part.v_hi; v += kThreads) store(v, dense_vec(copy[v - part.v_lo]));
        } else {
            for (int v = part.v_lo + (int)threadIdx.x; v < part.v_hi; v += kBatch * kThreads) {
                uint4 raw[kBatch];
                part.load(v, raw);
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (v + i * kThreads < part.v_hi) store(v + i * kThreads, dense_vec(raw[i]));
            }
        }
        if (!zero) {
            for (int i = threadIdx.x; i < a.top; i += kThreads) {
                const Kept k = kept[i];
                kept_prob[i] = prob(k.t);
                if (k.j >= 0) {   // open addressing; a second entry for the same place is noted
                    uint32_t h = ((uint32_t)k.j * 2654435761u) & (uint32_t)(a.slots - 1);
                    for (;;) {
                        const uint32_t old = atomicCAS(&table[h], 0xFFFFFFFFu, (uint32_t)k.j);
                        if (old == 0xFFFFFFFFu) break;
                        if (old == (uint32_t)k.j) {
                            doubled = 1;
                            break;
                        }
                        h = (h + 1u) & (uint32_t)(a.slots - 1);
                    }
                }
            }
        }
        __syncthreads();   // the dense values of this CTA's part are written, the table is complete
        // the kept entries' places: their whole value, from the gathered logit
        if (!zero) {
            for (int i = threadIdx.x; i < a.top; i += kThreads) {
                const Kept k = kept[i];
                if (k.j < 0 || !part.owns(k.j)) continue;
                float p = kept_prob[i];
                if (doubled) {   // every copy of the entry writes the same sum
                    p = 0.0f;
                    for (int o = 0; o < a.top; ++o)
                        if (kept[o].j == k.j) p = __fadd_rn(p, kept_prob[o]);
                }
                out[k.j] = RV::narrow(__fsub_rn(dense_of(k.x), __fmul_rn(coef, p)));
            }
        }
    }

    // ---- the loss, last: the row's gradient is on its way by then.  In fp64: differences of logarithms that nearly cancel.
    if ((MODE & kWantLoss) && rank == 0) {
        double sum = 0.0;
        if (warp * 32 < a.top) {
            const double lse = soft_lse(st, a.inv_t), norm = given ? (double)t_lse : soft_lse(kst, a.inv_t);
            if (threadIdx.x == 0 && a.lse != nullptr) a.lse[r] = (float)lse;
            for (int i = threadIdx.x; i < a.top; i += kThreads) {
                const Kept k = kept[i];
                const float p = prob(k.t);
                if (p != 0.0f) sum += (double)p * (((double)k.t * a.inv_t - norm) - ((double)k.x * a.inv_t - lse));
            }
            sum = warp_sum(sum);
            if (lane == 0) warp_loss[warp] = sum;
        }
        if (a.top > 32) __syncthreads();
        if (threadIdx.x == 0) {
            double total = sum;   // the first warp's
            for (int w = 1; w < kept_warps; ++w) total += warp_loss[w];
            a.loss[r] = zero ? 0.0f : (float)((double)weight * (double)a.t * (double)a.t * total);
        }
    }
}

template <int DT, int MODE> int launch_distill(DistillArgs a, cudaStream_t st) {
    const int c = row_cluster(a.rows, row_vectors(a.vocab, DT));
    a.ahead = rows_ahead(c);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    cfg.blockDim = dim3(kThreads);
    // both wanted: a copy of the CTA's part, if it is one that a CTA takes (64 KB); the kept entries: at most 24 KB
    const int64_t per = (row_vectors(a.vocab, DT) + c - 1) / c;
    a.copy_vecs = MODE == (kWantLoss | kWantGrad) && per <= kPartVecs ? (int)per : 0;
    cfg.dynamicSmemBytes = (size_t)a.copy_vecs * 16u + (size_t)a.top * 16u + (size_t)a.slots * 4u;
    static DeviceCache opted;   // the shared-memory opt-in belongs to one device's copy of the kernel
    const int ok = opted.get([&]() -> int {
        if (cudaFuncSetAttribute(distill_kernel<DT, MODE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPartVecs * 16 + 24 * 1024) != cudaSuccess) {
            (void)cudaGetLastError();
            return -1;
        }
        return 1;
    });
    if (ok < 0) return MOSAIC_ERR_CUDA;
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
