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

// What a row's gradient needs:  coef P q_j = 2^((x_j - ref) c) * dense.
struct RowScale {
    float dense;   // with the loss: coef P, to be divided by the row's sum; from a saved log-sum-exp: complete
    float ref;     // from a saved log-sum-exp: T times it
    float coef;
    int live;      // 0: the row counts for nothing, 2: some vocabulary entry is kept twice
};

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
    double inv_t;
    float t, c;       // T, log2(e) / T
    int copy_vecs;    // vectors of the copy in shared memory (0: none)
    int first_wave;   // CTAs of the vocabulary kernel that run at once
    int slots;        // of the table of kept places: a power of two, at least 2 * top
    float* loss;
    float* lse;
    // workspace
    RowScale* scale;    // [rows]
    float2* stat;       // [rows] maximum and sum of the row
    double* row_norm;   // [rows] log of what the kept exponentials are divided by
    float2* kept;       // [rows, top] the kept entries' probabilities and the student's logits there
};

constexpr int kWantLoss = 1, kWantGrad = 2;

// A kept logit's probability under the teacher's own log-sum-exp.
__device__ __forceinline__ float teacher_p(float t, float t_lse, double inv_t) { return expf((float)((double)t * inv_t - (double)t_lse)); }

__device__ __forceinline__ float dense_of(float x, float ref, float dense, float c) { return __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(x, ref), c)), dense); }

// The call's launches, each of which may start under the one before it:
//   kept_kernel    the kept entries of all rows: gathers, probabilities, P, what the gradient of a row is scaled by
//   vocab_kernel   the whole vocabulary: softmax statistics and the dense gradient, P q
//   place_kernel   the loss, and the kept entries' places in the gradient, P q - p
// The loss alone needs the second, and a third that is both others at once.  All of the kept entries' work inside
// vocab_kernel made every row's barriers wait for the warps that did it: 137 us for the loss and gradient of 4096 x
// 32000 bf16, 125 us with a warp of its own for it, and 10 us for the sum of p alone.
//
// The kept entries' two launches are chains of dependent loads (place -> logit), so they are laid out for many rows in
// flight: a row's entries, four a thread at most and all asked for at once, by a warp (up to 128 of them; four rows a
// CTA) or by a CTA of eight.
constexpr int kKeptEach = 4;
constexpr int kKeptWarpRows = 4;
template <bool WARP> struct KeptShape {
    static constexpr int kThreads = WARP ? 32 * kKeptWarpRows : kMaxTop / kKeptEach;
    static constexpr int kGroup = WARP ? 32 : kThreads;      // threads of a row
    static constexpr int kRows = kThreads / kGroup;
};
template <bool WARP> struct KeptShared {
    SoftStat stat[8];
    double sum[8];
};
template <bool WARP> __device__ __forceinline__ int kept_rank() { return WARP ? (int)threadIdx.x & 31 : (int)threadIdx.x; }
template <bool WARP> __device__ __forceinline__ int64_t kept_row() { return WARP ? (int64_t)blockIdx.x * kKeptWarpRows + (threadIdx.x >> 5) : (int64_t)blockIdx.x; }
template <bool WARP> __device__ __forceinline__ void kept_sync() {
    if (WARP) __syncwarp();
    else __syncthreads();
}
// Sum over the row's threads, in each of them.
template <bool WARP> __device__ __forceinline__ double kept_sum(double v, KeptShared<WARP>& sh) {
    v = warp_sum(v);
    if (!WARP) {
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sh.sum[threadIdx.x >> 5] = v;
        __syncthreads();
        v = 0.0;
        for (int w = 0; w < 8; ++w) v += sh.sum[w];
    }
    return v;
}

// One row's kept entries in the hands of its threads.
template <int DT, bool WARP> struct KeptRow {
    using RV = RowVec<DT>;
    int j[kKeptEach];      // place, -1: absent
    float t[kKeptEach];    // the teacher's logit
    float x[kKeptEach];    // the student's there
    SoftStat st;           // renormalised: the kept logits' statistics
    float inv;             // 1 / st.s
    float t_lse;
    bool given;

    __device__ __forceinline__ KeptRow(const DistillArgs& a, int64_t r, KeptShared<WARP>& sh) {
        const int me = kept_rank<WARP>();
        given = a.t_lse != nullptr;
        t_lse = given ? a.t_lse[r] : 0.0f;
        const typename RV::Elem* row = reinterpret_cast<const typename RV::Elem*>(a.S) + r * a.lds;
#pragma unroll
        for (int e = 0; e < kKeptEach; ++e) {
            const int i = me + e * KeptShape<WARP>::kGroup;
            j[e] = i < a.top ? a.t_indices[r * a.top + i] : -1;
            t[e] = i < a.top ? a.t_values[r * a.top + i] : 0.0f;
        }
        st = {-INFINITY, 0.0f};
#pragma unroll
        for (int e = 0; e < kKeptEach; ++e) {
            if (j[e] < 0 || j[e] >= (int)a.vocab) j[e] = -1;
            x[e] = j[e] >= 0 ? RV::widen(row[j[e]]) : 0.0f;
            if (j[e] < 0) t[e] = -INFINITY;
            st.m = fmaxf(st.m, t[e]);
        }
        if (!given) {
#pragma unroll
            for (int e = 0; e < kKeptEach; ++e) st.s = __fadd_rn(st.s, exp2_fast(__fmul_rn(__fsub_rn(t[e], soft_ref(st.m)), a.c)));
            st = soft_warp(st, a.c);
            if (!WARP) {
                if ((threadIdx.x & 31) == 0) sh.stat[threadIdx.x >> 5] = st;
                __syncthreads();
                st = soft_all(sh.stat, 8, a.c);
            }
        }
        inv = __fdividef(1.0f, st.s);
    }
    __device__ __forceinline__ float prob(int e, const DistillArgs& a) const {
        if (t[e] == -INFINITY) return 0.0f;
        return given ? teacher_p(t[e], t_lse, a.inv_t) : __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(t[e], soft_ref(st.m)), a.c)), inv);
    }
    // log of what the kept exponentials are divided by
    __device__ __forceinline__ double norm(const DistillArgs& a) const { return given ? (double)t_lse : soft_lse(st, a.inv_t); }
};

template <int DT, int MODE, bool WARP> __global__ void __launch_bounds__(KeptShape<WARP>::kThreads) kept_kernel(const __grid_constant__ DistillArgs a) {
    extern __shared__ uint32_t tables[];   // [rows of the CTA][slots] places seen, to find doubled ones
    __shared__ KeptShared<WARP> sh;
    allow_next_kernel();
    const int64_t r = kept_row<WARP>();
    const int me = kept_rank<WARP>();
    if (WARP && r >= a.rows) return;
    uint32_t* table = tables + (WARP ? (threadIdx.x >> 5) * a.slots : 0);
    const float weight = a.row_weight != nullptr ? a.row_weight[r] : 1.0f;
    const float g = a.grad_rows != nullptr ? a.grad_rows[r] : 1.0f;
    const float saved_lse = MODE == kWantGrad ? a.lse[r] : 0.0f;
    for (int i = me; i < a.slots; i += KeptShape<WARP>::kGroup) table[i] = 0xFFFFFFFFu;
    KeptRow<DT, WARP> k(a, r, sh);
    kept_sync<WARP>();
    float mass = 0.0f;
    bool doubled = false;   // some vocabulary entry is kept twice
#pragma unroll
    for (int e = 0; e < kKeptEach; ++e) {
        const int i = me + e * KeptShape<WARP>::kGroup, j = k.j[e];
        const float p = k.prob(e, a);
        mass = __fadd_rn(mass, p);
        if (i < a.top) a.kept[r * a.top + i] = make_float2(p, k.x[e]);
        if (j < 0) continue;
        uint32_t h = ((uint32_t)j * 2654435761u) & (uint32_t)(a.slots - 1);   // open addressing
        for (;;) {
            const uint32_t old = atomicCAS(&table[h], 0xFFFFFFFFu, (uint32_t)j);
            if (old == 0xFFFFFFFFu) break;
            if (old == (uint32_t)j) {
                doubled = true;
                break;
            }
            h = (h + 1u) & (uint32_t)(a.slots - 1);
        }
    }
    doubled = WARP ? __any_sync(0xFFFFFFFFu, doubled) : __syncthreads_or(doubled) != 0;
    if (k.given) mass = (float)kept_sum<WARP>((double)mass, sh);
    else mass = k.st.s == 0.0f ? 0.0f : (k.st.s < INFINITY ? 1.0f : NAN);   // NaN and +inf among the kept logits: NaN
    if (me == 0) {
        RowScale s;
        s.coef = __fmul_rn(__fmul_rn(__fmul_rn(g, a.grad_scale), weight), a.t);
        s.dense = __fmul_rn(s.coef, mass);
        s.ref = 0.0f;
        s.live = weight == 0.0f || mass == 0.0f ? 0 : (doubled ? 2 : 1);
        if (MODE == kWantGrad) {   // T times the saved log-sum-exp, rounded, and what the rounding left out as a factor
            const double at = (double)saved_lse * (double)a.t;
            s.ref = (float)at;
            if (fabsf(s.ref) <= 3.402823466e38f) s.dense = __fmul_rn(s.dense, exp2_fast(__fmul_rn((float)((double)s.ref - at), a.c)));
        }
        a.scale[r] = s;
        if (MODE & kWantLoss) a.row_norm[r] = k.norm(a);
    }
}

// One row by a CTA or a cluster of them.  MODE: what is wanted; with kWantGrad alone the saved log-sum-exp is an input.
//   loss alone   one pass over the row for its softmax statistics
//   gradient     one pass that reads and writes
//   both         the first pass leaves the CTA's part of the row in shared memory, the second reads it there
// Bound by memory and the exponentials together: loss and gradient of 4096 x 32000 bf16 take 98 us, DRAM 59 % busy and
// an instruction issued in 71 % of the cycles; a copy of the same bytes takes 84 us.  Three CTAs of 512 an SM: 116 us for the
// call against 127 with two, 128 with four (32 registers), 136 with six of 256 (their copies of a row do not fit).
template <int DT, int MODE, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, kRowCtas) vocab_kernel(const __grid_constant__ DistillArgs a) {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    constexpr bool kLoss = (MODE & kWantLoss) != 0, kGrad = (MODE & kWantGrad) != 0;
    __shared__ SoftStat warp_stat[kWarps];
    __shared__ SoftStat cta_stat[kMaxCluster];   // written by the CTAs of the cluster
    extern __shared__ uint4 copy[];              // the CTA's part of the row (both wanted)

    cg::cluster_group cluster = cg::this_cluster();
    const int n_ctas = CLUSTER ? (int)cluster.num_blocks() : 1, rank = CLUSTER ? (int)cluster.block_rank() : 0;
    const int64_t r = CLUSTER ? blockIdx.x >> (__ffs(n_ctas) - 1) : blockIdx.x;   // a power of two
    const int vocab = (int)a.vocab;
    const RowPart<DT> part(a.S, r, a.lds, vocab, rank, n_ctas);
    const bool held = kGrad && kLoss && part.v_hi - part.v_lo <= a.copy_vecs;
    allow_next_kernel();
    if (CLUSTER && kLoss) cluster_arrive();   // waited for before the first write to another CTA
    // the kept entries' launch is most likely over when a CTA of a later wave starts; the first wave waits after its pass
    const bool late = (int)blockIdx.x < a.first_wave;
    RowScale scale = {0.0f, 0.0f, 0.0f, 0};
    if (kGrad && !(kLoss && late)) {
        await_previous_kernel();
        scale = a.scale[r];
    }

    const int v0 = part.v_lo + (int)threadIdx.x;
    const int lone = part.single();
    const float lone_x = lone >= 0 ? part.at(lone) : -INFINITY;
    uint4 raw[kBatch];
    SoftStat st = {-INFINITY, 0.0f};
    if (kLoss) {
        for (int v = v0; v < part.v_hi; v += kBatch * kThreads) {
            part.load(v, raw);
            if (held) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (v + i * kThreads < part.v_hi) copy[v + i * kThreads - part.v_lo] = raw[i];
            }
            soft_batch<DT>(raw, batch_max<DT>(raw), a.c, st);
        }
        if (lone >= 0) st = soft_merge(st, soft_one(lone_x, a.c), a.c);
        st = soft_warp(st, a.c);
        if ((threadIdx.x & 31) == 0) warp_stat[threadIdx.x >> 5] = st;
        if (kGrad && late) {
            await_previous_kernel();
            scale = a.scale[r];
        }
        if (CLUSTER) cluster_wait();
        __syncthreads();
        if (!kGrad && threadIdx.x >= 32 && !CLUSTER) return;
        st = soft_all(warp_stat, kWarps, a.c);
        if (CLUSTER) {
            if (threadIdx.x < n_ctas) *cluster.map_shared_rank(&cta_stat[rank], threadIdx.x) = st;
            cluster.sync();
            st = soft_all(cta_stat, n_ctas, a.c);
        }
        if (rank == 0 && threadIdx.x == 0) a.stat[r] = make_float2(st.m, st.s);
    }
    if (!kGrad) return;

    // ---- gradient; a row that counts for nothing gets zeros whatever it holds
    const float ref = kLoss ? soft_ref(st.m) : scale.ref, dense = kLoss ? __fdiv_rn(scale.dense, st.s) : scale.dense;
    const Pair minus_ref = pair_of(-ref, -ref), cc = pair_of(a.c, a.c), dd = pair_of(dense, dense);
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
    if (lone >= 0) out[lone] = scale.live ? RV::narrow(dense_of(lone_x, ref, dense, a.c)) : (Elem)0;
    if (!scale.live) {
        for (int v = v0; v < part.v_hi; v += kThreads) store(v, make_uint4(0u, 0u, 0u, 0u));
        return;
    }
    for (int v = v0; v < part.v_hi; v += kBatch * kThreads) {
        if (held) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (v + i * kThreads < part.v_hi) raw[i] = copy[v + i * kThreads - part.v_lo];
        } else {
            part.load(v, raw);
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (v + i * kThreads < part.v_hi) {
                float f[RV::kElems];
#pragma unroll
                for (int e = 0; e < RV::kElems; e += 2)
                    split(mul2(soft_pair(RV::get(raw[i], e), RV::get(raw[i], e + 1), minus_ref, cc), dd), f[e], f[e + 1]);
                store(v + i * kThreads, RV::pack(f));
            }
        }
    }
}

template <int DT, int MODE, bool WARP> __global__ void __launch_bounds__(KeptShape<WARP>::kThreads) place_kernel(const __grid_constant__ DistillArgs a) {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    constexpr bool kLoss = (MODE & kWantLoss) != 0, kGrad = (MODE & kWantGrad) != 0;
    constexpr int kGroup = KeptShape<WARP>::kGroup;
    __shared__ KeptShared<WARP> sh;
    const int64_t r = kept_row<WARP>();
    const int me = kept_rank<WARP>();
    if (WARP && r >= a.rows) return;
    const float weight = a.row_weight != nullptr ? a.row_weight[r] : 1.0f;
    double sum = 0.0, lse = 0.0;
    if constexpr (!kGrad) {   // the kept entries, all of it
        const KeptRow<DT, WARP> k(a, r, sh);
        const double norm = k.norm(a);
        await_previous_kernel();
        const float2 stat = a.stat[r];
        lse = soft_lse({stat.x, stat.y}, a.inv_t);
#pragma unroll
        for (int e = 0; e < kKeptEach; ++e) {   // in fp64: differences of logarithms that nearly cancel
            const float p = k.prob(e, a);
            if (p != 0.0f) sum += (double)p * (((double)k.t[e] * a.inv_t - norm) - ((double)k.x[e] * a.inv_t - lse));
        }
    } else {
        int j[kKeptEach];
        float t[kKeptEach];
        float2 px[kKeptEach];
#pragma unroll
        for (int e = 0; e < kKeptEach; ++e) {
            const int i = me + e * kGroup;
            j[e] = i < a.top ? a.t_indices[r * a.top + i] : -1;
            t[e] = kLoss && i < a.top ? a.t_values[r * a.top + i] : 0.0f;
        }
        await_previous_kernel();
        const RowScale s = a.scale[r];
        const float2 stat = kLoss ? a.stat[r] : make_float2(0.0f, 0.0f);
        const double norm = kLoss ? a.row_norm[r] : 0.0;
#pragma unroll
        for (int e = 0; e < kKeptEach; ++e) {
            const int i = me + e * kGroup;
            px[e] = i < a.top ? a.kept[r * a.top + i] : make_float2(0.0f, 0.0f);
        }
        if (s.live) {   // the kept places' whole value, from the gathered logit
            const float ref = kLoss ? soft_ref(stat.x) : s.ref, dense = kLoss ? __fdiv_rn(s.dense, stat.y) : s.dense;
            Elem* out = reinterpret_cast<Elem*>(a.dS) + r * a.ldd;
#pragma unroll
            for (int e = 0; e < kKeptEach; ++e) {
                if (j[e] < 0 || j[e] >= (int)a.vocab) continue;
                float p = px[e].x;
                if (s.live == 2) {   // some entry occurs twice: every copy writes the same sum
                    p = 0.0f;
                    for (int o = 0; o < a.top; ++o)
                        if (a.t_indices[r * a.top + o] == j[e]) p = __fadd_rn(p, a.kept[r * a.top + o].x);
                }
                out[j[e]] = RV::narrow(__fsub_rn(dense_of(px[e].y, ref, dense, a.c), __fmul_rn(s.coef, p)));
            }
        }
        if (!kLoss) return;
        lse = soft_lse({stat.x, stat.y}, a.inv_t);
#pragma unroll
        for (int e = 0; e < kKeptEach; ++e)
            if (px[e].x != 0.0f) sum += (double)px[e].x * (((double)t[e] * a.inv_t - norm) - ((double)px[e].y * a.inv_t - lse));
    }
    sum = kept_sum<WARP>(sum, sh);
    if (me == 0) {
        a.loss[r] = weight == 0.0f ? 0.0f : (float)((double)weight * (double)a.t * (double)a.t * sum);
        if (a.lse != nullptr) a.lse[r] = (float)lse;
    }
}

// The launches before and after the vocabulary's.
template <int DT, int MODE, bool WARP> int launch_kept(const DistillArgs& a, bool first, cudaLaunchAttribute* overlap, cudaStream_t st) {
    using Shape = KeptShape<WARP>;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.rows + Shape::kRows - 1) / Shape::kRows));
    cfg.blockDim = dim3(Shape::kThreads);
    cfg.stream = st;
    if (first) {
        cfg.dynamicSmemBytes = (size_t)Shape::kRows * (size_t)a.slots * 4u;   // at most 8 KB
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, kept_kernel<DT, MODE, WARP>, a));
    } else {
        cfg.attrs = overlap;
        cfg.numAttrs = 1;
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, place_kernel<DT, MODE, WARP>, a));
    }
    return MOSAIC_OK;
}

template <int DT, int MODE> int launch_distill(DistillArgs a, cudaStream_t st) {
    const int c = row_cluster(a.rows, row_vectors(a.vocab, DT));
    // both wanted: a copy of the CTA's part, if it is one that a CTA takes (64 KB)
    const int64_t per = (row_vectors(a.vocab, DT) + c - 1) / c;
    a.copy_vecs = MODE == (kWantLoss | kWantGrad) && per <= kPartVecs ? (int)per : 0;
    a.first_wave = sm_count() * kRowCtas;
    static DeviceCache opted;   // the shared-memory opt-in belongs to one device's copy of a kernel
    const int ok = opted.get([&]() -> int {
        if (cudaFuncSetAttribute(vocab_kernel<DT, MODE, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPartVecs * 16) != cudaSuccess ||
            cudaFuncSetAttribute(vocab_kernel<DT, MODE, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPartVecs * 16) != cudaSuccess) {
            (void)cudaGetLastError();
            return -1;
        }
        return 1;
    });
    if (ok < 0) return MOSAIC_ERR_CUDA;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)c;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    const bool warp_rows = a.top <= 32 * kKeptEach;
    if (MODE & kWantGrad) {
        const int rc = warp_rows ? launch_kept<DT, MODE, true>(a, true, attr, st) : launch_kept<DT, MODE, false>(a, true, attr, st);
        if (rc != MOSAIC_OK) return rc;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)a.copy_vecs * 16u;
    cfg.stream = st;
    cfg.attrs = (MODE & kWantGrad) ? attr : attr + 1;
    cfg.numAttrs = ((MODE & kWantGrad) ? 1 : 0) + (c > 1 ? 1 : 0);
    if (c > 1) MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, vocab_kernel<DT, MODE, true>, a));
    else MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, vocab_kernel<DT, MODE, false>, a));
    return warp_rows ? launch_kept<DT, MODE, true>(a, false, attr, st) : launch_kept<DT, MODE, false>(a, false, attr, st);
}

bool overlap(const void* a, size_t an, const void* b, size_t bn) {
    const char *x = static_cast<const char*>(a), *y = static_cast<const char*>(b);
    return x != nullptr && y != nullptr && an > 0 && bn > 0 && x < y + bn && y < x + an;
}
size_t span(int64_t rows, int64_t cols, int64_t ld, size_t elem) { return ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * elem; }

template <int MODE> int distill(DistillArgs a, int64_t top, float temperature, int dtype, void* ws, size_t ws_bytes, void* stream) {
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
    const size_t need = mosaic_distill_workspace_bytes(a.rows, top);
    if (ws == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return MOSAIC_ERR_MISALIGNED;
    if (ws_bytes < need) return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
    a.scale = static_cast<RowScale*>(ws);
    a.stat = reinterpret_cast<float2*>(a.scale + n);
    a.row_norm = reinterpret_cast<double*>(a.stat + n);
    a.kept = reinterpret_cast<float2*>(a.row_norm + n);
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

extern "C" size_t mosaic_distill_workspace_bytes(int64_t rows, int64_t top) {
    if (rows <= 0 || top <= 0) return 0;
    return align_up((size_t)rows * (sizeof(RowScale) + 8u + 8u + (size_t)top * 8u), 256);
}

extern "C" int mosaic_distill_loss(const void* S, int64_t rows, int64_t vocab, int64_t lds, int dtype, const float* t_values,
                                   const int32_t* t_indices, int64_t top, const float* t_lse, const float* row_weight, float temperature,
                                   float* loss, float* lse, void* ws, size_t ws_bytes, void* stream) {
    DistillArgs a = {};
    a.S = S; a.rows = rows; a.vocab = vocab; a.lds = lds;
    a.t_values = t_values; a.t_indices = t_indices; a.t_lse = t_lse; a.row_weight = row_weight;
    a.loss = loss; a.lse = lse;
    return distill<kWantLoss>(a, top, temperature, dtype, ws, ws_bytes, stream);
}

extern "C" int mosaic_distill_grad(const void* S, int64_t rows, int64_t vocab, int64_t lds, int dtype, const float* t_values,
                                   const int32_t* t_indices, int64_t top, const float* t_lse, const float* row_weight, float temperature,
                                   const float* lse, const float* grad_rows, float grad_scale, void* dS, int64_t ldd, void* ws, size_t ws_bytes,
                                   void* stream) {
    DistillArgs a = {};
    a.S = S; a.rows = rows; a.vocab = vocab; a.lds = lds; a.dS = dS; a.ldd = ldd;
    a.t_values = t_values; a.t_indices = t_indices; a.t_lse = t_lse; a.row_weight = row_weight;
    a.lse = const_cast<float*>(lse); a.grad_rows = grad_rows; a.grad_scale = grad_scale;
    return distill<kWantGrad>(a, top, temperature, dtype, ws, ws_bytes, stream);
}

extern "C" int mosaic_distill_loss_grad(const void* S, int64_t rows, int64_t vocab, int64_t lds, int dtype, const float* t_values,
                                        const int32_t* t_indices, int64_t top, const float* t_lse, const float* row_weight, float temperature,
                                        float* loss, float* lse, const float* grad_rows, float grad_scale, void* dS, int64_t ldd, void* ws, size_t ws_bytes,
                                   void* stream) {
    DistillArgs a = {};
    a.S = S; a.rows = rows; a.vocab = vocab; a.lds = lds; a.dS = dS; a.ldd = ldd;
    a.t_values = t_values; a.t_indices = t_indices; a.t_lse = t_lse; a.row_weight = row_weight;
    a.loss = loss; a.lse = lse; a.grad_rows = grad_rows; a.grad_scale = grad_scale;
    return distill<kWantLoss | kWantGrad>(a, top, temperature, dtype, ws, ws_bytes, stream);
}
