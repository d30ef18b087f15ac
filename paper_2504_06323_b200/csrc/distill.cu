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
    int live;      // 0: the row counts for nothing
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
    int* doubled;       // [rows] some vocabulary entry is kept twice
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
constexpr int kKeptWarps = 8;
inline int kept_warps(int top) { return top <= 64 ? 1 : top >= 64 * kKeptWarps ? kKeptWarps : (top + 63) / 64; }

// One row's kept entries in the hands of a CTA of one to eight warps.  Shared memory: [top] each of place, teacher's
// logit, student's logit; [slots] of the table (gradient).
template <int DT> struct KeptRow {
    using RV = RowVec<DT>;
    int* j;            // -1: absent
    float* t;
    float* x;
    uint32_t* table;
    SoftStat st;       // renormalised: the kept logits' statistics
    double norm;       // log of what the kept exponentials are divided by
    float inv;         // 1 / st.s
    float t_lse;
    bool given;

    __device__ __forceinline__ KeptRow(const DistillArgs& a, int64_t r, unsigned char* dyn, SoftStat* warp_stat) {
        j = reinterpret_cast<int*>(dyn);
        t = reinterpret_cast<float*>(j + a.top);
        x = t + a.top;
        table = reinterpret_cast<uint32_t*>(x + a.top);
        given = a.t_lse != nullptr;
        t_lse = given ? a.t_lse[r] : 0.0f;
        const typename RV::Elem* row = reinterpret_cast<const typename RV::Elem*>(a.S) + r * a.lds;
        const int n = (int)blockDim.x, warps = n >> 5;
        st = {-INFINITY, 0.0f};
        for (int i = threadIdx.x; i < a.top; i += n) {
            int at = a.t_indices[r * a.top + i];
            if (at < 0 || at >= (int)a.vocab) at = -1;
            const float v = at >= 0 ? a.t_values[r * a.top + i] : -INFINITY;
            j[i] = at;
            t[i] = v;
            x[i] = at >= 0 ? RV::widen(row[at]) : 0.0f;
            if (!given) st = soft_merge(st, soft_one(v, a.c), a.c);
        }
        if (!given) {
            st = soft_warp(st, a.c);
            if (warps > 1) {
                if ((threadIdx.x & 31) == 0) warp_stat[threadIdx.x >> 5] = st;
                __syncthreads();
                st = soft_all(warp_stat, warps, a.c);
            }
        }
        inv = __fdividef(1.0f, st.s);
        norm = given ? (double)t_lse : soft_lse(st, a.inv_t);
    }
    __device__ __forceinline__ float prob(int i, const DistillArgs& a) const {
        const float v = t[i];
        if (v == -INFINITY) return 0.0f;
        return given ? teacher_p(v, t_lse, a.inv_t) : __fmul_rn(exp2_fast(__fmul_rn(__fsub_rn(v, soft_ref(st.m)), a.c)), inv);
    }
};
// Sum over the CTA, in thread 0; `part` holds a warp's each.  With a barrier, if there is more than one warp.
template <class T> __device__ __forceinline__ T kept_sum(T v, T* part) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    const int warps = (int)blockDim.x >> 5;
    if (warps == 1) return v;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < warps; ++w) v += part[w];
    return v;
}

template <int DT, int MODE> __global__ void __launch_bounds__(32 * kKeptWarps) kept_kernel(const __grid_constant__ DistillArgs a) {
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ SoftStat warp_stat[kKeptWarps];
    __shared__ float warp_mass[kKeptWarps];
    allow_next_kernel();
    const int64_t r = blockIdx.x;
    const int n = (int)blockDim.x;
    const float weight = a.row_weight != nullptr ? a.row_weight[r] : 1.0f;
    const float g = a.grad_rows != nullptr ? a.grad_rows[r] : 1.0f;
    const float saved_lse = MODE == kWantGrad ? a.lse[r] : 0.0f;
    KeptRow<DT> k(a, r, dyn, warp_stat);
    for (int i = threadIdx.x; i < a.slots; i += n) k.table[i] = 0xFFFFFFFFu;
    __syncthreads();
    float mass = 0.0f;
    bool doubled = false;   // some vocabulary entry is kept twice
    for (int i = threadIdx.x; i < a.top; i += n) {
        const float p = k.prob(i, a);
        const int j = k.j[i];
        mass = __fadd_rn(mass, p);
        a.kept[r * a.top + i] = make_float2(p, k.x[i]);
        if (j < 0) continue;
        uint32_t h = ((uint32_t)j * 2654435761u) & (uint32_t)(a.slots - 1);   // open addressing
        for (;;) {
            const uint32_t old = atomicCAS(&k.table[h], 0xFFFFFFFFu, (uint32_t)j);
            if (old == 0xFFFFFFFFu) break;
            if (old == (uint32_t)j) {
                doubled = true;
                break;
            }
            h = (h + 1u) & (uint32_t)(a.slots - 1);
        }
    }
    doubled = __syncthreads_or(doubled) != 0;
    mass = kept_sum(mass, warp_mass);
    if (threadIdx.x == 0) {
        if (!k.given) mass = k.st.s == 0.0f ? 0.0f : (k.st.s < INFINITY ? 1.0f : NAN);   // NaN and +inf among the kept logits: NaN
        RowScale s;
        s.coef = __fmul_rn(__fmul_rn(__fmul_rn(g, a.grad_scale), weight), a.t);
        s.dense = __fmul_rn(s.coef, mass);
        s.ref = 0.0f;
        s.live = weight == 0.0f || mass == 0.0f ? 0 : 1;
        if (MODE == kWantGrad) {   // T times the saved log-sum-exp, rounded, and what the rounding left out as a factor
            const double at = (double)saved_lse * (double)a.t;
            s.ref = (float)at;
            if (fabsf(s.ref) <= 3.402823466e38f) s.dense = __fmul_rn(s.dense, exp2_fast(__fmul_rn((float)((double)s.ref - at), a.c)));
        }
        a.scale[r] = s;
        a.row_norm[r] = k.norm;
        a.doubled[r] = doubled ? 1 : 0;
    }
}

// One row by a CTA or a cluster of them.  MODE: what is wanted; with kWantGrad alone the saved log-sum-exp is an input.
//   loss alone   one pass over the row for its softmax statistics
//   gradient     one pass that reads and writes
//   both         the first pass leaves the CTA's part of the row in shared memory, the second reads it there
// Bound by memory: a copy of the same bytes takes 84 us at 4096 x 32000 bf16.
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
            soft_batch<DT>(raw, a.c, st);
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

template <int DT, int MODE> __global__ void __launch_bounds__(32 * kKeptWarps) place_kernel(const __grid_constant__ DistillArgs a) {
    using RV = RowVec<DT>;
    using Elem = typename RV::Elem;
    constexpr bool kLoss = (MODE & kWantLoss) != 0, kGrad = (MODE & kWantGrad) != 0;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ SoftStat warp_stat[kKeptWarps];
    __shared__ double warp_loss[kKeptWarps];
    const int64_t r = blockIdx.x;
    const int n = (int)blockDim.x;
    const float weight = a.row_weight != nullptr ? a.row_weight[r] : 1.0f;
    if (kLoss) {   // in fp64: differences of logarithms that nearly cancel
        double sum = 0.0, lse;
        if constexpr (kGrad) {
            await_previous_kernel();
            const float2 stat = a.stat[r];
            lse = soft_lse({stat.x, stat.y}, a.inv_t);
            const double norm = a.row_norm[r];
            for (int i = threadIdx.x; i < a.top; i += n) {
                const float2 px = a.kept[r * a.top + i];
                if (px.x != 0.0f) sum += (double)px.x * (((double)a.t_values[r * a.top + i] * a.inv_t - norm) - ((double)px.y * a.inv_t - lse));
            }
        } else {
            KeptRow<DT> k(a, r, dyn, warp_stat);
            await_previous_kernel();
            const float2 stat = a.stat[r];
            lse = soft_lse({stat.x, stat.y}, a.inv_t);
            for (int i = threadIdx.x; i < a.top; i += n) {
                const float p = k.prob(i, a);
                if (p != 0.0f) sum += (double)p * (((double)k.t[i] * a.inv_t - k.norm) - ((double)k.x[i] * a.inv_t - lse));
            }
        }
        sum = kept_sum(sum, warp_loss);
        if (threadIdx.x == 0) {
            a.loss[r] = weight == 0.0f ? 0.0f : (float)((double)weight * (double)a.t * (double)a.t * sum);
            if (a.lse != nullptr) a.lse[r] = (float)lse;
        }
    }
    if (kGrad) {
        if (!kLoss) await_previous_kernel();
        const RowScale s = a.scale[r];
        if (!s.live) return;   // zeros already
        const bool doubled = a.doubled[r] != 0;
        float ref = s.ref, dense = s.dense;
        if (kLoss) {
            const float2 stat = a.stat[r];
            ref = soft_ref(stat.x);
            dense = __fdiv_rn(dense, stat.y);
        }
        Elem* out = reinterpret_cast<Elem*>(a.dS) + r * a.ldd;
        for (int i = threadIdx.x; i < a.top; i += n) {   // their whole value, from the gathered logit
            const int j = a.t_indices[r * a.top + i];
            if (j < 0 || j >= (int)a.vocab) continue;
            const float2 px = a.kept[r * a.top + i];
            float p = px.x;
            if (doubled) {   // every copy of the entry writes the same sum
                p = 0.0f;
                for (int o = 0; o < a.top; ++o)
                    if (a.t_indices[r * a.top + o] == j) p = __fadd_rn(p, a.kept[r * a.top + o].x);
            }
            out[j] = RV::narrow(__fsub_rn(dense_of(px.y, ref, dense, a.c), __fmul_rn(s.coef, p)));
        }
    }
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
    cudaLaunchConfig_t kept = {};
    kept.gridDim = dim3((unsigned)a.rows);
    kept.blockDim = dim3(32 * kept_warps(a.top));
    kept.stream = st;
    kept.attrs = attr;
    if (MODE & kWantGrad) {
        kept.dynamicSmemBytes = (size_t)a.top * 12u + (size_t)a.slots * 4u;   // at most 20 KB
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&kept, kept_kernel<DT, MODE>, a));
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
    kept.dynamicSmemBytes = (MODE & kWantGrad) ? 0 : (size_t)a.top * 12u;
    kept.numAttrs = 1;
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&kept, place_kernel<DT, MODE>, a));
    return MOSAIC_OK;
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
    a.doubled = reinterpret_cast<int*>(a.kept + n * (size_t)top);
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
    return align_up((size_t)rows * (sizeof(RowScale) + 8u + 8u + 4u + (size_t)top * 8u), 256);
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
