// mosaic_top_logits: the k largest logits of every row, in order (value descending, index ascending), and
// the log-sum-exp of the whole row - what is kept of a teacher's answer for distillation.
//
// One pass over the row (rows.cuh).  Every thread knows the largest of its entries (64 of 32000); the
// k-th largest of those maxima is a value that at least k entries reach, and on rows in no particular order
// only a few more than k do.  It is found by bisection over the maxima's order-preserving bit patterns, one
// vote of the block a step.  The entries that reach it are collected and ranked exactly, under (value,
// index).  A row where more than the list holds reach it (masked rows, many ties, k near the number of
// threads) is selected digit by digit over all its entries instead.  Bound by memory.
#include <math.h>

#include "rows.cuh"

namespace cg = cooperative_groups;

namespace mosaic {
namespace {

constexpr int kListCap = 2048;   // entries collected per row
constexpr int kSlack = 8;        // candidates too many that are not worth another vote
constexpr int kRankMost = 256;   // up to here a list is ranked by counting, above it by a bitonic sort

struct TopArgs {
    const void* L;
    int64_t rows, vocab, ldl;
    int top;
    float* values;
    int32_t* indices;
    float* lse;
    double inv_t;
    float c;
};

// Order-preserving pattern: larger value <=> larger key; -0 and +0 are equal, every NaN is above +inf.
__device__ __forceinline__ uint32_t order_key(float x) {
    if (x != x) return 0xFFFFFFFFu;
    const uint32_t b = __float_as_uint(__fadd_rn(x, 0.0f));
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k); }
// One number that orders (value descending, index ascending) descending; distinct for distinct entries.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int col) { return ((uint64_t)key << 32) | (uint32_t)~(uint32_t)col; }

struct TopShared {
    uint64_t list[kListCap];
    SoftStat warp_stat[kWarps];
    SoftStat cta_stat[kMaxCluster];
    uint32_t cta_floor[kMaxCluster];
    uint32_t hist[256];
    uint32_t warp_count[kWarps];
    uint16_t owner[kThreads];
    uint32_t kept;
    uint32_t count;
    uint32_t digit, rest;
};

// The exact selection over a whole row by one CTA, digit by digit: leaves the k entries in list[0, k).
template <int DT> __device__ void select_all(const RowPart<DT>& row, int top, TopShared& sh) {
    const int cols = row.cols, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t prefix = 0u, mask = 0u, want = (uint32_t)top;   // the want-th largest among the keys that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += kThreads) sh.hist[i] = 0u;
        __syncthreads();
        for (int j0 = 0; j0 < cols; j0 += kThreads) {
            const int j = j0 + (int)threadIdx.x;
            const uint32_t key = j < cols ? order_key(row.at(j)) : 0u;
            const bool in = j < cols && (key & mask) == prefix;
            const uint32_t d = (key >> shift) & 255u;
            // a warp whose entries all fall into one bin adds them at once (masked rows)
            const uint32_t members = __ballot_sync(0xFFFFFFFFu, in);
            if (members != 0u) {
                const uint32_t d0 = __shfl_sync(0xFFFFFFFFu, d, __ffs(members) - 1);
                if (__all_sync(0xFFFFFFFFu, !in || d == d0)) {
                    if (lane == 0) atomicAdd(&sh.hist[d0], (uint32_t)__popc(members));
                } else if (in) {
                    atomicAdd(&sh.hist[d], 1u);
                }
            }
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint32_t left = want;
            int d = 255;
            while (d > 0 && sh.hist[d] < left) left -= sh.hist[d--];
            sh.digit = (uint32_t)d;
            sh.rest = left;
        }
        __syncthreads();
        prefix |= sh.digit << shift;
        mask |= 255u << shift;
        want = sh.rest;
        __syncthreads();
    }
    // `prefix` is the k-th largest key; `want` of the entries equal to it are kept, the first by index
    if (threadIdx.x == 0) sh.count = 0u;
    __syncthreads();
    uint32_t equal_before = 0u;
    for (int j0 = 0; j0 < cols; j0 += kThreads) {
        const int j = j0 + (int)threadIdx.x;
        const uint32_t key = j < cols ? order_key(row.at(j)) : 0u;
        const bool equal = j < cols && key == prefix;
        const uint32_t votes = __ballot_sync(0xFFFFFFFFu, equal);
        if (lane == 0) sh.warp_count[warp] = (uint32_t)__popc(votes);
        __syncthreads();
        uint32_t before = equal_before + (uint32_t)__popc(votes & ((1u << lane) - 1u));
        uint32_t total = 0u;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) before += sh.warp_count[w];
            total += sh.warp_count[w];
        }
        if ((j < cols && key > prefix) || (equal && before < want)) sh.list[atomicAdd(&sh.count, 1u)] = entry_of(key, j);
        equal_before += total;
        __syncthreads();
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads, kRowCtas) top_logits_kernel(const __grid_constant__ TopArgs a) {
    using RV = RowVec<DT>;
    __shared__ TopShared sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int n_ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t r = blockIdx.x >> (__ffs(n_ctas) - 1);   // a power of two
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int vocab = (int)a.vocab;
    const RowPart<DT> part(a.L, r, a.ldl, vocab, rank, n_ctas);
    const int lone = part.single();
    const float lone_x = lone >= 0 ? part.at(lone) : -INFINITY;
    if (threadIdx.x == 0) {
        sh.count = 0u;
        sh.kept = 0u;
    }
    if (n_ctas > 1) cluster_arrive();   // waited for before the first write to another CTA

    SoftStat st = {-INFINITY, 0.0f};
    for (int v = part.v_lo + (int)threadIdx.x; v < part.v_hi; v += kBatch * kThreads) {
        uint4 raw[kBatch];
        part.load(v, raw);
        soft_batch<DT>(raw, a.c, st);
    }
    if (lone >= 0) st = soft_merge(st, soft_one(lone_x, a.c), a.c);
    // the thread's largest entry, as a 16-bit pattern rounded down (a NaN makes the sum NaN: above all)
    const bool any = part.v_lo + (int)threadIdx.x < part.v_hi || lone >= 0;
    const uint32_t mine = any ? (st.s != st.s ? 0xFFFFu : order_key(st.m) >> 16) : 0u;

    // a pattern that at least `top` of the threads' maxima reach, the largest or one that few more do (0: all entries
    // are candidates)
    uint32_t floor_key = 0u;
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t trial = floor_key | (1u << bit);
        const int n = __syncthreads_count(mine >= trial);
        if (n >= a.top) {
            floor_key = trial;
            if (n <= a.top + kSlack) break;
        }
    }
    st = soft_warp(st, a.c);
    if (lane == 0) sh.warp_stat[warp] = st;
    if (n_ctas > 1) cluster_wait();
    __syncthreads();
    st = soft_all(sh.warp_stat, kWarps, a.c);
    if (n_ctas > 1) {   // a part's floor holds for the row: the highest of them serves all
        if (threadIdx.x < n_ctas) {
            *cluster.map_shared_rank(&sh.cta_stat[rank], threadIdx.x) = st;
            *cluster.map_shared_rank(&sh.cta_floor[rank], threadIdx.x) = floor_key;
        }
        cluster.sync();
        st = soft_all(sh.cta_stat, n_ctas, a.c);
        for (int i = 0; i < n_ctas; ++i) floor_key = sh.cta_floor[i] > floor_key ? sh.cta_floor[i] : floor_key;
    }
    if (rank == 0 && threadIdx.x == 0 && a.lse != nullptr) a.lse[r] = (float)soft_lse(st, a.inv_t);

    // ---- candidates into the first CTA's list
    {
        uint32_t* count = cluster.map_shared_rank(&sh.count, 0);
        uint64_t* list = cluster.map_shared_rank(sh.list, 0);
        const float least = floor_key == 0u ? -INFINITY : key_value(floor_key << 16);
        auto take = [&](float x, int j) {
            const uint32_t at = atomicAdd(count, 1u);
            if (at < kListCap) list[at] = entry_of(order_key(x), j);
        };
        if (lone >= 0 && !(lone_x < least)) take(lone_x, lone);
        // Few threads (about `top` of them) hold a candidate.  The whole block goes through their vectors, a vector or
        // two per thread, from L2.
        if (mine >= floor_key && part.v_lo + (int)threadIdx.x < part.v_hi) sh.owner[atomicAdd(&sh.kept, 1u)] = (uint16_t)threadIdx.x;
        __syncthreads();
        const int kept = (int)sh.kept;
        const int rounds = (part.v_hi - part.v_lo + kThreads - 1) / kThreads;
        for (int u = (int)threadIdx.x; u < kept * rounds; u += kThreads) {
            const int v = part.v_lo + sh.owner[u % kept] + (u / kept) * kThreads;
            if (v >= part.v_hi) continue;
            const uint4 w = ld_stream16(part.vec(v));
            uint32_t mask = reach_mask<DT>(w, least);
            while (mask != 0u) {
                const int e = __ffs(mask) - 1;
                mask &= mask - 1u;
                take(RV::any(w, e), part.first(v) + e);
            }
        }
    }
    if (n_ctas > 1) cluster.sync();
    else __syncthreads();
    if (rank != 0) return;
    uint32_t n = sh.count;
    __syncthreads();
    if (n > kListCap) {
        select_all<DT>(part, a.top, sh);
        n = (uint32_t)a.top;
        __syncthreads();
    }

    // ---- exact order of the list
    float* values = a.values + r * a.top;
    int32_t* indices = a.indices + r * a.top;
    auto emit = [&](uint32_t place, uint64_t entry) {
        const int j = (int)~(uint32_t)entry;
        const uint32_t key = (uint32_t)(entry >> 32);
        // the logit's own bits: the key has lost the sign of zero and a NaN's payload
        values[place] = key == 0x80000000u || key == 0xFFFFFFFFu ? part.at(j) : key_value(key);
        indices[place] = j;
    };
    if (n <= kRankMost) {
        // a group of `share` threads counts the larger entries of one candidate
        uint32_t share = 2u;
        while (share < 32u && n * share * 2u <= kThreads) share *= 2u;
        for (uint32_t i0 = 0; i0 < n; i0 += kThreads / share) {
            const uint32_t i = i0 + threadIdx.x / share;
            const uint64_t me = i < n ? sh.list[i] : 0ull;
            uint32_t above = 0u;
            for (uint32_t o = threadIdx.x % share; o < n; o += share) above += sh.list[o] > me ? 1u : 0u;
            for (uint32_t o = share / 2u; o > 0u; o >>= 1) above += __shfl_xor_sync(0xFFFFFFFFu, above, o);
            if (i < n && threadIdx.x % share == 0u && above < (uint32_t)a.top) emit(above, me);
        }
        return;
    }
    uint32_t size = kRankMost * 2;
    while (size < n) size *= 2u;
    for (uint32_t i = n + threadIdx.x; i < size; i += kThreads) sh.list[i] = 0ull;   // below every entry (a column's complement is not 0)
    __syncthreads();
    for (uint32_t k = 2u; k <= size; k <<= 1) {
        for (uint32_t d = k >> 1; d > 0u; d >>= 1) {
            for (uint32_t p = threadIdx.x; p < size / 2u; p += kThreads) {
                const uint32_t lo = 2u * d * (p / d) + (p % d), hi = lo + d;
                const uint64_t x = sh.list[lo], y = sh.list[hi];
                if ((x < y) == ((lo & k) == 0u)) {
                    sh.list[lo] = y;
                    sh.list[hi] = x;
                }
            }
            __syncthreads();
        }
    }
    for (uint32_t i = threadIdx.x; i < (uint32_t)a.top; i += kThreads) emit(i, sh.list[i]);
}

template <int DT> int launch_top(TopArgs a, cudaStream_t st) {
    const int c = row_cluster(a.rows, row_vectors(a.vocab, DT));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(a.rows * c));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)c;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, top_logits_kernel<DT>, a));
    return MOSAIC_OK;
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" int mosaic_top_logits(const void* L, int64_t rows, int64_t vocab, int64_t ldl, int dtype, int64_t top, float temperature,
                                 float* values, int32_t* indices, float* lse, void* stream) {
    if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (rows < 0 || rows > 0x7FFFFFFF / kMaxCluster || vocab <= 0 || vocab > kMaxRow || ldl < vocab || top < 1 || top > kMaxTop || top > vocab)
        return MOSAIC_ERR_INVALID_ARG;
    if (!(temperature >= 1.17549435e-38f) || !(temperature <= 3.402823466e38f)) return MOSAIC_ERR_INVALID_ARG;
    if (rows == 0) return MOSAIC_OK;
    if (L == nullptr || values == nullptr || indices == nullptr) return MOSAIC_ERR_NULL_PTR;
    const size_t es = elem_size(dtype);
    if ((reinterpret_cast<uintptr_t>(L) & (es - 1u)) != 0 ||
        ((reinterpret_cast<uintptr_t>(values) | reinterpret_cast<uintptr_t>(indices) | reinterpret_cast<uintptr_t>(lse)) & 3u) != 0)
        return MOSAIC_ERR_MISALIGNED;
    {   // outputs must overlap neither the logits nor one another
        const size_t n = (size_t)rows;
        const char* p[4] = {static_cast<const char*>(L), reinterpret_cast<const char*>(values), reinterpret_cast<const char*>(indices),
                            reinterpret_cast<const char*>(lse)};
        const size_t len[4] = {((n - 1u) * (size_t)ldl + (size_t)vocab) * es, n * (size_t)top * 4u, n * (size_t)top * 4u, lse != nullptr ? n * 4u : 0u};
        for (int i = 0; i < 4; ++i)
            for (int o = i + 1; o < 4; ++o)
                if (len[i] > 0 && len[o] > 0 && p[i] < p[o] + len[o] && p[o] < p[i] + len[i]) return MOSAIC_ERR_ALIASING;
    }
    TopArgs a = {};
    a.L = L; a.rows = rows; a.vocab = vocab; a.ldl = ldl; a.top = (int)top;
    a.values = values; a.indices = indices; a.lse = lse;
    a.inv_t = 1.0 / (double)temperature;
    a.c = (float)(1.4426950408889634 / (double)temperature);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == MOSAIC_BF16 ? launch_top<MOSAIC_BF16>(a, st) : launch_top<MOSAIC_F32>(a, st);
}
