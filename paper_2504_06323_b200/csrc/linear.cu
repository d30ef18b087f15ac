// mosaic_linear / mosaic_linear_backward: a projection's matrix product with its bias, activation and residual
// in the epilogue, and the three products of its gradient - all on the tensor cores (bf16 in, fp32 sums).
//
//     forward    Z = X W^T + b,  Y = act(Z) + R          [tokens, out]
//     backward   dZ = dY * act'(Z);  dX = dZ W  [tokens, in],  dW = dZ^T X  [out, in],  db = sum over tokens of dZ
//
// One kernel computes all of them as   out[j, i] = sum_c A[i, c] B[j, c]:  the matrix instruction's 128 rows run
// along the CONTIGUOUS dimension of the output, its columns along the rows of the output.  The accumulator of a
// fixed column is then a run of adjacent output elements across the lanes of a warp: the epilogue reads and writes
// 64 adjacent bytes per instruction whatever the alignment, the bias is one register per lane, and few tokens mean
// a narrow instruction instead of one mostly filled with nothing.
//     forward    A = W  (contraction contiguous)   B = X   (contraction contiguous)
//     dX         A = W  (contraction = rows)       B = dZ  (contraction contiguous)
//     dW         A = X  (contraction = rows)       B = dZ  (contraction = rows)
// "Contraction = rows" operands are MN-major for tcgen05.mma; nothing is transposed.
#include <cooperative_groups.h>

#include "linear.cuh"
#include "umma.cuh"

namespace cg = cooperative_groups;

namespace mosaic {
namespace {

constexpr int kMI = 128;               // rows of the matrix instruction: adjacent output elements
constexpr int kMC = 64;                // contraction steps per stage (128 bytes: one swizzle row)
constexpr int kMMaxSplit = 8;          // CTAs (one cluster) that share one tile's contraction
constexpr uint32_t kMBox = 64 * 64 * 2;   // an MN-major box: 64 elements x 64 contraction steps

struct MmArgs {
    int64_t n_i, n_j, n_c;             // extents
    int tiles_i, tiles_j, stages, split;
    int first_pair;                    // >= 0: the tiles are quarters of the pair kernel's tiles from this one on
    int pair_i, pair_j;                // its tiles
    uint16_t* out;
    int64_t ld_out;
    const uint16_t* bias;              // [n_i] or null
    const uint16_t* resid;             // [n_j, n_i] or null
    int64_t ld_resid;
    uint16_t* z;                       // [n_j, n_i] or null: the value before the activation
    int64_t ld_z;
    int act;
    int pairs;                         // out, resid and z (those there are) take two elements a word: 4-byte bases, even ld
    int* status;
};

// Two adjacent output elements a word.  A lane holds element i of rows j and j + 1 (lo, hi); after the exchange with its
// neighbour an even lane holds elements i, i + 1 of row j, an odd one i - 1, i of row j + 1.  Its own inverse.
__device__ __forceinline__ uint32_t exchange(uint32_t w, bool odd) {
    const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, w, 1);
    return odd ? __byte_perm(other, w, 0x7632) : __byte_perm(w, other, 0x5410);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return (uint32_t)__bfloat16_as_ushort(p.x) | ((uint32_t)__bfloat16_as_ushort(p.y) << 16);
}

// N accumulator columns of a warp into the output: v[e] belongs to element (i, j + e), e < n; i0 is lane 0's i.
template <int N> __device__ __forceinline__ void epilogue(const MmArgs& a, float (&v)[N], float bias, int64_t i0, int64_t j, int n) {
    const int lane = (int)threadIdx.x & 31;
    const int64_t i = i0 + lane;
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = __fadd_rn(v[e], bias);
    if (a.pairs && i0 + 32 <= a.n_i) {   // whole words: half the instructions of the element by element form below
        const bool odd = (lane & 1) != 0;
        const int64_t at = i & ~(int64_t)1, row = j + (lane & 1);
        uint32_t r[N / 2];
        if (a.resid != nullptr) {
            const uint16_t* p = a.resid + row * a.ld_resid + at;
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_resid) r[e / 2] = e + (lane & 1) < n ? *reinterpret_cast<const uint32_t*>(p) : 0u;
        }
        if (a.z != nullptr) {
            uint16_t* p = a.z + row * a.ld_z + at;
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_z) {
                const uint32_t w = exchange(pack2(v[e], v[e + 1]), odd);
                if (e + (lane & 1) < n) *reinterpret_cast<uint32_t*>(p) = w;
            }
        }
        if (a.act != MOSAIC_ACT_NONE) activate_all(v, a.act);
        if (a.resid != nullptr) {
#pragma unroll
            for (int e = 0; e < N; e += 2) {
                const uint32_t w = exchange(r[e / 2], odd);
                v[e] = __fadd_rn(v[e], __uint_as_float(w << 16));
                v[e + 1] = __fadd_rn(v[e + 1], __uint_as_float(w & 0xFFFF0000u));
            }
        }
        uint16_t* p = a.out + row * a.ld_out + at;
        if (n >= N) {
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_out) *reinterpret_cast<uint32_t*>(p) = exchange(pack2(v[e], v[e + 1]), odd);
        } else {
#pragma unroll
            for (int e = 0; e < N; e += 2, p += 2 * a.ld_out) {
                const uint32_t w = exchange(pack2(v[e], v[e + 1]), odd);
                if (e + (lane & 1) < n) *reinterpret_cast<uint32_t*>(p) = w;
            }
        }
        return;
    }
    if (i >= a.n_i) return;
    if (a.z != nullptr) {
        uint16_t* p = a.z + j * a.ld_z + i;
#pragma unroll
        for (int e = 0; e < N; ++e, p += a.ld_z)
            if (e < n) *p = f32_to_bf16(v[e]);
    }
    if (a.act != MOSAIC_ACT_NONE) activate_all(v, a.act);
    if (a.resid != nullptr) {
        const uint16_t* p = a.resid + j * a.ld_resid + i;
#pragma unroll
        for (int h = 0; h < N; h += N / 2) {   // half of them on their way before the first is used
            uint16_t r[N / 2];
#pragma unroll
            for (int e = 0; e < N / 2; ++e) {
                r[e] = 0;
                if (h + e < n) asm volatile("ld.global.u16 %0, [%1];" : "=h"(r[e]) : "l"(p));   // volatile: not one by one with the additions
                p += a.ld_resid;
            }
#pragma unroll
            for (int e = 0; e < N / 2; ++e) v[h + e] = __fadd_rn(v[h + e], bf16_to_f32(r[e]));
        }
    }
    uint16_t* p = a.out + j * a.ld_out + i;
#pragma unroll
    for (int e = 0; e < N; ++e, p += a.ld_out)
        if (e < n) *p = f32_to_bf16(v[e]);
}
template <int N> __device__ __forceinline__ void tmem_load(uint32_t addr, float (&v)[N]) {
    if constexpr (N == 16) tmem_load16(addr, v);
    else tmem_load32(addr, v);
}
__device__ __forceinline__ void pair_tile(int tile, int tiles_i, int tiles_j, int* ti, int* tj);
// Four adjacent elements, or the first n of them.
__device__ __forceinline__ void store4(uint16_t* p, const float (&y)[4], bool words, int64_t n) {
    if (words) {
        reinterpret_cast<uint32_t*>(p)[0] = pack2(y[0], y[1]);
        reinterpret_cast<uint32_t*>(p)[1] = pack2(y[2], y[3]);
    } else {
#pragma unroll
        for (int h = 0; h < 4; ++h)
            if (h < n) p[h] = f32_to_bf16(y[h]);
    }
}

// One output tile of kMI x BN per cluster; its contraction is split over the cluster's CTAs.  Each of them adds up and writes
// an equal share of the tile's columns: the others push their partial sums of it into its shared memory (the stages, free
// by then), and it adds them in the CTAs' order.  Bound by the loads of a tile's operands into one SM (about 110 GB/s an
// SM for wide tiles) or, with few tokens, by the weights' stream: 37 tokens, 4096 outputs from 8807, 18.0 us against
// 11.2 of the weights alone; 512 tokens, 4096 from 4096, 23 us.  One CTA an SM (its stages fill shared memory), so a CTA
// never waits for tensor memory that another one of this kernel holds.
constexpr int kMSub = 2;     // 64 contraction steps each a stage: eight instructions a barrier
constexpr int kMRoles = 2;   // loader, MMA issue; then the epilogue: four warps (a quarter of tensor memory's lanes each), eight for wide tiles
__host__ __device__ constexpr int mm_warps(int bn) { return bn >= 256 ? 16 : bn >= 64 ? 8 : 4; }
__host__ __device__ constexpr int mm_threads(int bn) { return 32 * (kMRoles + mm_warps(bn)); }

template <bool A_MN, bool B_MN, int BN>
__global__ void __launch_bounds__(mm_threads(BN)) mm_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map,
                                                       const __grid_constant__ MmArgs a) {
    constexpr uint32_t kABytes = kMI * kMC * 2, kBBytes = BN * kMC * 2, kHalf = kABytes + kBBytes, kStage = kMSub * kHalf;
    constexpr uint32_t kCols = BN < 32 ? 32 : BN;
    constexpr uint32_t kDesc = instr_desc(A_MN, B_MN, kMI, BN);
    extern __shared__ unsigned char mm_smem_raw[];
    __shared__ uint64_t full[8], empty[8], acc_full;
    __shared__ uint32_t tmem_slot;
    __shared__ int err_word;
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(mm_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    volatile int* err = &err_word;
    const int split = a.split, rank = (int)(blockIdx.x % (unsigned)split);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = (int)(blockIdx.x / (unsigned)split);
    int64_t i0 = (int64_t)(tile % a.tiles_i) * kMI, j0 = (int64_t)(tile / a.tiles_i) * BN;
    if (BN == 128 && a.first_pair >= 0) {   // what is left over of the pair kernel's tiles
        int ti, tj;
        pair_tile(a.first_pair + tile / 4, a.pair_i, a.pair_j, &ti, &tj);
        i0 = (int64_t)ti * 256 + (tile & 1) * 128;
        j0 = (int64_t)tj * 256 + ((tile >> 1) & 1) * 128;
    }
    const int64_t steps = (a.n_c + kMSub * kMC - 1) / (kMSub * kMC);
    const int s0 = (int)(steps * rank / split), s1 = (int)(steps * (rank + 1) / split);   // split <= steps: never empty

    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(&full[s], 1u);
            mbar_init(&empty[s], 1u);
        }
        mbar_init(&acc_full, 1u);
        *err = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    uint32_t issued = 0;
    allow_next_kernel();   // not before this CTA has its tensor memory: the next kernel's CTAs wait for it with theirs in hand
    await_previous_kernel();

    if (warp == 0) {
        if (lane == 0) {
            for (int s = s0; s < s1; ++s) {
                const uint32_t it = (uint32_t)(s - s0), slot = it % (uint32_t)a.stages, ph = (it / (uint32_t)a.stages) & 1u;
                if (!mbar_wait(&empty[slot], ph ^ 1u, err)) break;
                mbar_expect_tx(&full[slot], kStage);
#pragma unroll
                for (int h = 0; h < kMSub; ++h) {
                    unsigned char* sa = ring + (size_t)slot * kStage + (size_t)h * kHalf;
                    unsigned char* sb = sa + kABytes;
                    const int c = (s * kMSub + h) * kMC;
                    if (A_MN) {
#pragma unroll
                        for (int b = 0; b < kMI / 64; ++b) tma_load_box(sa + (size_t)b * kMBox, &a_map, &full[slot], (int)i0 + b * 64, c);
                    } else {
                        tma_load_box(sa, &a_map, &full[slot], c, (int)i0);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int b = 0; b < BN / 64; ++b) tma_load_box(sb + (size_t)b * kMBox, &b_map, &full[slot], (int)j0 + b * 64, c);
                    } else {
                        tma_load_box(sb, &b_map, &full[slot], c, (int)j0);
                    }
                }
                issued = it + 1u;
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            bool ok = true;
            for (int s = s0; s < s1; ++s) {
                const uint32_t it = (uint32_t)(s - s0), slot = it % (uint32_t)a.stages, ph = (it / (uint32_t)a.stages) & 1u;
                if (!mbar_wait(&full[slot], ph, err)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t stage = smem_u32(ring + (size_t)slot * kStage);
#pragma unroll
                for (int k = 0; k < kMSub * kMC / 16; ++k) {
                    // 16 contraction steps further: 16 swizzle rows (MN-major) or 32 bytes along one (K-major)
                    const uint32_t sa = stage + (uint32_t)(k / (kMC / 16)) * kHalf, sb = sa + kABytes, kk = (uint32_t)(k % (kMC / 16));
                    const uint64_t da = operand_desc(sa + kk * (A_MN ? 2048u : 32u), A_MN ? kMBox : 16u);
                    const uint64_t db = operand_desc(sb + kk * (B_MN ? 2048u : 32u), B_MN ? kMBox : 16u);
                    umma_bf16(tmem, da, db, kDesc, (it > 0 || k > 0) ? 1u : 0u);
                }
                umma_commit(&empty[slot]);
            }
            if (ok) umma_commit(&acc_full);
        }
    }
    __syncwarp();
    const bool done = warp >= 2 && mbar_wait(&acc_full, 0u, err);
    tc_fence_after();
    const int q = warp & 3;
    const int n_cols = (int)(a.n_j - j0 < BN ? (a.n_j > j0 ? a.n_j - j0 : 0) : BN);
    const int per = (n_cols + split - 1) / split;   // columns of the tile that a CTA of the cluster adds up and writes
    float* part = reinterpret_cast<float*>(ring);   // [split][per][kMI]: the cluster's partial sums of this CTA's columns
    if (split > 1) {
        // Every CTA's accumulator is complete, so its loads have been consumed, before its stages take partial sums.
        __syncwarp();
        cluster_arrive();
        cluster_wait();
    }
    if (done) {
        constexpr int kChunk = BN < 32 ? 16 : 32, kSets = mm_warps(BN) / 4;   // warps of a quarter take chunks in turn
        const int64_t i = i0 + q * 32 + lane;
        const float bias = a.bias != nullptr && i < a.n_i ? bf16_to_f32(a.bias[i]) : 0.0f;
#pragma unroll 1
        for (int c0 = ((warp - kMRoles) >> 2) * kChunk; c0 < n_cols; c0 += kSets * kChunk) {
            float v[kChunk];
            tmem_load<kChunk>(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)c0, v);
            if (split > 1) {
                int owner = c0 / per, at = c0 - owner * per;
                uint32_t to = cluster_addr(part + ((size_t)rank * per + at) * kMI + q * 32 + lane, owner);
#pragma unroll
                for (int e = 0; e < kChunk; ++e) {
                    if (c0 + e < n_cols) store_remote(to, v[e]);
                    to += kMI * 4;
                    if (++at == per) {
                        at = 0;
                        ++owner;
                        to = cluster_addr(part + (size_t)rank * per * kMI + q * 32 + lane, owner < split ? owner : 0);
                    }
                }
            } else {
                epilogue<kChunk>(a, v, bias, i0 + q * 32, j0 + c0, n_cols - c0);
                __syncwarp();
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
    }
    if (threadIdx.x == 0 && *err != 0) {
        // a role gave up: let the loads of the last stages land before shared memory is reused or left (bounded)
        for (uint32_t back = 1; back <= (uint32_t)a.stages && back <= issued; ++back) {
            const uint32_t it = issued - back, slot = it % (uint32_t)a.stages, ph = (it / (uint32_t)a.stages) & 1u;
            const long long t0 = clock64();
            while (!mbar_try_wait(&full[slot], ph) && clock64() - t0 < kWaitCycles) {
            }
        }
        if (a.status != nullptr) atomicExch(a.status, 1);
    }
    if (split > 1) {
        __syncwarp();
        cluster_arrive();
        // Four adjacent elements a thread and turn; the residual's are on their way while the partial sums come in.
        constexpr int kTurns = 4;
        const int mine = n_cols - rank * per < per ? n_cols - rank * per : per, quads = mine > 0 ? mine * (kMI / 4) : 0;
        uint32_t r[kTurns][2];
        const auto fetch = [&](int e0) {
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                const int e = e0 + u * mm_threads(BN);
                const int64_t oi = i0 + 4 * (e % (kMI / 4)), oj = j0 + rank * per + e / (kMI / 4);
                r[u][0] = r[u][1] = 0;
                if (a.resid == nullptr || e >= quads || oi >= a.n_i) continue;
                const uint16_t* p = a.resid + oj * a.ld_resid + oi;
                if (a.pairs && oi + 4 <= a.n_i) {
                    r[u][0] = reinterpret_cast<const uint32_t*>(p)[0];
                    r[u][1] = reinterpret_cast<const uint32_t*>(p)[1];
                } else {
                    r[u][0] = p[0] | (oi + 1 < a.n_i ? (uint32_t)p[1] << 16 : 0u);
                    r[u][1] = (oi + 2 < a.n_i ? (uint32_t)p[2] : 0u) | (oi + 3 < a.n_i ? (uint32_t)p[3] << 16 : 0u);
                }
            }
        };
        fetch((int)threadIdx.x);
        __syncwarp();
        cluster_wait();
        for (int e0 = (int)threadIdx.x; e0 < quads; e0 += kTurns * mm_threads(BN)) {
            if (e0 != (int)threadIdx.x) fetch(e0);
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                const int e = e0 + u * mm_threads(BN);
                if (e >= quads) break;
                const float4* from = reinterpret_cast<const float4*>(part) + e;
                const float4 first = *from;
                float y[4] = {first.x, first.y, first.z, first.w};
                for (int p = 1; p < split; ++p) {   // in the CTAs' order
                    const float4 more = from[p * per * (kMI / 4)];
                    y[0] = __fadd_rn(y[0], more.x);
                    y[1] = __fadd_rn(y[1], more.y);
                    y[2] = __fadd_rn(y[2], more.z);
                    y[3] = __fadd_rn(y[3], more.w);
                }
                const int64_t oi = i0 + 4 * (e % (kMI / 4)), oj = j0 + rank * per + e / (kMI / 4);
                const bool words = a.pairs && oi + 4 <= a.n_i;
                if (a.bias != nullptr) {
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        if (oi + h < a.n_i) y[h] = __fadd_rn(y[h], bf16_to_f32(a.bias[oi + h]));
                }
                if (a.z != nullptr) store4(a.z + oj * a.ld_z + oi, y, words, a.n_i - oi);
                activate_all(y, a.act);
                if (a.resid != nullptr) {
#pragma unroll
                    for (int h = 0; h < 4; ++h)
                        y[h] = __fadd_rn(y[h], __uint_as_float((h & 1) ? r[u][h / 2] & 0xFFFF0000u : r[u][h / 2] << 16));
                }
                store4(a.out + oj * a.ld_out + oi, y, words, a.n_i - oi);
            }
        }
    }
}

// ---------------------------------------------------------------- large products
// Two CTAs (a cluster, two SMs) share each matrix instruction: 256 x 256 output elements, each CTA holding its half
// of both operands in shared memory (64 KB a stage for 256 x 256 x 128 products: half of what a CTA alone would have
// to load for the same work) and 128 x 256 of the accumulator in its tensor memory, twice: the epilogue of a tile
// runs under the products of the next.  Persistent: a pair takes tile after tile.  The tiles go band by band
// (kPBand tiles of output rows), so that the tiles in flight share operands in L2.  Bound by the tensor pipe, 76 % busy at
// 14336 outputs from 4096 and 2048 tokens with bias, silu and Z (179 us, of which 147 are the flop at the measured peak).
constexpr int kPTile = 256, kPHalf = 128;
constexpr int kPSub = 2;   // 64 contraction steps each: eight instructions a barrier (with four, 1377 instead of 1505 Tflop/s at 4096 x 13824 x 5120)
constexpr int kPStages = 3;
constexpr uint32_t kPOperand = kPHalf * kMC * 2, kPStage = kPSub * 2 * kPOperand;
constexpr int kPEpiWarps = 16;   // four per quarter of the lanes
constexpr int kPThreads = 64 + 32 * kPEpiWarps;
constexpr int kPBand = 8;
constexpr size_t kPSmem = (size_t)kPStages * kPStage + 1024;

__device__ __forceinline__ void pair_tile(int tile, int tiles_i, int tiles_j, int* ti, int* tj) {
    const int band = tile / (kPBand * tiles_i), in = tile - band * kPBand * tiles_i;
    const int width = tiles_j - band * kPBand < kPBand ? tiles_j - band * kPBand : kPBand;
    *ti = in / width;
    *tj = band * kPBand + in % width;
}

template <bool A_MN, bool B_MN>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPThreads, 1)
    mm_pair_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const __grid_constant__ MmArgs a, int tiles) {
    constexpr uint32_t kDesc = instr_desc(A_MN, B_MN, kPTile, kPTile);
    extern __shared__ unsigned char pair_smem_raw[];
    __shared__ uint64_t full[kPStages], empty[kPStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int err_word;
    unsigned char* ring = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(pair_smem_raw) + 1023u) & ~(uintptr_t)1023u);
    volatile int* err = &err_word;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int pair = (int)(blockIdx.x >> 1), pairs = (int)(gridDim.x >> 1);
    const int steps = (int)((a.n_c + kPSub * kMC - 1) / (kPSub * kMC));

    if (threadIdx.x == 0) {
        prefetch_map(&a_map);
        prefetch_map(&b_map);
        for (int s = 0; s < kPStages; ++s) {
            mbar_init(&full[s], 1u);    // first CTA's: both CTAs' loads of a stage have landed
            mbar_init(&empty[s], 1u);   // the products reading a stage have completed
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&acc_full[b], 1u);
            mbar_init(&acc_empty[b], 2u * kPEpiWarps);   // first CTA's: both epilogues have read the accumulator
        }
        *err = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    cluster.sync();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    uint32_t issued = 0;
    allow_next_kernel();   // not before this CTA has its tensor memory: the next kernel's CTAs wait for it with theirs in hand
    await_previous_kernel();

    if (warp == 0) {
        if (lane == 0) {
            uint32_t it = 0;
            bool ok = true;
            for (int tile = pair; tile < tiles && ok; tile += pairs) {
                int ti, tj;
                pair_tile(tile, a.tiles_i, a.tiles_j, &ti, &tj);
                const int i0 = ti * kPTile + rank * kPHalf, j0 = tj * kPTile + rank * kPHalf;
                for (int s = 0; s < steps; ++s, ++it) {
                    const uint32_t slot = it % kPStages, ph = (it / kPStages) & 1u;
                    if (!mbar_wait(&empty[slot], ph ^ 1u, err)) {
                        ok = false;
                        break;
                    }
                    if (rank == 0) mbar_expect_tx(&full[slot], 2u * kPStage);
                    const uint32_t bar = cluster_addr(&full[slot], 0u);
#pragma unroll
                    for (int h = 0; h < kPSub; ++h) {
                        unsigned char* sa = ring + (size_t)slot * kPStage + (size_t)h * 2u * kPOperand;
                        unsigned char* sb = sa + kPOperand;
                        const int c = (s * kPSub + h) * kMC;
                        if (A_MN) {
                            tma_load_box_pair(sa, &a_map, bar, i0, c);
                            tma_load_box_pair(sa + kMBox, &a_map, bar, i0 + 64, c);
                        } else {
                            tma_load_box_pair(sa, &a_map, bar, c, i0);
                        }
                        if (B_MN) {
                            tma_load_box_pair(sb, &b_map, bar, j0, c);
                            tma_load_box_pair(sb + kMBox, &b_map, bar, j0 + 64, c);
                        } else {
                            tma_load_box_pair(sb, &b_map, bar, c, j0);
                        }
                    }
                }
            }
            issued = it;
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            uint32_t it = 0, n = 0;
            bool ok = true;
            for (int tile = pair; tile < tiles && ok; tile += pairs, ++n) {
                const uint32_t buf = n & 1u;
                if (!mbar_wait_cluster(&acc_empty[buf], ((n >> 1) & 1u) ^ 1u, err)) break;
                tc_fence_after();
                for (int s = 0; s < steps; ++s, ++it) {
                    const uint32_t slot = it % kPStages, ph = (it / kPStages) & 1u;
                    if (!mbar_wait_cluster(&full[slot], ph, err)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t stage = smem_u32(ring + (size_t)slot * kPStage);
#pragma unroll
                    for (int k = 0; k < kPSub * kMC / 16; ++k) {
                        const uint32_t sa = stage + (uint32_t)(k / (kMC / 16)) * 2u * kPOperand, sb = sa + kPOperand, kk = (uint32_t)(k % (kMC / 16));
                        const uint64_t da = operand_desc(sa + kk * (A_MN ? 2048u : 32u), A_MN ? kMBox : 16u);
                        const uint64_t db = operand_desc(sb + kk * (B_MN ? 2048u : 32u), B_MN ? kMBox : 16u);
                        umma_bf16_pair(tmem + buf * 256u, da, db, kDesc, (s > 0 || k > 0) ? 1u : 0u);
                    }
                    umma_commit_pair(&empty[slot]);
                }
                if (ok) umma_commit_pair(&acc_full[buf]);
            }
        }
    } else {
        const int q = warp & 3, set = (warp - 2) >> 2;   // quarter of the lanes, quarter of the columns
        uint32_t n = 0;
        for (int tile = pair; tile < tiles; tile += pairs, ++n) {
            int ti, tj;
            pair_tile(tile, a.tiles_i, a.tiles_j, &ti, &tj);
            const uint32_t buf = n & 1u;
            const int64_t i0 = (int64_t)ti * kPTile + rank * kPHalf + q * 32, j0 = (int64_t)tj * kPTile;
            const int n_cols = (int)(a.n_j - j0 < kPTile ? a.n_j - j0 : kPTile);
            const float bias = a.bias != nullptr && i0 + lane < a.n_i ? bf16_to_f32(a.bias[i0 + lane]) : 0.0f;
            if (!mbar_wait(&acc_full[buf], (n >> 1) & 1u, err)) break;
            tc_fence_after();
#pragma unroll 1
            for (int c0 = set * 64; c0 < set * 64 + 64 && c0 < n_cols; c0 += 32) {
                float v[32];
                tmem_load32(tmem + ((uint32_t)(q * 32) << 16) + buf * 256u + (uint32_t)c0, v);
                epilogue<32>(a, v, bias, i0, j0 + c0, n_cols - c0);
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_at(cluster_addr(&acc_empty[buf], 0u));
        }
    }
    __syncwarp();
    tc_fence_before();
    cluster.sync();   // all products and reads of both CTAs are done, or a wait ran out and every role has left
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
    if (threadIdx.x == 0) {
        const bool failed = *err != 0 || *cluster.map_shared_rank(&err_word, rank ^ 1) != 0;
        if (failed && rank == 0) {   // let both CTAs' last loads land before shared memory is left (bounded)
            for (uint32_t back = 1; back <= (uint32_t)kPStages && back <= issued; ++back) {
                const uint32_t it = issued - back, slot = it % kPStages, ph = (it / kPStages) & 1u;
                const long long t0 = clock64();
                while (!mbar_try_wait(&full[slot], ph) && clock64() - t0 < kWaitCycles) {
                }
            }
        }
        if (failed && a.status != nullptr) atomicExch(a.status, 1);
    }
    cluster.sync();   // the error words have been read, the loads have landed
}

// Eight elements of a row from c on; zeros past the last column, which nothing is read of.  Ordinary loads here and in the
// kernels below, no read-only ones (nor __restrict__, which lets the compiler make them so): they may start while the
// kernel that writes what they read still runs, and nothing orders read-only loads behind the wait for it.
template <bool VEC> __device__ __forceinline__ void load8(const uint16_t* row, int64_t c, int64_t cols, uint32_t (&w)[4]) {
    if (VEC) {   // rows on 16-byte boundaries
        if (c + 8 <= cols) {
            const uint4 v = ld_stream16(row + c);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            return;
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = c + 2 * e < cols ? row[c + 2 * e] : 0u, hi = c + 2 * e + 1 < cols ? row[c + 2 * e + 1] : 0u;
        w[e] = lo | (hi << 16);
    }
}

// ---------------------------------------------------------------- few tokens
// A decoding step's one or two tokens (up to kFewTokens where rows are not aligned): the weights are read once for next
// to no arithmetic, so what counts is that they stream.  A CTA takes kFewRows weight rows and a quarter to an eighth of the contraction per warp; a lane
// multiplies 16 bytes of each row (VEC: rows on 16-byte boundaries; else element by element, any alignment) with the
// tokens' values from L1.  fp32 sums: per lane in order, over the lanes by a butterfly, over the warps in their order.
// Bound by memory; no shared-memory ring, tensor memory or cluster to set up.
// 11008 outputs from 4096, one token: 16.3 us, 5.5 TB/s, against 19.3 us on the tensor cores; three tokens 23.7 against
// 19.2, so from there on only rows that TMA cannot read come here (46 us at four; copying them first costs more).
constexpr int kFewTokens = 4, kFewVector = 2, kFewRows = 4, kFewWarps = 8;
template <int M, bool VEC>
__global__ void __launch_bounds__(32 * kFewWarps, VEC && M == 1 ? 5 : M <= 2 ? 4 : 3) few_kernel(const uint16_t* X, int64_t ldx, const uint16_t* W, int64_t ldw,
                                                             const __grid_constant__ MmArgs a) {
    __shared__ float part[kFewWarps][kFewRows][M];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t o0 = (int64_t)blockIdx.x * kFewRows;
    float acc[kFewRows][M] = {};
    await_previous_kernel();
    const uint16_t* w[kFewRows];
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) w[r] = W + (o0 + r < a.n_i ? o0 + r : o0) * ldw;   // past the end: the first row again, not stored
    if (VEC) {
        // chunks of 256 contraction steps, dealt to the warps in turn; even and odd steps are summed apart
        Pair two[kFewRows][M];
#pragma unroll
        for (int r = 0; r < kFewRows; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) two[r][m] = pair_of(0.0f, 0.0f);
#pragma unroll 1
        for (int64_t c = warp * 256 + lane * 8; c < a.n_c; c += kFewWarps * 256) {
            uint32_t x[M][4], y[kFewRows][4];
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) load8<true>(w[r], c, a.n_c, y[r]);
#pragma unroll
            for (int m = 0; m < M; ++m) load8<true>(X + m * ldx, c, a.n_c, x[m]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                Pair xe[M];
#pragma unroll
                for (int m = 0; m < M; ++m) xe[m] = widen2(x[m][e]);
#pragma unroll
                for (int r = 0; r < kFewRows; ++r) {
                    const Pair ye = widen2(y[r][e]);
#pragma unroll
                    for (int m = 0; m < M; ++m) two[r][m] = fma2(ye, xe[m], two[r][m]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < kFewRows; ++r)
#pragma unroll
            for (int m = 0; m < M; ++m) {
                float lo, hi;
                split(two[r][m], lo, hi);
                acc[r][m] = __fadd_rn(lo, hi);
            }
    } else {
#pragma unroll 8
        for (int64_t c = warp * 32 + lane; c < a.n_c; c += kFewWarps * 32) {
            float x[M];
#pragma unroll
            for (int m = 0; m < M; ++m) x[m] = bf16_to_f32(X[m * ldx + c]);
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) {
                const float y = bf16_to_f32(w[r][c]);
#pragma unroll
                for (int m = 0; m < M; ++m) acc[r][m] = __fmaf_rn(y, x[m], acc[r][m]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kFewRows; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float v = acc[r][m];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v = __fadd_rn(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
            if (lane == 0) part[warp][r][m] = v;
        }
    __syncthreads();
    if (threadIdx.x >= kFewRows * M) return;
    const int r = threadIdx.x % kFewRows, m = threadIdx.x / kFewRows;
    const int64_t i = o0 + r;
    if (i >= a.n_i) return;
    float v = 0.0f;
    for (int k = 0; k < kFewWarps; ++k) v = __fadd_rn(v, part[k][r][m]);
    v = __fadd_rn(v, a.bias != nullptr ? bf16_to_f32(a.bias[i]) : 0.0f);
    if (a.z != nullptr) a.z[m * a.ld_z + i] = f32_to_bf16(v);
    v = activate(v, a.act);
    if (a.resid != nullptr) v = __fadd_rn(v, bf16_to_f32(a.resid[m * a.ld_resid + i]));
    a.out[m * a.ld_out + i] = f32_to_bf16(v);
}

// ---------------------------------------------------------------- elementwise passes
// dst[r, c] = src[r, c] * act'(z[r, c]) (z null: a plain copy), dst with rows on 16-byte boundaries; column sums of
// the unrounded values over the rows of this CTA's band into partial[band, c], or, of the only band, into db[c] if wanted.  A warp
// takes 256 columns, a lane eight of them (16 bytes where src and z have 16-byte rows), the CTA's eight warps every eighth
// row; the warps' sums meet in shared memory in their order.  Bound by the latency of a row's loads at the occupancy
// that the slopes' registers leave: 1001 x 8807 with silu 18 us from cold caches (gelu 21), an instruction issued in 64 %
// of the cycles, 8 us of them the bytes.  In a row of launches, with the column sums, 16 (gelu 19, no activation 13); four
// rows' loads at once (128 registers) cost 2.4 more.
constexpr int kSlopeWarps = 8, kSlopeCols = 256;
template <bool VEC>
__global__ void __launch_bounds__(32 * kSlopeWarps) slope_kernel(const uint16_t* src, int64_t ld_src, const uint16_t* z, int64_t ld_z, int act, uint16_t* dst,
                                                                 int64_t ld_dst, int64_t rows, int64_t cols, int64_t band, float* partial, uint16_t* db) {
    __shared__ float sums[kSlopeWarps][kSlopeCols];
    allow_next_kernel();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t c = (int64_t)blockIdx.x * kSlopeCols + lane * 8;
    const int64_t r0 = (int64_t)blockIdx.y * band, r1 = r0 + band < rows ? r0 + band : rows;
    await_previous_kernel();
    float sum[8] = {};
    if (c < cols) {
        for (int64_t r = r0 + warp; r < r1; r += kSlopeWarps) {
            uint32_t w[4], y[4];
            load8<VEC>(src + r * ld_src, c, cols, w);
            if (z != nullptr) load8<VEC>(z + r * ld_z, c, cols, y);
            float v[8], s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float((e & 1) ? (w[e >> 1] & 0xFFFF0000u) : (w[e >> 1] << 16));
            if (z != nullptr) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s[e] = __uint_as_float((e & 1) ? (y[e >> 1] & 0xFFFF0000u) : (y[e >> 1] << 16));
                slope_all(s, act);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = __fmul_rn(v[e], s[e]);
                // dZ is rounded to bf16 here because the tensor cores take bf16; the column sums are not
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2(v[2 * e], v[2 * e + 1]);
            }
            if (dst != nullptr) *reinterpret_cast<uint4*>(dst + r * ld_dst + c) = make_uint4(w[0], w[1], w[2], w[3]);   // rows are padded to whole vectors
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] = __fadd_rn(sum[e], v[e]);
        }
    }
    if (partial == nullptr && db == nullptr) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[warp][lane * 8 + e] = sum[e];
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * kSlopeCols + threadIdx.x;
    if (col >= cols) return;
    float total = 0.0f;
    for (int w = 0; w < kSlopeWarps; ++w) total = __fadd_rn(total, sums[w][threadIdx.x]);
    if (db != nullptr) db[col] = f32_to_bf16(total);
    else partial[(int64_t)blockIdx.y * cols + col] = total;
}
constexpr int kSumCols = 128;
__global__ void __launch_bounds__(kSumCols) column_sum_kernel(const float* partial, int64_t bands, int64_t cols, uint16_t* out) {
    allow_next_kernel();
    await_previous_kernel();
    const int64_t c = (int64_t)blockIdx.x * kSumCols + threadIdx.x;
    if (c >= cols) return;
    float sum = 0.0f;
#pragma unroll 8
    for (int64_t b = 0; b < bands; ++b) sum = __fadd_rn(sum, partial[b * cols + c]);
    out[c] = f32_to_bf16(sum);
}

// ---------------------------------------------------------------- host side
// Nanoseconds, measured with the contractions' lengths from 16 to 138 steps: 64 contraction steps of a pair's 256 x 256,
// of a CTA's 128 x 256, 128 x 128 and narrower tiles; an epilogue's column; a launch or a further wave; a shared contraction.
constexpr int64_t kPairStep = 350, kPairFixed = 6900, kWideStep = 454, kMidStep = 294, kNarrowStep = 260, kTileColumn = 5, kFixed = 3600,
                  kSplitFixed = 2000, kSplitColumn = 10, kSecondLaunch = 2000;

struct Matrix {
    const void* p;
    int64_t rows, cols, ld;
    size_t bytes() const { return rows > 0 ? ((size_t)(rows - 1) * (size_t)ld + (size_t)cols) * 2u : 0u; }
    bool tma_ok() const { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (rows <= 1 || ld % 8 == 0); }
    int64_t padded_ld() const { return (cols + 7) / 8 * 8; }
    size_t padded_bytes() const { return align_up((size_t)rows * (size_t)padded_ld() * 2u, 256); }
};

// Bands of rows: a CTA's eight warps take four rows each of the shortest; at most 64 bands.
int64_t band_rows(int64_t rows) { return rows <= 32 * 64 ? 32 : (rows + 63) / 64; }
int64_t bands_of(int64_t rows) { return (rows + band_rows(rows) - 1) / band_rows(rows); }

// A launch that may start under the one before it; `cluster` CTAs a cluster.
struct Launch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    Launch(dim3 grid, int threads, size_t smem, cudaStream_t st, int cluster = 1) {
        attr[0] = early_start();
        attr[1] = cluster_of(cluster);
        cfg.gridDim = grid;
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 2 : 1;
    }
};

int run_slope(const Matrix& src, const void* z, int64_t ld_z, int act, void* dst, int64_t ld_dst, float* partial, void* db, cudaStream_t st) {
    const int64_t bands = bands_of(src.rows);
    if (bands > 0) {
        Launch l(dim3((unsigned)((src.cols + kSlopeCols - 1) / kSlopeCols), (unsigned)bands), 32 * kSlopeWarps, 0, st);
        const Matrix zm{z, src.rows, src.cols, ld_z};
        const bool vec = src.tma_ok() && (z == nullptr || zm.tma_ok());
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, vec ? slope_kernel<true> : slope_kernel<false>, static_cast<const uint16_t*>(src.p), src.ld,
                                           static_cast<const uint16_t*>(z), ld_z, act, static_cast<uint16_t*>(dst), ld_dst, src.rows, src.cols,
                                           band_rows(src.rows), partial, bands == 1 ? static_cast<uint16_t*>(db) : nullptr));
    }
    if (db != nullptr && bands != 1) {   // of one band the sums are final
        Launch l(dim3((unsigned)((src.cols + kSumCols - 1) / kSumCols)), kSumCols, 0, st);
        MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, column_sum_kernel, static_cast<const float*>(partial), bands, src.cols, static_cast<uint16_t*>(db)));
    }
    return MOSAIC_OK;
}

// A matrix TMA can read: itself, or a copy at *ws (advanced) with rows on 16-byte boundaries.
int readable(Matrix& m, char** ws, cudaStream_t st) {
    if (m.rows == 0 || m.tma_ok()) return MOSAIC_OK;
    const int rc = run_slope(m, nullptr, 0, MOSAIC_ACT_NONE, *ws, m.padded_ld(), nullptr, nullptr, st);
    if (rc != MOSAIC_OK) return rc;
    m.p = *ws;
    m.ld = m.padded_ld();
    *ws += m.padded_bytes();
    return MOSAIC_OK;
}

template <bool A_MN, bool B_MN> int encode_operands(CUtensorMap* a_map, CUtensorMap* b_map, const Matrix& A, const Matrix& B, int rows_a, int rows_b) {
    const bool a_ok = A_MN ? encode_bf16(a_map, A.p, A.rows, A.cols, A.ld, kMC, 64) : encode_bf16(a_map, A.p, A.rows, A.cols, A.ld, rows_a, kMC);
    const bool b_ok = B_MN ? encode_bf16(b_map, B.p, B.rows, B.cols, B.ld, kMC, 64) : encode_bf16(b_map, B.p, B.rows, B.cols, B.ld, rows_b, kMC);
    return a_ok && b_ok ? MOSAIC_OK : MOSAIC_ERR_CUDA;
}

template <int BN> constexpr size_t kMRing = 196 * 1024 / ((size_t)(kMI + BN) * kMC * 2 * kMSub) * ((size_t)(kMI + BN) * kMC * 2 * kMSub);   // one CTA an SM
template <bool A_MN, bool B_MN, int BN> bool opt_in() {
    static DeviceCache opted;
    return opted.get([]() -> int {
        if (cudaFuncSetAttribute(mm_kernel<A_MN, B_MN, BN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMRing<BN> + 1024) == cudaSuccess) return 1;
        (void)cudaGetLastError();
        return -1;
    }) > 0;
}

// Clusters of `split` one-an-SM CTAs that run at a time: fewer than the SMs divided by split, as a cluster's SMs are of
// one processing cluster (148 SMs hold 33 clusters of four and 15 of eight).
int64_t resident_clusters(int split) {
    if (split == 1) return sm_count();
    static DeviceCache held[kMMaxSplit + 1];
    return held[split].get([&]() -> int {
        if (opt_in<false, false, 64>()) {
            Launch l(dim3((unsigned)split), mm_threads(64), kMRing<64> + 1024, nullptr, split);
            int n = 0;
            if (cudaOccupancyMaxActiveClusters(&n, mm_kernel<false, false, 64>, &l.cfg) == cudaSuccess && n > 0) return n;
            (void)cudaGetLastError();
        }
        const int n = sm_count() / split;
        return n > 0 ? n : 1;
    });
}

// What mm_kernel's tiles would take, and the CTAs that share one's contraction (each keeps two stages or more).
struct MmPlan {
    int64_t nanoseconds;
    int split;
};
MmPlan plan_mm(int64_t tiles, int64_t steps, int64_t bn) {
    MmPlan best = {0, 1};
    const int64_t step = bn == 256 ? kWideStep : bn == 128 ? kMidStep : kNarrowStep;
    for (int split = 1; split <= kMMaxSplit && (split == 1 || steps >= 4 * split); ++split) {
        const int64_t held = resident_clusters(split), waves = (tiles + held - 1) / held;
        const int64_t c = waves * ((steps + split - 1) / split * step + bn * kTileColumn + kFixed + (split > 1 ? kSplitFixed + bn * kSplitColumn : 0));
        if (split == 1 || c < best.nanoseconds) best = {c, split};
    }
    return best;
}

template <bool A_MN, bool B_MN, int BN>
int launch_mm(const Matrix& A, const Matrix& B, MmArgs a, int64_t tiles, int split, cudaStream_t st) {
    static_assert(kMRing<BN> >= (size_t)(BN + kMMaxSplit) * kMI * 4, "the partial sums lie where the stages were");
    CUtensorMap a_map, b_map;
    if (encode_operands<A_MN, B_MN>(&a_map, &b_map, A, B, kMI, BN) != MOSAIC_OK || !opt_in<A_MN, B_MN, BN>()) return MOSAIC_ERR_CUDA;
    a.tiles_i = (int)((a.n_i + kMI - 1) / kMI);
    a.split = split;
    a.stages = (int)(kMRing<BN> / ((size_t)(kMI + BN) * kMC * 2 * kMSub));
    if (tiles * split > 0x7FFFFFFF) return MOSAIC_ERR_INVALID_ARG;
    Launch l(dim3((unsigned)(tiles * split)), mm_threads(BN), kMRing<BN> + 1024, st, split);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, mm_kernel<A_MN, B_MN, BN>, a_map, b_map, a));
    return MOSAIC_OK;
}

template <bool A_MN, bool B_MN> int launch_pair(const Matrix& A, const Matrix& B, MmArgs a, int64_t tiles, cudaStream_t st) {
    CUtensorMap a_map, b_map;
    if (encode_operands<A_MN, B_MN>(&a_map, &b_map, A, B, kPHalf, kPHalf) != MOSAIC_OK) return MOSAIC_ERR_CUDA;
    a.tiles_i = a.pair_i;
    a.tiles_j = a.pair_j;
    static DeviceCache opted;
    const int ok = opted.get([&]() -> int {
        if (cudaFuncSetAttribute(mm_pair_kernel<A_MN, B_MN>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return -1;
        }
        return 1;
    });
    if (ok < 0) return MOSAIC_ERR_CUDA;
    const int64_t pairs = sm_count() / 2;
    Launch l(dim3((unsigned)(2 * (tiles < pairs ? tiles : pairs))), kPThreads, kPSmem, st);   // the cluster is the kernel's own
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, mm_pair_kernel<A_MN, B_MN>, a_map, b_map, a, (int)tiles));
    return MOSAIC_OK;
}

// out[j, i] = sum_c A B; A: [n_i, n_c] (or [n_c, n_i] if A_MN), B likewise.
template <bool A_MN, bool B_MN> int run_mm(const Matrix& A, const Matrix& B, MmArgs a, cudaStream_t st) {
    const int64_t steps = (a.n_c + kMC - 1) / kMC, sms = sm_count();
    const auto even = [](const void* p, int64_t ld) { return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & 3u) == 0 && ld % 2 == 0); };
    a.pairs = even(a.out, a.ld_out) && even(a.resid, a.ld_resid) && even(a.z, a.ld_z) ? 1 : 0;
    const int64_t pi = (a.n_i + kPTile - 1) / kPTile, pj = (a.n_j + kPTile - 1) / kPTile, large = pi * pj, pairs = sms / 2;
    if (large > 0x0FFFFFFF) return MOSAIC_ERR_INVALID_ARG;
    a.pair_i = (int)pi;
    a.pair_j = (int)pj;
    a.first_pair = -1;
    // Which kernel and tile: what each would take.
    const int64_t ti = (a.n_i + kMI - 1) / kMI;
    MmPlan plan = {0, 1};
    int64_t bn = 0;
    for (int64_t w = B_MN ? 64 : 16; w <= 256; w *= 2) {
        const MmPlan p = plan_mm(ti * ((a.n_j + w - 1) / w), steps, w);
        if (bn == 0 || p.nanoseconds < plan.nanoseconds) {
            plan = p;
            bn = w;
        }
        if (w >= a.n_j) break;
    }
    // The pair kernel, and its last wave, if of few tiles, in quarters whose contraction is shared (14336 x 2048 outputs
    // from 4096, 448 tiles for 74 pairs: 178 instead of 184 us).
    const int64_t waves = large / pairs, rest = large % pairs, wave = steps * kPairStep;
    const MmPlan quarters = plan_mm(rest * 4, steps, 128);
    const bool cut = waves > 0 && rest > 0 && quarters.nanoseconds + kSecondLaunch < wave;
    if (waves * wave + (cut ? quarters.nanoseconds + kSecondLaunch : rest > 0 ? wave : 0) + kPairFixed < plan.nanoseconds) {
        const int rc = launch_pair<A_MN, B_MN>(A, B, a, cut ? waves * pairs : large, st);
        if (rc != MOSAIC_OK || !cut) return rc;
        a.first_pair = (int)(waves * pairs);
        return launch_mm<A_MN, B_MN, 128>(A, B, a, rest * 4, quarters.split, st);
    }
    const int64_t tiles = ti * ((a.n_j + bn - 1) / bn);
    if constexpr (!B_MN) {
        if (bn == 16) return launch_mm<A_MN, B_MN, 16>(A, B, a, tiles, plan.split, st);
        if (bn == 32) return launch_mm<A_MN, B_MN, 32>(A, B, a, tiles, plan.split, st);
    }
    if (bn == 64) return launch_mm<A_MN, B_MN, 64>(A, B, a, tiles, plan.split, st);
    return bn == 128 ? launch_mm<A_MN, B_MN, 128>(A, B, a, tiles, plan.split, st) : launch_mm<A_MN, B_MN, 256>(A, B, a, tiles, plan.split, st);
}

int launch_few(const Matrix& x, const Matrix& w, const MmArgs& a, cudaStream_t st) {
    using Kernel = void (*)(const uint16_t*, int64_t, const uint16_t*, int64_t, MmArgs);
    static const Kernel plain[kFewTokens] = {few_kernel<1, false>, few_kernel<2, false>, few_kernel<3, false>, few_kernel<4, false>};
    static const Kernel vector[kFewVector] = {few_kernel<1, true>, few_kernel<2, true>};
    const Kernel kernel = x.tma_ok() && w.tma_ok() ? vector[a.n_j - 1] : plain[a.n_j - 1];
    const int64_t ctas = (a.n_i + kFewRows - 1) / kFewRows;
    Launch l(dim3((unsigned)ctas), 32 * kFewWarps, 0, st);
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&l.cfg, kernel, static_cast<const uint16_t*>(x.p), x.ld,
                                       static_cast<const uint16_t*>(w.p), w.ld, a));
    return MOSAIC_OK;
}

bool overlap(const Matrix& a, const Matrix& b) {
    const char *x = static_cast<const char*>(a.p), *y = static_cast<const char*>(b.p);
    return x != nullptr && y != nullptr && a.bytes() > 0 && b.bytes() > 0 && x < y + b.bytes() && y < x + a.bytes();
}

// null / element alignment / leading dimension of a matrix that is there (rows > 0)
int check_bf16(const Matrix& m) {
    if (m.ld < m.cols) return MOSAIC_ERR_INVALID_ARG;
    if (m.rows > 0 && m.p == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(m.p) & 1u) != 0) return MOSAIC_ERR_MISALIGNED;
    return MOSAIC_OK;
}
constexpr int64_t kMostExtent = 0x7FFFFFFF - 1024;
bool extents_ok(int64_t m, int64_t n, int64_t k) { return m >= 0 && n > 0 && k > 0 && m <= kMostExtent && n <= kMostExtent && k <= kMostExtent; }
bool act_ok(int act) { return act >= MOSAIC_ACT_NONE && act <= MOSAIC_ACT_SILU; }

int check_workspace(const void* ws, size_t ws_bytes, size_t need) {
    if (need == 0) return MOSAIC_OK;
    if (ws == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return MOSAIC_ERR_MISALIGNED;
    return ws_bytes < need ? MOSAIC_ERR_WORKSPACE_TOO_SMALL : MOSAIC_OK;
}

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
    if (tokens <= (x.tma_ok() && w.tma_ok() ? kFewVector : kFewTokens)) return launch_few(x, w, a, st);
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
