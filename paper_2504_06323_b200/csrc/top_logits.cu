// mosaic_top_logits: the k largest logits of every row, in order (value descending, index ascending), and
// the log-sum-exp of the whole row - what is kept of a teacher's answer for distillation.
//
// Two launches, the second of which starts under the first:
//   sweep_kernel    streams the rows once: softmax statistics, and the largest entry of every group of entries that
//                   lie together (128 bytes, or 16 where k is near the number of such groups), as a 16-bit pattern
//   pick_kernel     a small CTA a row.  The k-th largest of the group maxima is a value that at least k entries reach,
//                   and on rows in no particular order only a few more than k do.  It is found by bisection over the
//                   patterns; only the groups that reach it (k of them and a few) are read again; their entries that
//                   reach it are ranked exactly, under (value, index).  A row where more than the list holds reach it
//                   (masked rows, many ties) or that has a NaN is selected digit by digit over all its entries.
// The first is bound by memory.  The second is a chain of short dependent steps: small CTAs, so that many rows'
// chains overlap; inside the sweep, three CTAs an SM, the same steps took as long again as the sweep itself (98 us for
// 4096 x 32000 bf16 instead of 77, of which the sweep is 50 at DRAM 64 % busy and an instruction in 73 % of the cycles).
#include <math.h>

#include "rows.cuh"

namespace mosaic {
namespace {

// Entries a list is ranked by counting up to, then by sorted runs of 32, above by a bitonic sort of the whole.  Counting
// costs the list's square (342 entries, 512 threads: 12000 cycles, and 13000 sorted whole), a run's sort fifteen exchanges.
__host__ __device__ constexpr uint32_t count_most(int n) { return n == 32 ? 256u : 128u; }
constexpr uint32_t kRunsMost = 1024u;

struct TopArgs {
    const void* L;
    int64_t rows, vocab, ldl;
    int top;
    float* values;
    int32_t* indices;
    float* lse;
    double inv_t;
    float c;
    int part_vecs, parts;    // vectors of a row that a CTA sweeps, CTAs a row
    int group_shift;         // a group is 2^group_shift vectors: 8, or 1
    int groups;              // patterns a row has room for, a multiple of 8
    int list_cap;            // candidates that fit
    // workspace
    float2* stat;            // [rows, parts]
    uint16_t* patterns;      // [rows, groups]
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

// ---------------------------------------------------------------- sweep
// The largest entry of each of a batch's vectors; with `wide`, of each run of eight lanes' vectors (in every lane).
// Returns the largest of the thread's own batch.
template <int DT> __device__ __forceinline__ float group_max(const uint4 (&raw)[kBatch], bool wide, float (&m)[kBatch]) {
    float own;
    using RV = RowVec<DT>;
    static_assert(kBatch == 4, "two vectors' bf16 maxima share a register");
    if constexpr (DT == MOSAIC_BF16) {
        uint32_t w[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            uint32_t a = raw[i].x, b = raw[i].z, h;
            asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(raw[i].y));
            asm("max.bf16x2 %0, %0, %1;" : "+r"(b) : "r"(raw[i].w));
            asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(b));
            h = __funnelshift_l(a, a, 16);
            asm("max.bf16x2 %0, %0, %1;" : "+r"(a) : "r"(h));
            w[i] = a;   // both halves
        }
        uint32_t p = __byte_perm(w[0], w[1], 0x5410), q = __byte_perm(w[2], w[3], 0x5410), o2 = p;
        asm("max.bf16x2 %0, %0, %1;" : "+r"(o2) : "r"(q));
        own = fmaxf(__uint_as_float(o2 << 16), __uint_as_float(o2 & 0xFFFF0000u));
        if (wide) {
#pragma unroll
            for (int o = 1; o < 8; o <<= 1) {
                const uint32_t pp = __shfl_xor_sync(0xFFFFFFFFu, p, o), qq = __shfl_xor_sync(0xFFFFFFFFu, q, o);
                asm("max.bf16x2 %0, %0, %1;" : "+r"(p) : "r"(pp));
                asm("max.bf16x2 %0, %0, %1;" : "+r"(q) : "r"(qq));
            }
        }
        m[0] = __uint_as_float(p << 16);
        m[1] = __uint_as_float(p & 0xFFFF0000u);
        m[2] = __uint_as_float(q << 16);
        m[3] = __uint_as_float(q & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            m[i] = fmaxf(fmaxf(RV::get(raw[i], 0), RV::get(raw[i], 1)), fmaxf(RV::get(raw[i], 2), RV::get(raw[i], 3)));
            own = i == 0 ? m[0] : fmaxf(own, m[i]);
            if (wide) {
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) m[i] = fmaxf(m[i], __shfl_xor_sync(0xFFFFFFFFu, m[i], o));
            }
        }
    }
    return own;
}

// Small CTAs, many an SM: while one waits for its loads the others compute (4096 x 32000 bf16 with the pick: 256 threads
// and six CTAs 77 us, 512 and three 82, 512 and two 90, 256 and eight - 32 registers - 84).
constexpr int kSweepThreads = 256, kSweepCtas = 6;
template <int DT> __global__ void __launch_bounds__(kSweepThreads, kSweepCtas) sweep_kernel(const __grid_constant__ TopArgs a) {
    __shared__ SoftStat warp_stat[kSweepThreads / 32];
    allow_next_kernel();
    const int64_t r = blockIdx.x;
    const int p = (int)blockIdx.y;
    RowPart<DT> part(a.L, r, a.ldl, (int)a.vocab, p, a.parts);
    const int nv = (part.cols - part.head) / RowVec<DT>::kElems;
    part.v_lo = p * a.part_vecs;   // parts begin on a group's boundary
    part.v_hi = part.v_lo + a.part_vecs < nv ? part.v_lo + a.part_vecs : nv;
    const int lane = threadIdx.x & 31;
    const bool wide = a.group_shift != 0;
    uint16_t* patterns = a.patterns + r * a.groups;
    SoftStat st = {-INFINITY, 0.0f};
    // whole warps stay together (their lanes share groups): up to the last vector of the part, rounded to the block
    for (int v = part.v_lo + (int)threadIdx.x; v - (int)threadIdx.x < part.v_hi; v += kBatch * kSweepThreads) {
        uint4 raw[kBatch];
        part.template load<kSweepThreads>(v, raw);
        float m[kBatch];
        const float own = group_max<DT>(raw, wide, m);
        soft_batch<DT>(raw, own, a.c, st);
        if (wide) {   // lane i of a run writes the pattern of the run's vectors of batch i
            const int i = lane & 3, u = v - (lane & 7) + i * kSweepThreads;
            const float mi = (i & 2) ? ((i & 1) ? m[3] : m[2]) : ((i & 1) ? m[1] : m[0]);
            if ((lane & 7) < kBatch && u < part.v_hi) patterns[u >> 3] = (uint16_t)(order_key(mi) >> 16);
        } else {
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (v + i * kSweepThreads < part.v_hi) patterns[v + i * kSweepThreads] = (uint16_t)(order_key(m[i]) >> 16);
        }
    }
    const int lone = part.single();
    if (lone >= 0) st = soft_merge(st, soft_one(part.at(lone), a.c), a.c);
    st = soft_warp(st, a.c);
    if (lane == 0) warp_stat[threadIdx.x >> 5] = st;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    st = soft_all(warp_stat, kSweepThreads / 32, a.c);
    if (threadIdx.x == 0) a.stat[r * a.parts + p] = make_float2(st.m, st.s);
}

// ---------------------------------------------------------------- pick
struct PickShared {
    uint32_t hist[256];
    uint32_t warp_count[16];
    uint32_t count;
    uint32_t digit, rest;
};

// The exact selection over a whole row by one CTA, digit by digit: leaves the k entries in list[0, k).
template <int DT, int T> __device__ void select_all(const RowPart<DT>& row, int top, uint64_t* list, PickShared& sh) {
    const int cols = row.cols, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t prefix = 0u, mask = 0u, want = (uint32_t)top;   // the want-th largest among the keys that share the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = threadIdx.x; i < 256; i += T) sh.hist[i] = 0u;
        __syncthreads();
        for (int j0 = 0; j0 < cols; j0 += T) {
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
    for (int j0 = 0; j0 < cols; j0 += T) {
        const int j = j0 + (int)threadIdx.x;
        const uint32_t key = j < cols ? order_key(row.at(j)) : 0u;
        const bool equal = j < cols && key == prefix;
        const uint32_t votes = __ballot_sync(0xFFFFFFFFu, equal);
        if (lane == 0) sh.warp_count[warp] = (uint32_t)__popc(votes);
        __syncthreads();
        uint32_t before = equal_before + (uint32_t)__popc(votes & ((1u << lane) - 1u));
        uint32_t total = 0u;
        for (int w = 0; w < T / 32; ++w) {
            if (w < warp) before += sh.warp_count[w];
            total += sh.warp_count[w];
        }
        if ((j < cols && key > prefix) || (equal && before < want)) list[atomicAdd(&sh.count, 1u)] = entry_of(key, j);
        equal_before += total;
        __syncthreads();
    }
}

// N threads a row: a warp (four rows a CTA), 128 or 512 (a row a CTA).
template <int N> __device__ __forceinline__ void pick_sync() {
    if (N == 32) __syncwarp();
    else __syncthreads();
}
// What they share.
struct PickRow {
    uint32_t votes[2][16];   // of each warp
    uint32_t count;      // candidates found
    uint32_t kept;       // groups that hold some
    int all;             // the list is no use: the row is selected over all its entries
};

// The first `top` of n entries of a list, exactly and in order, by N threads (me: this one's number).
template <int DT, int N> __device__ __forceinline__ void emit_list(const RowPart<DT>& part, const TopArgs& a, int64_t r, uint64_t* list, uint32_t n, uint32_t me) {
    float* values = a.values + r * a.top;
    int32_t* indices = a.indices + r * a.top;
    auto emit = [&](uint32_t place, uint64_t entry) {
        const int j = (int)~(uint32_t)entry;
        const uint32_t key = (uint32_t)(entry >> 32);
        // the logit's own bits: the key has lost the sign of zero and a NaN's payload
        values[place] = key == 0x80000000u || key == 0xFFFFFFFFu ? part.at(j) : key_value(key);
        indices[place] = j;
    };
    if (n <= count_most(N)) {   // an entry's place is the number of larger ones, counted two at a time by `share` threads
        if (me == 0 && (n & 1u)) list[n] = 0ull;   // (room for n entries is room for an even number)
        pick_sync<N>();
        uint32_t share = 1u;
        while (share < 32u && n * share * 2u <= (uint32_t)N) share *= 2u;
        const uint32_t pairs = (n + 1u) / 2u;
        const ulonglong2* two = reinterpret_cast<const ulonglong2*>(list);
        for (uint32_t i0 = 0; i0 < n; i0 += N / share) {
            const uint32_t i = i0 + me / share;
            const uint64_t mine = i < n ? list[i] : 0ull;
            uint32_t above = 0u;
#pragma unroll 4
            for (uint32_t o = me % share; o < pairs; o += share) {
                const ulonglong2 x = two[o];
                above += (x.x > mine ? 1u : 0u) + (x.y > mine ? 1u : 0u);
            }
            for (uint32_t o = share / 2u; o > 0u; o >>= 1) above += __shfl_xor_sync(0xFFFFFFFFu, above, o);
            if (i < n && me % share == 0u && above < (uint32_t)a.top) emit(above, mine);
        }
        return;
    }
    if (N > 32 && n <= kRunsMost) {   // an entry's place is its place in its run and the larger ones of each other run
        const uint32_t lane = threadIdx.x & 31u, runs = (n + 31u) / 32u;
        for (uint32_t run = me >> 5; run < runs; run += N / 32) {
            const uint32_t i = run * 32u + lane;
            uint64_t x = i < n ? list[i] : 0ull;
            for (uint32_t k = 2u; k <= 32u; k <<= 1) {
                for (uint32_t d = k >> 1; d > 0u; d >>= 1) {
                    const uint64_t y = __shfl_xor_sync(0xFFFFFFFFu, x, d);
                    const bool larger = ((lane & d) == 0u) == ((lane & k) == 0u);   // the lane that keeps the larger of the two
                    if (larger == (y > x)) x = y;
                }
            }
            list[i] = x;
        }
        pick_sync<N>();
        for (uint32_t i = me; i < n; i += N) {
            const uint64_t mine = list[i];
            uint32_t place = i & 31u;
#pragma unroll 4
            for (uint32_t run = 0; run < runs; ++run) {
                const uint64_t* in = list + run * 32u;
                uint32_t above = 0u;
#pragma unroll
                for (uint32_t s = 16u; s > 0u; s >>= 1) above += in[above + s - 1u] > mine ? s : 0u;
                above += in[above] > mine ? 1u : 0u;
                place += run == i >> 5 ? 0u : above;
            }
            if (place < (uint32_t)a.top) emit(place, mine);
        }
        return;
    }
    uint32_t size = 2048u;
    if (N == 32) size = 512u;
    while (size < n) size *= 2u;
    for (uint32_t i = n + me; i < size; i += N) list[i] = 0ull;   // below every entry (a column's complement is not 0)
    pick_sync<N>();
    for (uint32_t k = 2u; k <= size; k <<= 1) {
        for (uint32_t d = k >> 1; d > 0u; d >>= 1) {
            for (uint32_t p = me; p < size / 2u; p += N) {
                const uint32_t lo = 2u * p - (p & (d - 1u)), hi = lo + d;
                const uint64_t x = list[lo], y = list[hi];
                if ((x < y) == ((lo & k) == 0u)) {
                    list[lo] = y;
                    list[hi] = x;
                }
            }
            pick_sync<N>();
        }
    }
    for (uint32_t i = me; i < (uint32_t)a.top; i += N) emit(i, list[i]);
}

__host__ __device__ constexpr int pick_threads(int n) { return n == 32 ? 128 : n; }   // of a CTA

template <int DT, int N> __global__ void __launch_bounds__(pick_threads(N)) pick_kernel(const __grid_constant__ TopArgs a) {
    using RV = RowVec<DT>;
    constexpr bool WARP = N == 32;
    constexpr int kPickThreads = pick_threads(N), kRows = kPickThreads / N;   // threads and rows of a CTA
    // Loads in flight and steps unrolled, where a thread has that many: a CTA of 512 has one or two, and comes to its code for
    // the first time, when every further line of it is a wait.
    constexpr int kInFlight = WARP ? 8 : N == 128 ? 4 : 1, kAhead = N == 512 ? 1 : 4;
    __shared__ PickRow rows[kRows];
    __shared__ PickShared sh;
    extern __shared__ __align__(16) unsigned char dyn[];
    const int slot = WARP ? (int)threadIdx.x >> 5 : 0, me = (int)threadIdx.x & (N - 1), lane = (int)threadIdx.x & 31;
    const size_t row_bytes = (size_t)a.list_cap * 10u + (size_t)a.groups * 2u;
    uint64_t* list = reinterpret_cast<uint64_t*>(dyn + slot * row_bytes);              // [list_cap] candidates
    uint32_t* pairs = reinterpret_cast<uint32_t*>(list + a.list_cap);                  // [groups / 2] patterns, two a word
    uint16_t* owner = reinterpret_cast<uint16_t*>(pairs + a.groups / 2);               // [list_cap] groups that hold candidates
    PickRow& row = rows[slot];
    const int64_t r = (int64_t)blockIdx.x * kRows + slot;
    const bool there = r < a.rows;
    if (me == 0) {
        row.count = row.kept = 0u;
        row.all = 0;
    }
    pick_sync<N>();   // before another warp finds a NaN
    await_previous_kernel();
    if (there) {
        const RowPart<DT> part(a.L, r, a.ldl, (int)a.vocab, 0, 1);
        const int nv = part.v_hi, n_groups = (nv + (1 << a.group_shift) - 1) >> a.group_shift, words = (n_groups + 1) / 2;
        // the singles' threads ask for their element now
        const int t = me, n_lone = part.head + part.tail;
        const int lone = t < n_lone ? (t < part.head ? t : part.cols - part.tail + (t - part.head)) : -1;
        const float lone_x = lone >= 0 ? part.at(lone) : -INFINITY;
        const uint32_t* in = reinterpret_cast<const uint32_t*>(a.patterns + r * a.groups);
        uint32_t top_pattern = 0u;
        for (int i = me; i < words; i += N) {
            uint32_t w = in[i];
            if (2 * i + 1 >= n_groups) w &= 0xFFFFu;   // nothing behind the last group
            pairs[i] = w;
            top_pattern = max(top_pattern, max(w & 0xFFFFu, w >> 16));
        }
        SoftStat st = {-INFINITY, 0.0f};
        if (me >= N - 32) {   // the last warp, which has the least to do elsewhere
            for (int p = lane; p < a.parts; p += 32) {
                const float2 s = a.stat[r * a.parts + p];
                st = soft_merge(st, {s.x, s.y}, a.c);
            }
            st = soft_warp(st, a.c);
            if (lane == 0 && st.s != st.s) row.all = 1;   // a NaN
        }
        // ---- a pattern that at least `top` of the groups' maxima reach, the largest or one that few more do (0: all
        // entries are candidates): steps of growing size down from the largest, then bisection of the last
        top_pattern = __reduce_max_sync(0xFFFFFFFFu, top_pattern);
        if (!WARP) {
            if (lane == 0) sh.warp_count[threadIdx.x >> 5] = top_pattern;
            __syncthreads();
            for (int w = 0; w < kPickThreads / 32; ++w) top_pattern = max(top_pattern, sh.warp_count[w]);
        } else {
            __syncwarp();
        }
        uint32_t floor_key = 0u;
        if (n_groups >= a.top) {
            const int slack = 8 + a.top / 8;   // candidates too many that are not worth another step
            int vote = 0;
            auto reach = [&](uint32_t trial) -> int {   // groups that do
                uint32_t n = 0u;
#pragma unroll kAhead
                for (int i = me; i < words; i += N) {
                    const uint32_t w = pairs[i];
                    n += ((w & 0xFFFFu) >= trial ? 1u : 0u) + ((w >> 16) >= trial ? 1u : 0u);
                }
                n = __reduce_add_sync(0xFFFFFFFFu, n);
                if (!WARP) {
                    vote ^= 1;   // two sets in turn: the one before last has been read by all
                    if (lane == 0) row.votes[vote][threadIdx.x >> 5] = n;
                    __syncthreads();
                    n = __reduce_add_sync(0xFFFFFFFFu, lane < N / 32 ? row.votes[vote][lane] : 0u);
                }
                return (int)n;
            };
            uint32_t high = top_pattern + 1u, step = 32u, low;   // fewer than `top` reach `high`
            int n;
            for (;;) {
                low = high > step ? high - step : 0u;
                n = reach(low);
                if (n >= a.top || low == 0u) break;
                high = low;
                step *= 2u;
            }
            while (n > a.top + slack && high - low > 1u) {
                const uint32_t mid = low + (high - low) / 2u;
                const int m = reach(mid);
                if (m >= a.top) {
                    low = mid;
                    n = m;
                } else {
                    high = mid;
                }
            }
            floor_key = low;
        }
        const float least = floor_key == 0u ? -INFINITY : key_value(floor_key << 16);

        // ---- the groups that reach it, and their entries that do
        for (int i = me; i < words; i += N) {
            const uint32_t w = pairs[i];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = h != 0 ? w >> 16 : w & 0xFFFFu;
                if (2 * i + h < n_groups && k >= floor_key) {
                    const uint32_t at = atomicAdd(&row.kept, 1u);
                    if (at < (uint32_t)a.list_cap) owner[at] = (uint16_t)(2 * i + h);
                }
            }
        }
        auto take = [&](float x, int j) {
            const uint32_t at = atomicAdd(&row.count, 1u);
            if (at < (uint32_t)a.list_cap) list[at] = entry_of(order_key(x), j);
        };
        if (lone >= 0 && !(lone_x < least)) take(lone_x, lone);
        pick_sync<N>();
        const uint32_t kept = row.kept;
        bool all = row.all != 0 || kept > (uint32_t)a.list_cap;
        if (!all) {
            const int per = 1 << a.group_shift, work = (int)kept * per;
            for (int u0 = me; u0 < work; u0 += kInFlight * N) {
                uint4 w[kInFlight];
                int v[kInFlight];
#pragma unroll
                for (int i = 0; i < kInFlight; ++i) {
                    const int u = u0 + i * N;
                    v[i] = u < work ? owner[u >> a.group_shift] * per + (u & (per - 1)) : nv;
                    if (v[i] < nv) w[i] = ld_stream16(part.vec(v[i]));
                }
#pragma unroll
                for (int i = 0; i < kInFlight; ++i) {
                    uint32_t mask = v[i] < nv ? reach_mask<DT>(w[i], least) : 0u;
                    while (mask != 0u) {
                        const int e = __ffs(mask) - 1;
                        mask &= mask - 1u;
                        take(RV::any(w[i], e), part.first(v[i]) + e);
                    }
                }
            }
            pick_sync<N>();
            all = row.count > (uint32_t)a.list_cap;
        }
        if (!all) emit_list<DT, N>(part, a, r, list, row.count, (uint32_t)me);
        if (me == N - 32 && a.lse != nullptr) a.lse[r] = (float)soft_lse(st, a.inv_t);   // last: a long fp64 logarithm
        if (me == 0) row.all = all ? 1 : 0;
    }
    // ---- rows whose list is no use, by the whole CTA
    __syncthreads();
    for (int s = 0; s < kRows; ++s) {
        if (!rows[s].all) continue;
        const int64_t rr = (int64_t)blockIdx.x * kRows + s;
        const RowPart<DT> part(a.L, rr, a.ldl, (int)a.vocab, 0, 1);
        uint64_t* l = reinterpret_cast<uint64_t*>(dyn + s * row_bytes);
        select_all<DT, kPickThreads>(part, a.top, l, sh);
        __syncthreads();
        emit_list<DT, kPickThreads>(part, a, rr, l, (uint32_t)a.top, threadIdx.x);
        __syncthreads();
    }
}

// Everything a call's sizes decide.  Groups are eight vectors (128 bytes: what is read again lies together), or one
// where `top` comes near their number: the k-th largest of barely more than k maxima is far down, and most of the row
// a candidate.
void plan_top(TopArgs& a, int dtype) {
    const int64_t nv = row_vectors(a.vocab, dtype);
    a.group_shift = a.top * 4 <= (nv / 8) * 3 ? 3 : 0;
    a.groups = (int)(((nv + 7) / 8 * 8 >> a.group_shift) + 7) / 8 * 8;
    if (a.groups < 8) a.groups = 8;
    a.list_cap = 512;
    while (a.list_cap < 3 * a.top && a.list_cap < 4096) a.list_cap *= 2;
    int64_t per = 4096;   // 64 KB; less where the rows alone would leave SMs idle
    while (per > kSweepThreads && a.rows * ((nv + per - 1) / per) < sm_count() * kSweepCtas) per /= 2;
    a.part_vecs = (int)per;
    a.parts = nv > 0 ? (int)((nv + per - 1) / per) : 1;
}
constexpr int64_t kMostVocab = 1 << 20;   // entries of a row: its patterns lie in the shared memory of one CTA
constexpr int kMostGroups = 32768;        // 2^20 fp32 entries
constexpr size_t kPickSmem = 4096 * 10 + kMostGroups * 2;

template <int DT, int N> int launch_pick(const TopArgs& a, cudaStream_t st) {
    constexpr int kRows = pick_threads(N) / N;
    static DeviceCache opted;   // the shared-memory opt-in belongs to one device's copy of the kernel
    const int ok = opted.get([&]() -> int {
        if (cudaFuncSetAttribute(pick_kernel<DT, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPickSmem) != cudaSuccess) {
            (void)cudaGetLastError();
            return -1;
        }
        return 1;
    });
    if (ok < 0) return MOSAIC_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.rows + kRows - 1) / kRows));
    cfg.blockDim = dim3(pick_threads(N));
    cfg.dynamicSmemBytes = (size_t)kRows * ((size_t)a.list_cap * 10u + (size_t)a.groups * 2u);
    // Where a CTA's row is all that an SM gets, it asks for the shared memory that spreads the rows evenly: four CTAs that
    // start early on one SM while another has none took 28.0 instead of 25.5 us (301 x 50001 fp32).
    const int64_t per_sm = (a.rows + sm_count() - 1) / sm_count();
    if (N == 512 && per_sm <= 4) {
        size_t even = 220 * 1024 / (size_t)per_sm - 3 * 1024;
        if (even > kPickSmem) even = kPickSmem;
        if (cfg.dynamicSmemBytes < even) cfg.dynamicSmemBytes = even;
    }
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    MOSAIC_CUDA_TRY(cudaLaunchKernelEx(&cfg, pick_kernel<DT, N>, a));
    return MOSAIC_OK;
}

template <int DT> int launch_top(const TopArgs& a, cudaStream_t st) {
    sweep_kernel<DT><<<dim3((unsigned)a.rows, (unsigned)a.parts), kSweepThreads, 0, st>>>(a);
    MOSAIC_LAUNCH_CHECK();
    // A row a warp where there are rows enough to fill the SMs so (4096 x 32000 bf16, k 64: 78 us, by 128 threads 82, by
    // 512 110); the fewer there are, the more threads make a row's steps short (1200 rows: 35 us by 128 threads, 47 by a
    // warp, 39 by 512; 301 x 50001 fp32, k 100: 25.5 us by 512 threads, 36 by 128, 51 by a warp).  A warp's row has a
    // quarter of a CTA's shared memory, and sorting a long list is a CTA's work (k 256: 153 us by 128 threads, 182).
    const bool small = 4u * ((size_t)a.list_cap * 10u + (size_t)a.groups * 2u) <= 64u * 1024u && a.top <= 128;
    if (small && a.rows >= 20 * sm_count()) return launch_pick<DT, 32>(a, st);
    return a.rows > 5 * sm_count() ? launch_pick<DT, 128>(a, st) : launch_pick<DT, 512>(a, st);
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" size_t mosaic_top_logits_workspace_bytes(int64_t rows, int64_t vocab, int dtype, int64_t top) {
    if (rows <= 0 || vocab <= 0 || vocab > kMostVocab || top < 1 || top > kMaxTop || (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16)) return 0;
    TopArgs a = {};
    a.rows = rows; a.vocab = vocab; a.top = (int)top;
    plan_top(a, dtype);
    return align_up((size_t)rows * ((size_t)a.parts * sizeof(float2) + (size_t)a.groups * 2u), 256);
}

extern "C" int mosaic_top_logits(const void* L, int64_t rows, int64_t vocab, int64_t ldl, int dtype, int64_t top, float temperature,
                                 float* values, int32_t* indices, float* lse, void* ws, size_t ws_bytes, void* stream) {
    if (dtype != MOSAIC_F32 && dtype != MOSAIC_BF16) return MOSAIC_ERR_BAD_DTYPE;
    if (rows < 0 || rows > 0x7FFFFFFF || vocab <= 0 || vocab > kMostVocab || ldl < vocab || top < 1 || top > kMaxTop || top > vocab)
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
    if (ws == nullptr) return MOSAIC_ERR_NULL_PTR;
    if ((reinterpret_cast<uintptr_t>(ws) & 255u) != 0) return MOSAIC_ERR_MISALIGNED;
    if (ws_bytes < mosaic_top_logits_workspace_bytes(rows, vocab, dtype, top)) return MOSAIC_ERR_WORKSPACE_TOO_SMALL;
    TopArgs a = {};
    a.L = L; a.rows = rows; a.vocab = vocab; a.ldl = ldl; a.top = (int)top;
    a.values = values; a.indices = indices; a.lse = lse;
    a.inv_t = 1.0 / (double)temperature;
    a.c = (float)(1.4426950408889634 / (double)temperature);
    plan_top(a, dtype);
    a.patterns = static_cast<uint16_t*>(ws);   // rows of 16 bytes
    a.stat = reinterpret_cast<float2*>(a.patterns + (size_t)rows * (size_t)a.groups);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == MOSAIC_BF16 ? launch_top<MOSAIC_BF16>(a, st) : launch_top<MOSAIC_F32>(a, st);
}
