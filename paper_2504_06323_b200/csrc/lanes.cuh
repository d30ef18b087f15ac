// Eight adjacent bf16 elements of a row a lane, 256 a warp, at any alignment: what the elementwise passes read and write.
#pragma once
#include "linear.cuh"

namespace mosaic {
#ifdef __CUDACC__
constexpr int kLaneCols = 8, kWarpCols = 32 * kLaneCols, kTurn = 33;

// Columns c0 + 8 lane .. + 7 of a row (c0 a multiple of 8 and the same for the warp); zeros past the last column, which nothing is read
// of.  VEC: the row starts on a 16-byte boundary, one load a lane.  Otherwise the warp reads 32 adjacent elements a load, whose
// segments are whole whatever the alignment, and turns them round in `turn` (its own kTurn pieces of shared memory); with WORDS the
// words that its columns lie in, but at the row's ends: half the loads and a few more instructions, which pays where loads'
// latency counts (the gated slope pass: 64 -> 57 us with its product) and not where issue does (packing: 36.2 for 34.8, unpacking
// 20.5 for 18.8).
// The whole warp calls.  Ordinary loads, ordered behind the wait for the kernel before this one.
template <bool VEC, bool WORDS = false> __device__ __forceinline__ void lane_load8(const uint16_t* row, int64_t c0, int64_t cols, uint4* turn, uint32_t (&w)[4]) {
    const int lane = (int)threadIdx.x & 31;
    const int64_t c = c0 + lane * kLaneCols;
    if constexpr (VEC) {
        if (c + kLaneCols <= cols) {
            const uint4 v = ld_stream16(row + c);
            w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = c + 2 * e < cols ? row[c + 2 * e] : 0u, hi = c + 2 * e + 1 < cols ? row[c + 2 * e + 1] : 0u;
                w[e] = lo | (hi << 16);
            }
        }
    } else if (const int s = (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 1; WORDS && c0 >= s && c0 + kWarpCols < cols) {
        // whole words: from the element before, where the row begins in the middle of one
        const uint32_t* base = reinterpret_cast<const uint32_t*>(row + c0 - s);
        uint32_t x[4], last = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = base[e * 32 + lane];
        if (s != 0 && lane == 31) last = base[128];
        uint32_t* words = reinterpret_cast<uint32_t*>(turn);
        __syncwarp();   // what the warp read of its buffer before is in its registers
#pragma unroll
        for (int e = 0; e < 4; ++e) words[e * 32 + lane] = x[e];
        if (s != 0 && lane == 31) words[128] = last;
        __syncwarp();
        const uint4 v = turn[lane];
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
        if (s != 0) {
            const uint32_t next = words[4 * lane + 4];
            w[0] = __byte_perm(v.x, v.y, 0x5432);
            w[1] = __byte_perm(v.y, v.z, 0x5432);
            w[2] = __byte_perm(v.z, v.w, 0x5432);
            w[3] = __byte_perm(v.w, next, 0x5432);
        }
    } else {
        uint16_t x[kLaneCols];
#pragma unroll
        for (int e = 0; e < kLaneCols; ++e) {
            const int64_t at = c0 + e * 32 + lane;
            x[e] = at < cols ? row[at] : (uint16_t)0;
        }
        __syncwarp();   // what the warp read of its buffer before is in its registers
#pragma unroll
        for (int e = 0; e < kLaneCols; ++e) reinterpret_cast<uint16_t*>(turn)[e * 32 + lane] = x[e];
        __syncwarp();
        const uint4 v = turn[lane];
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
}

// The way back; columns from `cols` on are not written.
template <bool VEC, bool WORDS = false> __device__ __forceinline__ void lane_store8(uint16_t* row, int64_t c0, int64_t cols, uint4* turn, const uint32_t (&w)[4]) {
    const int lane = (int)threadIdx.x & 31;
    const int64_t c = c0 + lane * kLaneCols;
    if constexpr (VEC) {
        if (c + kLaneCols <= cols) {
            st_stream16(row + c, make_uint4(w[0], w[1], w[2], w[3]));
        } else {
#pragma unroll
            for (int e = 0; e < kLaneCols; ++e)
                if (c + e < cols) row[c + e] = (uint16_t)((e & 1) ? w[e >> 1] >> 16 : w[e >> 1]);
        }
    } else {
        __syncwarp();
        turn[lane] = make_uint4(w[0], w[1], w[2], w[3]);
        __syncwarp();
        if (WORDS && c0 + kWarpCols <= cols) {
            const int s = (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 1;
            const uint32_t* words = reinterpret_cast<const uint32_t*>(turn);
            uint32_t* base = reinterpret_cast<uint32_t*>(row + c0 - s);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = e * 32 + lane;
                if (s == 0) base[k] = words[k];
                else if (k > 0) base[k] = __byte_perm(words[k - 1], words[k], 0x5432);
            }
            // what shares its word with columns that are others' to write
            if (s != 0 && lane == 0) row[c0] = (uint16_t)words[0];
            if (s != 0 && lane == 31) row[c0 + kWarpCols - 1] = (uint16_t)(words[127] >> 16);
            return;
        }
#pragma unroll
        for (int e = 0; e < kLaneCols; ++e) {
            const int64_t at = c0 + e * 32 + lane;
            if (at < cols) row[at] = reinterpret_cast<const uint16_t*>(turn)[e * 32 + lane];
        }
    }
}

__device__ __forceinline__ float half_of(const uint32_t (&w)[4], int e) {
    return __uint_as_float((e & 1) ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}
#endif
}  // namespace mosaic
