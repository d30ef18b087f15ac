// Eight adjacent bf16 elements of a row a lane, 256 a warp, at any alignment: what the elementwise passes read and write.
#pragma once
#include "linear.cuh"

namespace mosaic {
#ifdef __CUDACC__
constexpr int kLaneCols = 8, kWarpCols = 32 * kLaneCols;

// Columns c0 + 8 lane .. + 7 of a row (c0 a multiple of 8 and the same for the warp); zeros past the last column, which nothing is read
// of.  VEC: the row starts on a 16-byte boundary, one load a lane.  Otherwise the warp reads 32 adjacent elements a load, whose
// segments are whole whatever the alignment, and turns them round in `turn` (its own 512 bytes of shared memory).  The
// whole warp calls.  Ordinary loads, ordered behind the wait for the kernel before this one.
template <bool VEC> __device__ __forceinline__ void lane_load8(const uint16_t* row, int64_t c0, int64_t cols, uint4* turn, uint32_t (&w)[4]) {
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
template <bool VEC> __device__ __forceinline__ void lane_store8(uint16_t* row, int64_t c0, int64_t cols, uint4* turn, const uint32_t (&w)[4]) {
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
