// Where an expert's rows lie: the offsets made safe, and the tiles that rows of every
// expert are cut into.
#pragma once

#include "layers.cuh"

namespace dc {

// Segment 0 holds the rows before the first expert, segment e + 1 those of expert e,
// segment experts + 1 the rows after the last: together they cover [0, rows) once,
// whatever the offsets hold (each is clamped to [0, rows] and to the largest before it).
struct Segments {
    int32_t *start;  // [experts + 3] first row of each segment, then rows
    int32_t *tile;   // [experts + 3] first whole tile of each segment, then the whole tiles in all
    int32_t *part;   // [experts + 3] first tile of each segment's last rows, then the tiles in all
    int count;       // experts + 2
};

// Float operands of a weight gradient are stored with each segment's rows rounded up to this.
constexpr int kPartRows = 32;

__host__ __device__ inline size_t segments_bytes(int experts) { return size_t(experts + 3) * 12; }

__device__ __forceinline__ Segments segments_at(void *smem, int experts)
{
    Segments s;
    s.start = static_cast<int32_t *>(smem);
    s.tile = s.start + experts + 3;
    s.part = s.tile + experts + 3;
    s.count = experts + 2;
    return s;
}

// By one warp: starts, then tiles of `rows_per_tile` rows, each `per` times. Whole tiles come
// first and those of the rows that are left over last, so that CTAs that take every so-manieth
// tile finish together (split: else a segment's short tile follows its whole ones, all in
// `tile`).
template <bool SPLIT>
__device__ __forceinline__ void build_segments(const Segments &s, const int64_t *offsets,
                                               int64_t rows, int experts, int rows_per_tile,
                                               int per)
{
    const int lane = threadIdx.x & 31;
    int64_t top = 0;
    if (lane == 0) {
        s.start[0] = 0;
        s.start[s.count] = int32_t(rows);
    }
    for (int e0 = 0; e0 <= experts; e0 += 32) {
        const int e = e0 + lane;
        int64_t v = e <= experts ? offsets[e] : 0;
        v = v < 0 ? 0 : v > rows ? rows : v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o && u > v) v = u;
        }
        if (v < top) v = top;
        if (e <= experts) s.start[e + 1] = int32_t(v);
        top = __shfl_sync(0xffffffffu, v, 31);
    }
    __syncwarp();
    int32_t base = 0;
    auto prefix = [&](int32_t *out, auto &&tiles_of) {
        for (int e0 = 0; e0 <= s.count; e0 += 32) {
            const int e = e0 + lane;
            const int32_t n = e < s.count ? tiles_of(s.start[e + 1] - s.start[e]) * per : 0;
            int32_t t = n;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int32_t u = __shfl_up_sync(0xffffffffu, t, o);
                if (lane >= o) t += u;
            }
            if (e <= s.count) out[e] = base + t - n;
            base += __shfl_sync(0xffffffffu, t, 31);
        }
    };
    if (SPLIT) {
        prefix(s.tile, [&](int32_t rows) { return rows / rows_per_tile; });
        prefix(s.part, [&](int32_t rows) { return rows % rows_per_tile ? 1 : 0; });
    } else {
        prefix(s.tile, [&](int32_t rows) { return rows / rows_per_tile + (rows % rows_per_tile ? 1 : 0); });
    }
    __syncwarp();
}

// The segment that holds tile t of a prefix over segments (t below the tiles in all).
__device__ __forceinline__ int find_segment(const int32_t *first, int count, int t)
{
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

}  // namespace dc
