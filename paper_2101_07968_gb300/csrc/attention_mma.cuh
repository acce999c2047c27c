// What the forward pass and the gradient of attention on the tensor cores share.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "attention.cuh"
#include "blackwell.cuh"

namespace dc {
namespace am {

constexpr int kTile = kMmaRows;                // rows and keys of a block of scores
constexpr uint32_t kBox = kTile * 128;         // bytes of 64 elements of each of a tile's rows

__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// the largest of three, one instruction; a NaN counts as none
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
    return m;
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float2 unpack2(uint32_t v, __nv_bfloat16) { return pair_of(reinterpret_cast<const __nv_bfloat16 *>(&v)); }
__device__ __forceinline__ float2 unpack2(uint32_t v, __half) { return pair_of(reinterpret_cast<const __half *>(&v)); }

// Bits 15 and 31 say whether any of eight elements is an infinity or NaN: an exponent of all ones carries over.
template <typename T>
__device__ __forceinline__ uint32_t not_finite(uint4 v)
{
    constexpr uint32_t e = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
    constexpr uint32_t one = std::is_same<T, __half>::value ? 0x04000400u : 0x00800080u;
    return ((v.x & e) + one) | ((v.y & e) + one) | ((v.z & e) + one) | ((v.w & e) + one);
}

// Sixteen bytes of a tile's row as the copies lay them: boxes of 64 elements, 128 bytes a row, the
// 16-byte unit turned by the row.
__device__ __forceinline__ uint4 tile_unit(const unsigned char *tile, int row, int unit)
{
    return *reinterpret_cast<const uint4 *>(tile + (unit >> 3) * kBox + row * 128 + (((unit & 7) ^ (row & 7)) << 4));
}

// Thread r of 128 looks through row r of a tile: whether it has an infinity or NaN. Rows from `rows` on
// are of another sequence, or of none: they become zeros.
template <typename T, int DP>
__device__ __forceinline__ bool look_through(unsigned char *tile, int r, int rows)
{
    uint32_t bad = 0;
    if (r < rows) {
#pragma unroll
        for (int u = 0; u < DP / 8; ++u) bad |= not_finite<T>(tile_unit(tile, r, u));
    } else {
#pragma unroll
        for (int u = 0; u < DP / 8; ++u)
            *reinterpret_cast<uint4 *>(tile + (u >> 3) * kBox + r * 128 + ((u & 7) << 4)) = make_uint4(0, 0, 0, 0);
        bw::fence_async();
    }
    return (bad & 0x80008000u) != 0;
}

// acc[lane][..] (+)= the sum of w[lane][c] B[c][..] over columns c of the lane's own range [from, end), on the
// CUDA cores: where B holds infinities or NaN that some lanes must not see, zero weights
// would not hide them. w: packed pairs in tensor memory, 16 columns for 32 c, at(c / 32); DP columns of acc.
template <typename T, int DP, typename At>
__device__ __forceinline__ void masked_product(uint32_t acc, At at, int groups, const unsigned char *tile, int row0, int from,
                                            int end, bool add)
{
    for (int d0 = 0; d0 < DP; d0 += 16) {
        float sum[16];
        __syncwarp();
        if (add) {
            bw::tmem_load(acc + d0, sum);
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) sum[j] = 0.0f;
        }
        for (int c0 = 0; c0 < groups * 32; c0 += 32) {
            float w[16];
            __syncwarp();
            bw::tmem_load(at(c0 / 32), w);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const int c = row0 + c0 + i;
                if (c < from || c >= end) continue;
                const float2 both = unpack2(__float_as_uint(w[i / 2]), T());
                const float x = i & 1 ? both.y : both.x;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint4 b = tile_unit(tile, c, d0 / 8 + u);
                    const float2 b0 = unpack2(b.x, T()), b1 = unpack2(b.y, T()), b2 = unpack2(b.z, T()), b3 = unpack2(b.w, T());
                    sum[8 * u] += x * b0.x;
                    sum[8 * u + 1] += x * b0.y;
                    sum[8 * u + 2] += x * b1.x;
                    sum[8 * u + 3] += x * b1.y;
                    sum[8 * u + 4] += x * b2.x;
                    sum[8 * u + 5] += x * b2.y;
                    sum[8 * u + 6] += x * b3.x;
                    sum[8 * u + 7] += x * b3.y;
                }
            }
        }
        uint32_t out[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) out[j] = __float_as_uint(sum[j]);
        __syncwarp();
        bw::tmem_store(acc + d0, out);
    }
    bw::tmem_stored();
}

// N neighbours of a lane's row, times `by`, to memory; D: what is left of the row from here.
template <typename T, int N>
__device__ __forceinline__ void put_row(T *y, const float (&v)[N], float by, int D, bool wide)
{
    if (wide) {
#pragma unroll
        for (int j = 0; j < N; j += 8)
            if (j < D)
                *reinterpret_cast<uint4 *>(y + j) =
                    make_uint4(pack2(v[j] * by, v[j + 1] * by, T()), pack2(v[j + 2] * by, v[j + 3] * by, T()),
                               pack2(v[j + 4] * by, v[j + 5] * by, T()), pack2(v[j + 6] * by, v[j + 7] * by, T()));
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < D) y[j] = from_float<T>(v[j] * by);
    }
}

template <int N>
__device__ __forceinline__ void put_floats(float *y, const float (&v)[N], float by, int D)
{
    if (D >= N && (reinterpret_cast<uintptr_t>(y) & 15) == 0) {
#pragma unroll
        for (int j = 0; j < N; j += 4)
            *reinterpret_cast<float4 *>(y + j) = make_float4(v[j] * by, v[j + 1] * by, v[j + 2] * by, v[j + 3] * by);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < D) y[j] = v[j] * by;
    }
}

// Zeros in the lane's row.
template <typename T>
__device__ __forceinline__ void put_zeros(T *y, int D, bool wide)
{
    if (wide) {
        for (int j = 0; j < D; j += 8) *reinterpret_cast<uint4 *>(y + j) = make_uint4(0, 0, 0, 0);
    } else {
        for (int j = 0; j < D; ++j) y[j] = from_float<T>(0.0f);
    }
}

// ------------------------------------------------------------------------------ host
// A map of [tokens][heads][D], copied in boxes of 64 elements of one head of 128 tokens.
bool heads_map(CUtensorMap &map, int dtype, const void *base, int32_t D, int32_t heads, int64_t tokens, int64_t head,
               int64_t token);

}  // namespace am
}  // namespace dc
