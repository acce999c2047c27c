// Norms of queries and keys for each head and the rotation by position, in one pass over both.
//
//   n = x rsqrt(mean(x^2) + eps), z = w n, and of the first `rotary` elements of z pairs turn by
//   position * base^(-2i / rotary): y1 = z1 cos - z2 sin, y2 = z2 cos + z1 sin.
// Gradient: g = dy turned back, dw = sum g n, u = w g, dx = rstd (u - n mean(u n)).
//
// Angles. A position times a frequency in turns, modulo one turn, is what counts: the host gives
// each pair's turns per position as a 64-bit binary fraction, and one 64-bit product, whose
// overflow drops the whole turns, is exact for positions of any size. Both sines are taken once a
// token and used for every head of it.
//
// Both directions are bound by memory: 2 (3) accesses of each element. A group of 8, 16 or 32 lanes
// takes a head, eight elements a lane as two runs of four: the two halves of four pairs, so that
// a pair is in one lane, and a run of the lanes is whole lines. A warp takes a token's heads in
// turn, so that the angles and the norms' weights stay in registers.
#include "layers.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 2;  // heads of a group that are on their way at once

// Four neighbours as floats.
template <typename T>
__device__ __forceinline__ void load4(const T *p, float *v)
{
    const Vec<T, 4> e = *reinterpret_cast<const Vec<T, 4> *>(p);
    const float2 a = pair_of(e.e), b = pair_of(e.e + 2);
    v[0] = a.x;
    v[1] = a.y;
    v[2] = b.x;
    v[3] = b.y;
}
template <typename T>
__device__ __forceinline__ void store4(T *p, const float *v)
{
    Vec<T, 4> e;
    put_pair(e.e, make_float2(v[0], v[1]));
    put_pair(e.e + 2, make_float2(v[2], v[3]));
    *reinterpret_cast<Vec<T, 4> *>(p) = e;
}

__device__ __forceinline__ void angle(int64_t position, uint64_t turns, float &c, float &s)
{
    const uint64_t at = uint64_t(position) * turns;  // of a turn, in units of 2^-64
    sincospif(float(int32_t(at >> 32)) * 0x1p-31f, &s, &c);
}

// A unit of work: heads [h0, h1) of a token, queries' heads first, then the keys'.
struct Unit {
    int64_t token;
    int32_t h0, h1;
};
__device__ __forceinline__ Unit unit_at(const HeadNormArgs &a, int64_t u)
{
    const int heads = a.heads[0] + a.heads[1];
    Unit q;
    q.token = u / a.parts;
    const int part = int(u - q.token * a.parts);
    q.h0 = part * a.per_part;
    q.h1 = min(heads, q.h0 + a.per_part);
    return q;
}

// Sums of weights' gradients: lanes of the block that hold the same elements, then the block's row.
// values [2][8] of each lane; partial [blocks][2][D].
template <int LANES>
__device__ __forceinline__ void add_up(const HeadNormArgs &a, float (&dw)[2][8], const int (&at)[2], bool mine)
{
    __shared__ float sums[2][kWarps][DC_HEAD_NORM_DIM_MAX];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int o = LANES; o < 32; o *= 2) dw[which][j] += __shfl_xor_sync(0xffffffffu, dw[which][j], o);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (lane < LANES && mine)
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[which][warp][at[j / 4] + j % 4] = dw[which][j];
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.D; i += kThreads) {
        const int which = i / a.D, e = i - which * a.D;
        float t = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) t += sums[which][w][e];
        a.partial[int64_t(blockIdx.x) * 2 * a.D + i] = t;
    }
}

template <typename T, int LANES, bool GRAD>
__global__ void __launch_bounds__(kThreads) head_norm_kernel(const __grid_constant__ HeadNormArgs a)
{
    constexpr int kHeads = 32 / LANES;  // at a time, of a warp
    const int lane = threadIdx.x % 32, l = lane % LANES, group = lane / LANES;
    const bool mine = l * 8 < a.D, turned = l * 8 < a.rotary;
    // first elements of the lane's two runs
    int at[2] = {8 * l, 8 * l + 4};
    if (turned && !a.interleaved) {
        at[0] = 4 * l;
        at[1] = a.rotary / 2 + 4 * l;
    }
    float w[2][8];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            w[which][j] = mine && a.w[which] ? to_float(static_cast<const T *>(a.w[which])[at[j / 4] + j % 4]) : 1.0f;
    float dw[2][8] = {};
    const float inverse = 1.0f / float(a.D);

    // One token after another (a block's warps take neighbours).
    const int64_t units = a.tokens * a.parts;
    for (int64_t u = int64_t(blockIdx.x) * kWarps + threadIdx.x / 32; u < units; u += int64_t(gridDim.x) * kWarps) {
        const Unit q = unit_at(a, u);
        float c[4], s[4];
        {
            const int64_t position = a.positions[q.token];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = 1.0f;
                s[j] = 0.0f;
                if (turned) angle(position, a.turns[4 * l + j], c[j], s[j]);
            }
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            const int first = which ? a.heads[0] : 0, end = min(q.h1, first + a.heads[which]);
            const T *x = static_cast<const T *>(a.x[which]) + q.token * a.token[which];
            const int64_t row = q.token * a.heads[which];
            const T *dy = GRAD ? static_cast<const T *>(a.dy[which]) + row * a.D : nullptr;
            T *y = static_cast<T *>(a.y[which]) + row * a.D;
            for (int h0 = max(q.h0, first); h0 < end; h0 += kHeads * kUnroll) {
                float v[kUnroll][8], d[GRAD ? kUnroll : 1][8];
#pragma unroll
                for (int i = 0; i < kUnroll; ++i) {
                    const int h = h0 + i * kHeads + group - first;
                    const bool there = mine && h + first < end;
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
                    if (there) {
                        load4(x + h * a.head[which] + at[0], v[i]);
                        load4(x + h * a.head[which] + at[1], v[i] + 4);
                    }
                    if constexpr (GRAD) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) d[i][j] = 0.0f;
                        if (there) {
                            load4(dy + int64_t(h) * a.D + at[0], d[i]);
                            load4(dy + int64_t(h) * a.D + at[1], d[i] + 4);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < kUnroll; ++i) {
                    const int h = h0 + i * kHeads + group - first;
                    // a pair (e, f) of v[j], turned by (c, s): halves of pairs are four apart, or neighbours
                    auto turn = [&](float(&t)[8], float sign) {
                        if (!a.interleaved) {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float e = t[j], f = t[j + 4];
                                t[j] = e * c[j] - sign * f * s[j];
                                t[j + 4] = f * c[j] + sign * e * s[j];
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float e = t[2 * j], f = t[2 * j + 1];
                                t[2 * j] = e * c[j] - sign * f * s[j];
                                t[2 * j + 1] = f * c[j] + sign * e * s[j];
                            }
                        }
                    };
                    float square = 0.0f, along = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) square += v[i][j] * v[i][j];
                    if constexpr (GRAD) {
                        if (turned) turn(d[i], -1.0f);
#pragma unroll
                        for (int j = 0; j < 8; ++j) along += d[i][j] * w[which][j] * v[i][j];
                    }
                    float rstd = 1.0f;
                    if (a.norm) {
#pragma unroll
                        for (int o = LANES / 2; o > 0; o /= 2) {
                            square += __shfl_xor_sync(0xffffffffu, square, o);
                            if (GRAD) along += __shfl_xor_sync(0xffffffffu, along, o);
                        }
                        rstd = rsqrtf(square * inverse + a.eps);
                    } else {
                        along = 0.0f;
                    }
                    float out[8];
                    if constexpr (GRAD) {
                        const float back = along * inverse * rstd * rstd;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            dw[which][j] += d[i][j] * (v[i][j] * rstd);
                            out[j] = rstd * (d[i][j] * w[which][j] - v[i][j] * back);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 8; ++j) out[j] = v[i][j] * rstd * w[which][j];
                        if (turned) turn(out, 1.0f);
                    }
                    if (mine && h + first < end) {
                        store4(y + int64_t(h) * a.D + at[0], out);
                        store4(y + int64_t(h) * a.D + at[1], out + 4);
                    }
                }
            }
        }
    }
    if (GRAD && a.partial) add_up<LANES>(a, dw, at, mine);
}

// Sizes and strides of any kind: a warp per head, four pairs a lane, one element an access. Pairs
// from rotary / 2 on are neighbours that do not turn; the last may be a single element.
template <typename T, bool GRAD>
__global__ void __launch_bounds__(kThreads) head_norm_any_kernel(const __grid_constant__ HeadNormArgs a)
{
    constexpr int kPairs = DC_HEAD_NORM_DIM_MAX / 2 / 32;
    const int lane = threadIdx.x % 32, half = a.rotary / 2;
    int e[kPairs][2];  // the pairs' elements; D and above: none
    float w[2][kPairs][2], dw[2][kPairs][2] = {};
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const int p = lane + 32 * j;
        e[j][0] = p >= half || a.interleaved ? 2 * p : p;
        e[j][1] = p >= half || a.interleaved ? 2 * p + 1 : p + half;
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                w[which][j][k] =
                    e[j][k] < a.D && a.w[which] ? to_float(static_cast<const T *>(a.w[which])[e[j][k]]) : 1.0f;
    }
    const float inverse = 1.0f / float(a.D);
    const int64_t units = a.tokens * a.parts;
    for (int64_t u = int64_t(blockIdx.x) * kWarps + threadIdx.x / 32; u < units; u += int64_t(gridDim.x) * kWarps) {
        const Unit q = unit_at(a, u);
        float c[kPairs], s[kPairs];
        const int64_t position = a.positions[q.token];
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            c[j] = 1.0f;
            s[j] = 0.0f;
            if (lane + 32 * j < half) angle(position, a.turns[lane + 32 * j], c[j], s[j]);
        }
        for (int at = q.h0; at < q.h1; ++at) {
            const int which = at >= a.heads[0], h = at - (which ? a.heads[0] : 0);
            const T *x = static_cast<const T *>(a.x[which]) + q.token * a.token[which] + h * a.head[which];
            const int64_t row = (q.token * a.heads[which] + h) * a.D;
            float v[kPairs][2], d[kPairs][2];
            float square = 0.0f, along = 0.0f;
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const bool there = e[j][k] < a.D;
                    v[j][k] = there ? to_float(x[e[j][k]]) : 0.0f;
                    square += v[j][k] * v[j][k];
                    if (GRAD) d[j][k] = there ? to_float(static_cast<const T *>(a.dy[which])[row + e[j][k]]) : 0.0f;
                }
            auto turn = [&](float(&t)[kPairs][2], float sign) {
#pragma unroll
                for (int j = 0; j < kPairs; ++j) {
                    const float p = t[j][0], r = t[j][1];
                    t[j][0] = p * c[j] - sign * r * s[j];
                    t[j][1] = r * c[j] + sign * p * s[j];
                }
            };
            auto weight = [&](int j, int k) { return which ? w[1][j][k] : w[0][j][k]; };
            if (GRAD) {
                turn(d, -1.0f);
#pragma unroll
                for (int j = 0; j < kPairs; ++j)
#pragma unroll
                    for (int k = 0; k < 2; ++k) along += d[j][k] * weight(j, k) * v[j][k];
            }
            float rstd = 1.0f;
            if (a.norm) {
#pragma unroll
                for (int o = 16; o > 0; o /= 2) {
                    square += __shfl_xor_sync(0xffffffffu, square, o);
                    if (GRAD) along += __shfl_xor_sync(0xffffffffu, along, o);
                }
                rstd = rsqrtf(square * inverse + a.eps);
            } else {
                along = 0.0f;
            }
            float out[kPairs][2];
            const float back = along * inverse * rstd * rstd;
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (GRAD) {
                        const float t = d[j][k] * (v[j][k] * rstd);
                        if (which) dw[1][j][k] += t;
                        else dw[0][j][k] += t;
                        out[j][k] = rstd * (d[j][k] * weight(j, k) - v[j][k] * back);
                    } else {
                        out[j][k] = v[j][k] * rstd * weight(j, k);
                    }
                }
            if (!GRAD) turn(out, 1.0f);
            T *y = static_cast<T *>(a.y[which]) + row;
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (e[j][k] < a.D) y[e[j][k]] = from_float<T>(out[j][k]);
        }
    }
    if (GRAD && a.partial) {
        __shared__ float sums[2][kWarps][DC_HEAD_NORM_DIM_MAX];
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (e[j][k] < a.D) sums[which][threadIdx.x / 32][e[j][k]] = dw[which][j][k];
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * a.D; i += kThreads) {
            const int which = i / a.D, at = i - which * a.D;
            float t = 0.0f;
#pragma unroll
            for (int r = 0; r < kWarps; ++r) t += sums[which][r][at];
            a.partial[int64_t(blockIdx.x) * 2 * a.D + i] = t;
        }
    }
}

// dw of both weights from the blocks' rows, in a fixed order: a warp per element.
__global__ void __launch_bounds__(kThreads)
weight_sums_kernel(const float *partial, int blocks, int D, float *dw_q, float *dw_k)
{
    const int i = blockIdx.x * kWarps + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (i >= 2 * D) return;
    float t = 0.0f;
    for (int b = lane; b < blocks; b += 32) t += partial[int64_t(b) * 2 * D + i];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
    float *out = i < D ? dw_q : dw_k;
    if (lane == 0 && out) out[i < D ? i : i - D] = t;
}

constexpr int kMostBlocks = 8 * 160;  // rows that the weights' gradients may have

template <typename T, bool GRAD>
cudaError_t launch(HeadNormArgs a, bool vector, cudaStream_t stream)
{
    int sms = 0;
    const cudaError_t e = sm_count(sms);
    if (e != cudaSuccess) return e;
    // Few tokens: heads are dealt to warps as finely as needed to fill the SMs
    const int heads = a.heads[0] + a.heads[1], lanes = a.D <= 64 ? 8 : a.D <= 128 ? 16 : 32;
    const int least = vector ? 32 / lanes * kUnroll : 1;
    const int64_t wanted = int64_t(sms) * 4 * kWarps;
    a.parts = 1;
    while (a.tokens * a.parts < wanted && heads > a.parts * least) a.parts *= 2;
    a.per_part = (heads + a.parts - 1) / a.parts;
    const int64_t blocks = (a.tokens * a.parts + kWarps - 1) / kWarps;
    int most = sms * 8 < kMostBlocks ? sms * 8 : kMostBlocks;
    const int grid = int(blocks < most ? blocks : most);
    if (!vector) {
        head_norm_any_kernel<T, GRAD><<<grid, kThreads, 0, stream>>>(a);
    } else {
        switch (lanes) {
            case 8: head_norm_kernel<T, 8, GRAD><<<grid, kThreads, 0, stream>>>(a); break;
            case 16: head_norm_kernel<T, 16, GRAD><<<grid, kThreads, 0, stream>>>(a); break;
            default: head_norm_kernel<T, 32, GRAD><<<grid, kThreads, 0, stream>>>(a);
        }
    }
    if (GRAD && a.partial)
        weight_sums_kernel<<<(2 * a.D + kWarps - 1) / kWarps, kThreads, 0, stream>>>(a.partial, grid, a.D, a.dw[0],
                                                                                     a.dw[1]);
    return cudaGetLastError();
}

// Runs of four elements: whole accesses, and no pair apart from its run's partner.
bool in_runs(int dtype, const HeadNormArgs &a, bool grad)
{
    const size_t bytes = 4 * size_t(dtype_bytes(dtype));
    auto fits = [&](const void *p) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; };
    bool ok = a.D % 8 == 0 && a.rotary % 8 == 0;
    for (int i = 0; i < 2; ++i)
        ok = ok && a.token[i] % 4 == 0 && a.head[i] % 4 == 0 && fits(a.x[i]) && fits(a.y[i]) &&
             (!grad || fits(a.dy[i]));
    return ok;
}

}  // namespace

size_t head_norm_workspace(int D) { return sizeof(float) * 2 * size_t(D) * kMostBlocks; }

cudaError_t launch_head_norm(int dtype, const HeadNormArgs &a, cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, return (launch<T, false>(a, in_runs(dtype, a, false), stream));)
}

cudaError_t launch_head_norm_grad(int dtype, const HeadNormArgs &a, cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, return (launch<T, true>(a, in_runs(dtype, a, true), stream));)
}

}  // namespace dc
