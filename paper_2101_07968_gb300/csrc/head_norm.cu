// Norms of queries and keys for each head and the rotation by position, in one pass over both.
//
//   n = x rsqrt(mean(x^2) + eps), z = w n, and of the first `rotary` elements of z pairs turn by
//   position * base^(-2i / rotary): y1 = z1 cos - z2 sin, y2 = z2 cos + z1 sin.
// Gradient: g = dy turned back, dw = sum g n, u = w g, dx = rstd (u - n mean(u n)).
//
// Angles. A position times a frequency in turns, modulo one turn, is what counts: the host gives
// each pair's turns per position as a 128-bit binary fraction (turns.cuh), and the upper half of its product with the
// position, whose overflow drops the whole turns, is good to 2^-48 of a turn for every 64-bit position (64 bits of
// fraction would be a whole turn off at 2^63). The sines take 32 bits of it. Both are taken once a token and used for
// every head of it.
//
// Both directions are bound by memory: 2 (3) accesses of each element. A group of 8, 16 or 32 lanes
// takes a head, eight elements a lane as two runs of four: the two halves of four pairs, so that
// a pair is in one lane, and a run of the lanes is whole lines. Blocks are dealt to queries and keys by
// their shares, so that a thread holds one weight and its gradient; a group takes a token's heads
// in turn with the angles in registers. What it takes next comes by asynchronous copies, each lane
// its own runs, several chunks ahead: loads to registers kept too few bytes on their way
// (32,768 tokens x 40 heads x 128, gradient: 419 us at 25 % occupancy and 31 % of the issue slots). Now 172 us, 5.8 TB/s,
// and 121 us forward, 5.5 TB/s; floats 319 us, 6.3 TB/s, and 219 us, 6.1 TB/s.
#include <type_traits>

#include "layers.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kUnroll = 2;  // heads in a chunk of a group

template <int N>
__device__ __forceinline__ void angle(const Turns<N> &turns, int64_t position, int pair, float &c, float &s)
{
    uint64_t at = uint64_t(position) * turns.upper[pair];  // of a turn, in units of 2^-64
    // the lower half counts for less than the 32 bits that are used, but for far positions (a branch that most
    // tokens do not take: without it 32,768 tokens x 40 heads x 128 take 187 us backward instead of 172)
    if (position != int64_t(int32_t(position))) {
        int p;  // (the lower half is not to be read ahead of the branch)
        asm volatile("mov.u32 %0, %1;" : "=r"(p) : "r"(pair));
        const uint64_t below = turns.below[p];
        at += __umul64hi(uint64_t(position), below);
        if (position < 0) at -= below;  // as an unsigned number it is 2^64 too large
    }
    sincospif(float(int32_t(at >> 32)) * 0x1p-31f, &s, &c);
}

// A unit of work: heads [h0, h1) of a token's queries or keys.
struct Unit {
    int64_t token;
    int32_t h0, h1;
};
__device__ __forceinline__ Unit unit_at(const HeadNormArgs &a, int which, int64_t u)
{
    // (tokens in parts are few)
    Unit q = {u, 0, a.heads[which]};
    if (a.parts[which] == 1) return q;
    q.token = int(u) / a.parts[which];
    const int part = int(u) % a.parts[which];
    q.h0 = part * a.per_part[which];
    q.h1 = min(a.heads[which], q.h0 + a.per_part[which]);
    return q;
}

template <int BYTES>
__device__ __forceinline__ void copy_ahead(void *to, const void *from)
{
    const uint32_t at = uint32_t(__cvta_generic_to_shared(to));
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(at), "l"(from) : "memory");
}

// The angles of four pairs: cosines, sines and their negatives.
struct Turn {
    float2 c[2], s[2], n[2];
};
// Turns four pairs: halves of pairs in v[0..1] and v[2..3], or neighbours.
__device__ __forceinline__ void turn(float2 (&v)[4], const Turn &t, bool interleaved)
{
    if (!interleaved) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float2 e = v[k], f = v[k + 2];
            v[k] = __ffma2_rn(e, t.c[k], __fmul2_rn(f, t.n[k]));
            v[k + 2] = __ffma2_rn(e, t.s[k], __fmul2_rn(f, t.c[k]));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float c = k & 1 ? t.c[k / 2].y : t.c[k / 2].x, s = k & 1 ? t.s[k / 2].y : t.s[k / 2].x;
            const float n = k & 1 ? t.n[k / 2].y : t.n[k / 2].x;
            v[k] = __ffma2_rn(make_float2(v[k].y, v[k].x), make_float2(n, s), __fmul2_rn(v[k], twice(c)));
        }
    }
}

template <typename T>
__device__ __forceinline__ void unpack(const Vec<T, 4> &run, float2 *v)
{
    v[0] = pair_of(run.e);
    v[1] = pair_of(run.e + 2);
}

// Blocks of an SM: what registers (128 a thread for the gradient, or it spills) and rings leave room for.
template <typename T, bool GRAD>
constexpr int kResident = GRAD ? 2 : 3;
// chunks in a warp's ring
template <typename T, bool GRAD>
constexpr int kRing = GRAD && sizeof(T) == 4 ? 3 : 4;

// PLAIN: every lane of a group has elements, all of them turn, and the halves of pairs are apart, which
// most heads are: no branch between the heads of a chunk, so that their instructions mix.
template <typename T, int LANES, bool GRAD, bool PLAIN>
__global__ void __launch_bounds__(kThreads, kResident<T, GRAD>) head_norm_kernel(const __grid_constant__ HeadNormArgs a, const __grid_constant__ Turns<LANES * 4> turns)
{
    constexpr int kGroups = 32 / LANES;
    constexpr int kRuns = kUnroll * 2 * (GRAD ? 2 : 1), kAhead = kRing<T, GRAD>;
    using Run = Vec<T, 4>;
    extern __shared__ __align__(16) unsigned char dyn[];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, l = lane % LANES, group = lane / LANES;
    Run *const ring = reinterpret_cast<Run *>(dyn) + size_t(warp) * kAhead * kRuns * 32 + lane;
    const int which = int(blockIdx.x) >= a.blocks[0];
    const int block = int(blockIdx.x) - (which ? a.blocks[0] : 0);
    const bool mine = PLAIN || l * 8 < a.D, turned = PLAIN || l * 8 < a.rotary, interleaved = !PLAIN && a.interleaved;
    // first elements of the lane's two runs
    int at[2] = {8 * l, 8 * l + 4};
    if (turned && !interleaved) {
        at[0] = 4 * l;
        at[1] = a.rotary / 2 + 4 * l;
    }
    float2 w[4], dw[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        w[k] = twice(1.0f);
        if (mine && a.w[which]) {
            const T *p = static_cast<const T *>(a.w[which]) + at[k / 2] + k % 2 * 2;
            w[k] = make_float2(to_float(p[0]), to_float(p[1]));
        }
        dw[k] = twice(0.0f);
    }
    const float inverse = 1.0f / float(a.D);
    const T *const x0 = static_cast<const T *>(a.x[which]);
    const int heads = a.heads[which];
    // a warp's groups take neighbouring units, and stay together: past the last unit, they do it again
    // and write nothing
    const int64_t units = a.tokens * a.parts[which], step = int64_t(a.blocks[which]) * kWarps * kGroups;
    const int64_t first = (int64_t(block) * kWarps + warp) * kGroups;
    const int per_unit = (a.per_part[which] + kUnroll - 1) / kUnroll * kUnroll;
    auto unit = [&](int64_t u) { return unit_at(a, which, u + group < units ? u + group : units - 1); };

    // chunks on their way: the next one's unit, and the first of its heads
    int64_t next = first;
    int to_h = 0, to_n = 0, filled = 0;
    const T *from = nullptr, *from_dy = nullptr;  // the lane's runs in the unit's first head
    const int64_t apart = at[1] - at[0], head = a.head[which];
    auto start = [&] {
        if (next >= units) return;
        const Unit q = unit(next);
        to_h = 0;
        to_n = q.h1 - q.h0;
        from = x0 + q.token * a.token[which] + q.h0 * head + at[0];
        if (GRAD) from_dy = static_cast<const T *>(a.dy[which]) + (q.token * heads + q.h0) * a.D + at[0];
    };
    auto bring = [&] {
        if (next < units) {
            Run *const p = ring + filled * kRuns * 32;
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                // past the last head: the first again, whose products are not used
                const int h = to_h + i < to_n ? to_h + i : 0;
                if (mine) {
                    const T *const p0 = from + h * head;
                    copy_ahead<sizeof(Run)>(p + 2 * i * 32, p0);
                    copy_ahead<sizeof(Run)>(p + (2 * i + 1) * 32, p0 + apart);
                    if (GRAD) {
                        const T *const p1 = from_dy + h * a.D;
                        copy_ahead<sizeof(Run)>(p + (2 * (kUnroll + i)) * 32, p1);
                        copy_ahead<sizeof(Run)>(p + (2 * (kUnroll + i) + 1) * 32, p1 + apart);
                    }
                }
            }
            filled = (filled + 1) % kAhead;
            to_h += kUnroll;
            if (to_h >= per_unit) {
                next += step;
                start();
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    start();
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i) bring();

    int used = 0;
    int64_t position = first < units ? a.positions[unit(first).token] : 0;
    for (int64_t u = first; u < units; u += step) {
        const Unit q = unit(u);
        const int count = u + group < units ? q.h1 - q.h0 : 0;
        Turn angles;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float2 c = twice(1.0f), s = twice(0.0f);
            if (turned) {
                const int i = 4 * l + 2 * j;
                angle(turns, position, i, c.x, s.x);
                angle(turns, position, i + 1, c.y, s.y);
            }
            const float2 n = make_float2(-s.x, -s.y);
            angles.c[j] = c;  // the gradient's turn back
            angles.s[j] = GRAD ? n : s;
            angles.n[j] = GRAD ? s : n;
        }
        if (u + step < units) position = a.positions[unit(u + step).token];
        T *y = static_cast<T *>(a.y[which]) + (q.token * heads + q.h0) * a.D + at[0];
        for (int h0 = 0; h0 < per_unit; h0 += kUnroll) {
            bring();
            asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
            const Run *const p = ring + used * kRuns * 32;
            used = (used + 1) % kAhead;
            float2 v[kUnroll][4], d[GRAD ? kUnroll : 1][4], g[GRAD ? kUnroll : 1][4];
            float sum[kUnroll], dot[kUnroll];
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                unpack(p[2 * i * 32], v[i]);
                unpack(p[(2 * i + 1) * 32], v[i] + 2);
                if constexpr (GRAD) {
                    unpack(p[2 * (kUnroll + i) * 32], d[i]);
                    unpack(p[(2 * (kUnroll + i) + 1) * 32], d[i] + 2);
                }
                if (!mine)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        v[i][k] = twice(0.0f);
                        if (GRAD) d[i][k] = twice(0.0f);
                    }
                float2 square = __fmul2_rn(v[i][0], v[i][0]), along = twice(0.0f);
#pragma unroll
                for (int k = 1; k < 4; ++k) square = __ffma2_rn(v[i][k], v[i][k], square);
                if constexpr (GRAD) {
                    if (turned) turn(d[i], angles, interleaved);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        g[i][k] = __fmul2_rn(d[i][k], w[k]);
                        along = __ffma2_rn(g[i][k], v[i][k], along);
                    }
                }
                sum[i] = square.x + square.y;
                dot[i] = along.x + along.y;
            }
#pragma unroll
            for (int o = LANES / 2; o > 0; o /= 2)
#pragma unroll
                for (int i = 0; i < kUnroll; ++i) {
                    sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
                    if (GRAD) dot[i] += __shfl_xor_sync(0xffffffffu, dot[i], o);
                }
#pragma unroll
            for (int i = 0; i < kUnroll; ++i) {
                const bool there = h0 + i < count;
                const float rstd = a.norm ? rsqrtf(sum[i] * inverse + a.eps) : 1.0f;
                float2 out[4];
                if constexpr (GRAD) {
                    const float2 r = twice(rstd), back = twice(-dot[i] * inverse * rstd * rstd);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const float2 n = __fmul2_rn(v[i][k], r);
                        if (there) dw[k] = __ffma2_rn(d[i][k], n, dw[k]);
                        // (without a norm x is not read: zero times an infinity would be)
                        out[k] = __fmul2_rn(g[i][k], r);
                        if (a.norm) out[k] = __ffma2_rn(n, back, out[k]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k) out[k] = __fmul2_rn(__fmul2_rn(v[i][k], twice(rstd)), w[k]);
                    if (turned) turn(out, angles, interleaved);
                }
                if (mine && there) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        Run e;
                        put_pair(e.e, out[2 * k]);
                        put_pair(e.e + 2, out[2 * k + 1]);
                        *reinterpret_cast<Run *>(y + (k ? apart : 0)) = e;
                    }
                }
                y += a.D;
            }
        }
    }
    if (GRAD && a.partial) {
        // lanes of the block that hold the same elements, in a fixed order; then the block's row
        __shared__ float sums[kWarps][DC_HEAD_NORM_DIM_MAX];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int o = LANES; o < 32; o *= 2) {
                dw[k].x += __shfl_xor_sync(0xffffffffu, dw[k].x, o);
                dw[k].y += __shfl_xor_sync(0xffffffffu, dw[k].y, o);
            }
        if (lane < LANES && mine)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                sums[warp][at[k / 2] + k % 2 * 2] = dw[k].x;
                sums[warp][at[k / 2] + k % 2 * 2 + 1] = dw[k].y;
            }
        __syncthreads();
        for (int e = threadIdx.x; e < a.D; e += kThreads) {
            float t = 0.0f;
#pragma unroll
            for (int r = 0; r < kWarps; ++r) t += sums[r][e];
            a.partial[int64_t(blockIdx.x) * a.D + e] = t;
        }
    }
}

// Sizes and strides of any kind: a warp per head, four pairs a lane, one element an access. Pairs
// from rotary / 2 on are neighbours that do not turn; the last may be a single element.
template <typename T, bool GRAD, int N>
__global__ void __launch_bounds__(kThreads) head_norm_any_kernel(const __grid_constant__ HeadNormArgs a,
                                                                 const __grid_constant__ Turns<N> turns)
{
    constexpr int kPairs = DC_HEAD_NORM_DIM_MAX / 2 / 32;
    const int lane = threadIdx.x % 32, half = a.rotary / 2;
    int e[kPairs][2];  // the pairs' elements; D and above: none
    float w[kPairs][2], dw[kPairs][2] = {};
    const int which = int(blockIdx.x) >= a.blocks[0], heads = a.heads[which];
    const int block = int(blockIdx.x) - (which ? a.blocks[0] : 0);
#pragma unroll
    for (int j = 0; j < kPairs; ++j) {
        const int p = lane + 32 * j;
        e[j][0] = p >= half || a.interleaved ? 2 * p : p;
        e[j][1] = p >= half || a.interleaved ? 2 * p + 1 : p + half;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            w[j][k] = e[j][k] < a.D && a.w[which] ? to_float(static_cast<const T *>(a.w[which])[e[j][k]]) : 1.0f;
    }
    const float inverse = 1.0f / float(a.D);
    const int64_t units = a.tokens * a.parts[which], step = int64_t(a.blocks[which]) * kWarps;
    for (int64_t u = int64_t(block) * kWarps + threadIdx.x / 32; u < units; u += step) {
        const Unit q = unit_at(a, which, u);
        float c[kPairs], s[kPairs];
        const int64_t position = a.positions[q.token];
#pragma unroll
        for (int j = 0; j < kPairs; ++j) {
            c[j] = 1.0f;
            s[j] = 0.0f;
            if (lane + 32 * j < half) angle(turns, position, lane + 32 * j, c[j], s[j]);
        }
        for (int h = q.h0; h < q.h1; ++h) {
            const T *x = static_cast<const T *>(a.x[which]) + q.token * a.token[which] + h * a.head[which];
            const int64_t row = (q.token * heads + h) * a.D;
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
                    // (a turn by nothing is none: zero times an infinity would reach the neighbour)
                    if (lane + 32 * j >= half) continue;
                    const float p = t[j][0], r = t[j][1];
                    t[j][0] = p * c[j] - sign * r * s[j];
                    t[j][1] = r * c[j] + sign * p * s[j];
                }
            };
            if (GRAD) {
                turn(d, -1.0f);
#pragma unroll
                for (int j = 0; j < kPairs; ++j)
#pragma unroll
                    for (int k = 0; k < 2; ++k) along += d[j][k] * w[j][k] * v[j][k];
            }
            float rstd = 1.0f;
            if (a.norm) {
#pragma unroll
                for (int o = 16; o > 0; o /= 2) {
                    square += __shfl_xor_sync(0xffffffffu, square, o);
                    if (GRAD) along += __shfl_xor_sync(0xffffffffu, along, o);
                }
                rstd = rsqrtf(square * inverse + a.eps);
            }
            float out[kPairs][2];
            const float back = along * inverse * rstd * rstd;
#pragma unroll
            for (int j = 0; j < kPairs; ++j)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if (GRAD) {
                        dw[j][k] += d[j][k] * (v[j][k] * rstd);
                        out[j][k] = a.norm ? rstd * (d[j][k] * w[j][k] - v[j][k] * back) : d[j][k] * w[j][k];
                    } else {
                        out[j][k] = v[j][k] * rstd * w[j][k];
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
        __shared__ float sums[kWarps][DC_HEAD_NORM_DIM_MAX];
#pragma unroll
        for (int j = 0; j < kPairs; ++j)
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (e[j][k] < a.D) sums[threadIdx.x / 32][e[j][k]] = dw[j][k];
        __syncthreads();
        for (int at = threadIdx.x; at < a.D; at += kThreads) {
            float t = 0.0f;
#pragma unroll
            for (int r = 0; r < kWarps; ++r) t += sums[r][at];
            a.partial[int64_t(blockIdx.x) * a.D + at] = t;
        }
    }
}

// dw of both weights from the blocks' rows, in a fixed order: 32 elements a block, a warp every
// 32nd row.
__global__ void __launch_bounds__(1024)
weight_sums_kernel(const float *partial, int q_blocks, int k_blocks, int D, float *dw_q, float *dw_k)
{
    __shared__ float sums[32][33];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, e = blockIdx.x * 32 + lane;
    float *const out = blockIdx.y ? dw_k : dw_q;
    const int first = blockIdx.y ? q_blocks : 0, end = blockIdx.y ? q_blocks + k_blocks : q_blocks;
    float t = 0.0f;
    if (e < D)
#pragma unroll 8
        for (int b = first + warp; b < end; b += 32) t += partial[int64_t(b) * D + e];
    sums[warp][lane] = t;
    __syncthreads();
    t = sums[lane][warp];
#pragma unroll
    for (int o = 16; o > 0; o /= 2) t += __shfl_xor_sync(0xffffffffu, t, o);
    const int at = blockIdx.x * 32 + warp;
    if (lane == 0 && at < D && out) out[at] = t;
}

constexpr int kMostBlocks = 4 * 160;  // rows that the weights' gradients may have

template <typename T, int LANES, bool GRAD, bool PLAIN>
cudaError_t launch_runs(const HeadNormArgs &a, const AllTurns &turns, cudaStream_t stream)
{
    constexpr int smem = kWarps * kRing<T, GRAD> * kUnroll * 2 * (GRAD ? 2 : 1) * 32 * int(sizeof(Vec<T, 4>));
    auto kernel = head_norm_kernel<T, LANES, GRAD, PLAIN>;
    static DeviceCache cache;
    int ready = 0;
    const cudaError_t e = cache.get(ready, [&](int &v) {
        v = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    });
    if (e != cudaSuccess) return e;
    kernel<<<a.blocks[0] + a.blocks[1], kThreads, smem, stream>>>(a, first_turns<LANES * 4>(turns));
    return cudaGetLastError();
}

template <typename T, bool GRAD>
cudaError_t launch(HeadNormArgs a, const AllTurns &turns, bool runs, cudaStream_t stream)
{
    int sms = 0;
    cudaError_t e = sm_count(sms);
    if (e != cudaSuccess) return e;
    // Few tokens: heads are dealt to warps as finely as needed to fill the SMs. Many: the blocks that
    // fit at a time, by the shares of queries and keys.
    const int lanes = a.D <= 64 ? 8 : a.D <= 128 ? 16 : 32, least = runs ? kUnroll : 1;
    const int units = kWarps * (runs ? 32 / lanes : 1);  // of a block at a time
    int most = sms * (runs ? kResident<T, GRAD> : 4);
    if (most > kMostBlocks) most = kMostBlocks;
    int64_t blocks[2];
    for (int i = 0; i < 2; ++i) {
        const HeadParts p = head_parts(a.tokens, a.heads[i], int64_t(sms) * units, least);
        a.parts[i] = p.parts;
        a.per_part[i] = p.per_part;
        blocks[i] = (a.tokens * a.parts[i] + units - 1) / units;
    }
    if (blocks[0] + blocks[1] > most) {
        int64_t q = int64_t(most) * a.heads[0] / (a.heads[0] + a.heads[1]);
        q = q < 1 ? 1 : q > most - 1 ? most - 1 : q;
        if (blocks[0] < q) q = blocks[0];
        const int64_t k = most - q;
        blocks[0] = q;
        if (blocks[1] > k) blocks[1] = k;
    }
    a.blocks[0] = int(blocks[0]);
    a.blocks[1] = int(blocks[1]);
    if (!runs) {
        const int grid = a.blocks[0] + a.blocks[1];
        if (a.rotary <= 128)
            head_norm_any_kernel<T, GRAD, 64><<<grid, kThreads, 0, stream>>>(a, first_turns<64>(turns));
        else
            head_norm_any_kernel<T, GRAD, 128><<<grid, kThreads, 0, stream>>>(a, turns);
        e = cudaGetLastError();
    } else {
        auto go = [&](auto plain) {
            constexpr bool kPlain = decltype(plain)::value;
            return lanes == 8    ? launch_runs<T, 8, GRAD, kPlain>(a, turns, stream)
                   : lanes == 16 ? launch_runs<T, 16, GRAD, kPlain>(a, turns, stream)
                                 : launch_runs<T, 32, GRAD, kPlain>(a, turns, stream);
        };
        e = a.D == 8 * lanes && a.rotary == a.D && !a.interleaved ? go(std::true_type()) : go(std::false_type());
    }
    if (e != cudaSuccess || !GRAD || !a.partial) return e;
    weight_sums_kernel<<<dim3((a.D + 31) / 32, 2), 1024, 0, stream>>>(a.partial, a.blocks[0], a.blocks[1], a.D, a.dw[0],
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

size_t head_norm_workspace(int D) { return sizeof(float) * size_t(D) * kMostBlocks; }

cudaError_t launch_head_norm(int dtype, const HeadNormArgs &a, const AllTurns &turns, cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, return (launch<T, false>(a, turns, in_runs(dtype, a, false), stream));)
}

cudaError_t launch_head_norm_grad(int dtype, const HeadNormArgs &a, const AllTurns &turns, cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, return (launch<T, true>(a, turns, in_runs(dtype, a, true), stream));)
}

}  // namespace dc
