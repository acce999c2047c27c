// The norm after a block, its gate, dropout and scaled residual, and the norm before the
// next block, in one pass over the rows; and the gradient of all of it.
//
// A block takes a contiguous run of rows, one at a time, 4, 8 or 16 elements a thread. Every row is read
// once and written once: bulk copies bring the next rows into a ring in shared memory while
// one is worked on, so that the latency of memory and the two sums of a row (four for the
// layer norm, whose mean is taken first: sums of squares of centred values lose nothing to
// cancellation) overlap. Rows off 16-byte boundaries come with the bytes around them (the arrays'
// first and last rows, where those would lie outside, are loaded by the threads). Above kWideD
// columns such rows, and any that are too long for the ring, are loaded straight into registers. The gradient computes the statistics again
// from the same rows and adds up the gradients of weights and gates in registers; what
// several runs share is written out per run and added in a fixed order by a second kernel.
//
// Measured (one GB300): 32,768 x 2,048 bfloat16, rms, dropout, a gate per 2,048 rows: 94 us, 5.7 TB/s,
// integer and floating issue 65 % busy (34 instructions an element; the generator's draws are
// eight of them). Gradient, 32,765 x 4,096 half, layer norm, dropout, one gate: 358 us, 4.5 TB/s, at 54 % of
// the issue slots with the 16 warps an SM that the sums in registers leave room for. One row
// of 2,048: 3.2 us in a graph.
#pragma once

#include "blackwell.cuh"
#include "layers.cuh"

namespace dc {
namespace norms {

// Elements of a row per thread (EL): 16, which spreads a row's sums over few shuffles, and
// for rows of up to 128 and 256 columns, that one warp takes, 4 and 8, so that its lanes
// have work.
constexpr int kElems = 16;
// Rows above this take blocks of 512 threads, with a ring of rows where there is room for two,
// and above twice this of 1,024. The three sums of the gradient of both norms do not fit the registers
// everywhere (bytes spilled a thread, bfloat16 and float): up to kWideD columns 0-32 and 12-220 with long gates,
// 4-240 and 136-500 with short ones; single warps, 64 registers, 4-188 and 12-460, off 16-byte
// boundaries 88-668; blocks of 512 with a ring 16-244 and 200-484; 1,024 threads, 64 registers,
// 752-1,752.
constexpr int kNarrow = 256, kWideD = kNarrow * kElems;
constexpr int elems_for(int D, bool vec)  // vec: rows on 16-byte boundaries
{
    // Without, an element takes a register of its own: 16 of three rows spill.
    return D > kWideD ? kElems : D <= 128 ? 4 : D <= 256 || !vec ? 8 : kElems;
}

struct Team {
    int size;  // threads
    int lane;
    int warps;
    float *buf;  // [2][4][32] shared
    int phase;

    // Sums of up to four values over the block, to every thread. Lanes halve the values
    // they carry as they add: four values cost one shuffle more than one.
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N])
    {
        static_assert(N >= 1 && N <= 4, "");
        constexpr uint32_t kAll = 0xffffffffu;
        const int l = lane & 31;
        float x;
        if (N > 2) {
            const bool hi = l & 16;
            const float send0 = hi ? v[0] : v[2], send1 = hi ? v[1] : (N > 3 ? v[3 % N] : 0.0f);
            const float a0 = (hi ? v[2] : v[0]) + __shfl_xor_sync(kAll, send0, 16);
            const float a1 = (hi ? (N > 3 ? v[3 % N] : 0.0f) : v[1]) + __shfl_xor_sync(kAll, send1, 16);
            const bool odd = l & 8;
            x = (odd ? a1 : a0) + __shfl_xor_sync(kAll, odd ? a0 : a1, 8);
        } else if (N == 2) {
            const bool hi = l & 16;
            x = (hi ? v[1] : v[0]) + __shfl_xor_sync(kAll, hi ? v[0] : v[1], 16);
            x += __shfl_xor_sync(kAll, x, 8);
        } else {
            x = v[0] + __shfl_xor_sync(kAll, v[0], 16);
            x += __shfl_xor_sync(kAll, x, 8);
        }
        x += __shfl_xor_sync(kAll, x, 4);
        x += __shfl_xor_sync(kAll, x, 2);
        x += __shfl_xor_sync(kAll, x, 1);
        // value i is in lanes 8 i .. 8 i + 7 (N > 2), 16 i .. (N == 2), or all
        constexpr int kSpan = N > 2 ? 8 : N == 2 ? 16 : 32;
        if (warps == 1) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = __shfl_sync(kAll, x, i * kSpan);
            return;
        }
        float *b = buf + phase * (4 * 32);
        phase ^= 1;
        if (l % kSpan == 0 && l / kSpan < N) b[(lane >> 5) * N + l / kSpan] = x;
        __syncthreads();
        // lane l adds the entries l, l + step, ..: step is a multiple of N, so they are all
        // of value l % N
        constexpr int kStep = N == 3 ? 24 : 32;
        x = 0.0f;
        if (l < kStep)
            for (int i = l; i < warps * N; i += kStep) x += b[i];
        if (N == 3) {
            x += __shfl_down_sync(kAll, x, 12);
            x += __shfl_down_sync(kAll, x, 6);
            x += __shfl_down_sync(kAll, x, 3);
        } else {
#pragma unroll
            for (int o = 16; o >= N; o >>= 1) x += __shfl_down_sync(kAll, x, o);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __shfl_sync(kAll, x, i);
    }
};

// Rows on their way: A arrays' rows r, r + 1, ... in `stages` slots of shared memory, taken in
// turn. A row's slot is filled again (fetch_next) once every thread is past that row, which a
// later barrier shows. Rows that start off 16-byte boundaries (SHIFTED) come with the bytes around them
// up to the next boundaries; where those would lie outside the array, the row is not copied.
template <typename T, int A, bool SHIFTED>
struct Ring {
    const T *src[A];
    unsigned char *mem;
    uint64_t *bars;
    int stages, D;
    int64_t first, end, rows;
    uint32_t *gave_up;
    int slot, phase;        // of the row in hand: advance() moves to the next
    int fill;               // slot of the next row to fetch, and that row (one thread)
    int64_t next;

    static __host__ __device__ size_t slot_bytes(int D)
    {
        return (size_t(D) * sizeof(T) + 15) / 16 * 16 + (SHIFTED ? 16 : 0);
    }
    // by integers: arrays that a call does without are NULL, and arithmetic on such a pointer
    // would let the compiler take it for a valid one
    __device__ __forceinline__ uintptr_t address(int a, int64_t r) const
    {
        return reinterpret_cast<uintptr_t>(src[a]) + uintptr_t(r) * uintptr_t(D) * sizeof(T);
    }
    __device__ __forceinline__ bool copied(int64_t r) const
    {
        bool ok = true;
        if (SHIFTED) {
#pragma unroll
            for (int a = 0; a < A; ++a)
                ok = ok && (!src[a] || ((address(a, r) & ~uintptr_t(15)) >= address(a, 0) &&
                                        ((address(a, r + 1) + 15) & ~uintptr_t(15)) <= address(a, rows)));
        }
        return ok;
    }
    __device__ __forceinline__ unsigned char *place(int slot, int a) const
    {
        return mem + uint32_t(slot * A + a) * uint32_t(slot_bytes(D));
    }
    __device__ __forceinline__ const T *at(int64_t r, int a) const  // the row in hand
    {
        return reinterpret_cast<const T *>(place(slot, a) + (SHIFTED ? address(a, r) & 15 : 0));
    }
    __device__ __forceinline__ void fetch_next()  // one thread
    {
        const int64_t r = next++;
        const uint32_t bar = bw::smem_addr(bars + fill);
        const int to = fill;
        if (++fill == stages) fill = 0;
        if (r >= end || *gave_up) return;
        if (!copied(r)) {
            bw::bar_arrive(bar);
            return;
        }
        auto bytes = [&](int a) {
            return uint32_t(((address(a, r + 1) + 15) & ~uintptr_t(15)) - (address(a, r) & ~uintptr_t(15)));
        };
        uint32_t all = 0;
#pragma unroll
        for (int a = 0; a < A; ++a)
            if (src[a]) all += bytes(a);
        bw::bar_arrive_bytes(bar, all);
#pragma unroll
        for (int a = 0; a < A; ++a)
            if (src[a])
                bw::copy_bytes(bw::smem_addr(place(to, a)), reinterpret_cast<const void *>(address(a, r) & ~uintptr_t(15)),
                               bytes(a), bar);
    }
    __device__ __forceinline__ void start()
    {
        slot = phase = fill = 0;
        next = first;
        if (threadIdx.x == 0) {
            *gave_up = 0;
            for (int i = 0; i < stages; ++i) bw::bar_init(bw::smem_addr(bars + i), 1);
            bw::bar_init_fence();
            for (int i = 0; i < stages; ++i) fetch_next();
        }
        __syncthreads();
    }
    // whether row r, the one in hand, is in its slot; otherwise it is to be read from memory
    __device__ __forceinline__ bool wait(int64_t r)
    {
        return bw::bar_wait(bw::smem_addr(bars + slot), uint32_t(phase), gave_up) && copied(r);
    }
    __device__ __forceinline__ void advance()
    {
        if (++slot == stages) {
            slot = 0;
            phase ^= 1;
        }
    }
};
constexpr int kMaxStages = 4;

// A thread's 16 elements of a row: V neighbours, then the same `size` groups on. Elements
// past D read as zero. FULL: there are none.
template <typename T, int V, bool FULL, int EL>
struct Row {
    static constexpr int kItems = EL / V;
    Vec<T, V> e[kItems];

    static __device__ __forceinline__ int column(int k, int lane, int size)
    {
        return ((k / V) * size + lane) * V + k % V;
    }
    static __device__ __forceinline__ bool inside(int k, int D, int lane, int size)
    {
        return FULL || column(k, lane, size) < D;
    }
    __device__ __forceinline__ void fill(float v)
    {
#pragma unroll
        for (int i = 0; i < (EL / 2); ++i) set(i, twice(v));
    }
    __device__ __forceinline__ void load(const T *p, int D, int lane, int size)
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            if (inside(i * V, D, lane, size))
                e[i] = *reinterpret_cast<const Vec<T, V> *>(p + column(i * V, lane, size));
            else
#pragma unroll
                for (int j = 0; j < V; ++j) e[i].e[j] = from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void load_or_ones(const void *p, int D, int lane, int size)
    {
        if (p)
            load(static_cast<const T *>(p), D, lane, size);
        else
            fill(1.0f);
    }
    // pairs of elements 2 i, 2 i + 1
    __device__ __forceinline__ float2 get(int i) const
    {
        if (V == 1) return make_float2(to_float(e[2 * i].e[0]), to_float(e[2 * i + 1].e[0]));
        return pair_of(&e[2 * i / V].e[V == 1 ? 0 : 2 * i % V]);
    }
    __device__ __forceinline__ void set(int i, float2 v)
    {
        if (V == 1) {
            e[2 * i].e[0] = from_float<T>(v.x);
            e[2 * i + 1].e[0] = from_float<T>(v.y);
        } else {
            put_pair(&e[2 * i / V].e[V == 1 ? 0 : 2 * i % V], v);
        }
    }
    // a pair with its elements past D at zero
    static __device__ __forceinline__ float2 only_inside(float2 v, int i, int D, int lane, int size)
    {
        if (!inside(2 * i, D, lane, size)) v.x = 0.0f;
        if (!inside(2 * i + 1, D, lane, size)) v.y = 0.0f;
        return v;
    }
    __device__ __forceinline__ void store(T *p, int D, int lane, int size) const
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i)
            if (inside(i * V, D, lane, size))
                *reinterpret_cast<Vec<T, V> *>(p + column(i * V, lane, size)) = e[i];
    }
};

// Zeros in place of this thread's dropped elements of row `row`.
template <int V, int EL>
__device__ __forceinline__ void drop_row(const DropRule &d, float2 (&v)[(EL / 2)], int64_t row, int D,
                                         int lane, int size)
{
    if (d.threshold == 0) return;
    const uint32_t limit = (d.threshold << 16) - 1u;  // see kept()
    const uint64_t z0 = d.seed + (uint64_t(d.offset + row * ((D + 3) / 4)) + 1u) * kGamma;
    if (V >= 4) {
        const uint64_t z1 = z0 + uint64_t(lane * (V / 4)) * kGamma;
        const uint64_t step = uint64_t(size * (V / 4)) * kGamma;
#pragma unroll
        for (int k = 0; k < EL; k += 4) {
            const uint64_t w = splitmix_output(z1 + (k / V) * step + (k % V / 4) * kGamma);
            const uint32_t lo = uint32_t(w), hi = uint32_t(w >> 32);
            if (!(lo << 16 > limit)) v[k / 2].x = 0.0f;
            if (!(lo > limit)) v[k / 2].y = 0.0f;
            if (!(hi << 16 > limit)) v[k / 2 + 1].x = 0.0f;
            if (!(hi > limit)) v[k / 2 + 1].y = 0.0f;
        }
    } else {
#pragma unroll
        for (int k = 0; k < EL; k += 4) {
            // Four neighbouring lanes want the four fields of one draw, for each k: every lane
            // draws for one of four k, and they pass them round.
            const int c = ((k + (lane & 3)) * size + (lane & ~3)) / 4;
            const uint64_t w = splitmix_output(z0 + uint64_t(c) * kGamma);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t lo = __shfl_sync(0xffffffffu, uint32_t(w), j, 4);
                const uint32_t hi = __shfl_sync(0xffffffffu, uint32_t(w >> 32), j, 4);
                const uint32_t x = lane & 2 ? hi : lo;
                if (!((lane & 1 ? x : x << 16) > limit)) (j & 1 ? v[(k + j) / 2].y : v[(k + j) / 2].x) = 0.0f;
            }
        }
    }
}

// Run b of P holds rows [rows b / P, rows (b+1) / P).
__host__ __device__ inline int64_t run_start(int64_t rows, int64_t P, int64_t b)
{
    return rows * b / P;
}

// A thread's own floats in shared memory: pairs i and i + 1 (i even) in one access.
struct Own {
    float4 *at;
    int size;

    __device__ __forceinline__ void put(int i, float2 a, float2 b) const
    {
        at[i / 2 * size] = make_float4(a.x, a.y, b.x, b.y);
    }
    __device__ __forceinline__ void get(int i, float2 (&v)[2]) const
    {
        const float4 q = at[i / 2 * size];
        v[0] = make_float2(q.x, q.y);
        v[1] = make_float2(q.z, q.w);
    }
};
constexpr int kOwn = 2;

// Gate rows of at least this many rows (LONG) are worked out once: gate * w_post * scale waits in
// shared memory. For the gradient one sum A of t * fhat then serves both the gate's
// gradient (w_post A) and, gate by gate, w_post's (gate A), which is added to the run's sums when
// the gate row changes. For shorter ones that costs more than it saves.
constexpr int kLongGate = 8;

// Resident blocks: 24 warps an SM, 32 with blocks of 512 threads. Two of those serve 8,192 x 5,120 in 96 us (layer norm) and x 3,001 in 88,
// one in 127 and 113 (x 8,192, whose blocks are full, 115 against 102).
template <typename T, int V, int FULL, bool HAS_F, bool HAS_H, bool LONG, bool RING, int MAXT, int EL>
__global__ void __launch_bounds__(MAXT, MAXT == kNarrow ? 3 : MAXT == 512 ? 2 : MAXT == 32 ? 32 : 1) norm_kernel(NormArgs a, int stages)
{
    using R = Row<T, V, (FULL > 0), EL>;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ float buf[2 * 4 * 32];
    __shared__ alignas(8) uint64_t bars[kMaxStages];
    __shared__ uint32_t gave_up;
    const int size = FULL > 1 ? FULL : int(blockDim.x), D = FULL > 1 ? FULL * EL : a.D, lane = threadIdx.x;
    Team team{size, lane, size / 32, buf, 0};
    const float inv = 1.0f / float(D);
    const int64_t r0 = run_start(a.rows, gridDim.x, blockIdx.x);
    const int64_t r1 = run_start(a.rows, gridDim.x, blockIdx.x + 1);
    const T *xp = static_cast<const T *>(a.x), *fp = static_cast<const T *>(a.f);
    const Own own_pre{reinterpret_cast<float4 *>(dyn) + lane, size};
    const Own own_post{own_pre.at + (EL / 4) * size, size};  // w_post * scale, LONG: times gate
    Ring<T, 2, V == 1> ring{{xp, fp}, dyn + kOwn * EL * size * sizeof(float), bars, stages, D, r0, r1, a.rows, &gave_up, 0, 0, 0, 0};
    if (RING) ring.start();
    R gate, post;
    if (HAS_H) {
        post.load_or_ones(a.w_pre, D, lane, size);
#pragma unroll
        for (int i = 0; i < (EL / 2); i += 2) own_pre.put(i, post.get(i), post.get(i + 1));
    }
    auto keep_post = [&] {
        post.load_or_ones(a.w_post, D, lane, size);
        auto v = [&](int i) {
            const float2 p = __fmul2_rn(post.get(i), twice(a.drop.scale));
            return LONG ? __fmul2_rn(p, gate.get(i)) : p;
        };
#pragma unroll
        for (int i = 0; i < (EL / 2); i += 2) own_post.put(i, v(i), v(i + 1));
    };
    if (HAS_F) {
        gate.fill(1.0f);
        keep_post();
    }
    int64_t g_end = r0;  // where the gate row in hand ends
    for (int64_t r = r0; r < r1; ++r) {
        if (HAS_F && a.gate && r >= g_end) {
            const int64_t g = r / a.rows_per_gate;
            g_end = (g + 1) * a.rows_per_gate;
            gate.load(static_cast<const T *>(a.gate) + g * D, D, lane, size);
            if (LONG) keep_post();
        }
        R x, f;
        const bool here = RING && ring.wait(r);
        x.load(here ? ring.at(r, 0) : xp + r * D, D, lane, size);
        if (HAS_F) f.load(here ? ring.at(r, 1) : fp + r * D, D, lane, size);
        bool refill = RING;
        auto taken = [&] {  // past a barrier: every thread has this row in registers
            if (refill && lane == 0) ring.fetch_next();
            refill = false;
        };
        if (RING && team.warps == 1) {
            __syncwarp();
            taken();
        }
        float2 y[(EL / 2)], w[2];
        auto centre = [&] {  // y - mean, and the reciprocal root of its mean square
            float s[1];
            if (a.layer) {
                float2 q = twice(0.0f);
#pragma unroll
                for (int i = 0; i < (EL / 2); ++i) q = __fadd2_rn(q, y[i]);
                s[0] = q.x + q.y;
                team.sum(s);
                taken();
                const float2 mean = twice(-s[0] * inv);
#pragma unroll
                for (int i = 0; i < (EL / 2); ++i)
                    y[i] = R::only_inside(__fadd2_rn(y[i], mean), i, D, lane, size);
            }
            float2 q = twice(0.0f);
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) q = __ffma2_rn(y[i], y[i], q);
            s[0] = q.x + q.y;
            team.sum(s);
            taken();
            return rsqrtf(s[0] * inv + a.eps);
        };
        if (HAS_F) {
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) y[i] = f.get(i);
            const float2 rstd = twice(centre()), alpha = twice(a.alpha);
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) {
                if (i % 2 == 0) own_post.get(i, w);
                y[i] = __fmul2_rn(__fmul2_rn(y[i], rstd), w[i % 2]);
                if (!LONG) y[i] = __fmul2_rn(y[i], gate.get(i));
            }
            drop_row<V, EL>(a.drop, y, r, D, lane, size);
            R o;
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) {
                y[i] = __ffma2_rn(alpha, x.get(i), y[i]);
                o.set(i, y[i]);
            }
            o.store(static_cast<T *>(a.y) + r * D, D, lane, size);
        } else {
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) y[i] = x.get(i);
        }
        if (HAS_H) {
            const float2 rstd = twice(centre());
            R o;
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) {
                if (i % 2 == 0) own_pre.get(i, w);
                o.set(i, __fmul2_rn(__fmul2_rn(y[i], rstd), w[i % 2]));
            }
            o.store(static_cast<T *>(a.h) + r * D, D, lane, size);
        }
        if (RING) ring.advance();
    }
    if (RING && gave_up)  // a copy is late: it still writes this block's memory
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

// ------------------------------------------------------------------------ gradient
// Per run: sums for w_post, w_pre, the gate row shared with the run before, the gate row
// shared with the run after.
constexpr int kSlots = 4;

template <typename T, int V, int FULL, bool HAS_F, bool HAS_H, bool LONG, bool RING, int MAXT, int EL>
__global__ void __launch_bounds__(MAXT, MAXT == kNarrow ? 2 : MAXT == 32 ? 32 : 1)
norm_grad_kernel(NormArgs a, float *partial, int stages)
{
    using R = Row<T, V, (FULL > 0), EL>;
    extern __shared__ __align__(16) unsigned char dyn[];
    __shared__ float buf[2 * 4 * 32];
    __shared__ alignas(8) uint64_t bars[kMaxStages];
    __shared__ uint32_t gave_up;
    const int size = FULL > 1 ? FULL : int(blockDim.x), D = FULL > 1 ? FULL * EL : a.D, lane = threadIdx.x;
    Team team{size, lane, size / 32, buf, 0};
    const float inv = 1.0f / float(D);
    const int64_t b = blockIdx.x, P = gridDim.x;
    const int64_t r0 = run_start(a.rows, P, b), r1 = run_start(a.rows, P, b + 1);
    const T *src[4] = {HAS_H ? static_cast<const T *>(a.x) : nullptr, static_cast<const T *>(a.dh),
                       static_cast<const T *>(a.dy), HAS_F ? static_cast<const T *>(a.f) : nullptr};
    // This thread's w_pre and (LONG) gate * w_post * scale as floats, four to an access: in
    // shared memory, where they cost no registers and no conversions.
    const Own own_pre{reinterpret_cast<float4 *>(dyn) + lane, size};
    const Own own_gp{own_pre.at + (EL / 4) * size, size};
    Ring<T, 4, V == 1> ring{{src[0], src[1], src[2], src[3]}, dyn + kOwn * EL * size * sizeof(float), bars, stages, D, r0, r1, a.rows, &gave_up, 0, 0, 0, 0};
    if (RING) ring.start();
    R post, gate;
    if (HAS_H) {
        post.load_or_ones(a.w_pre, D, lane, size);
#pragma unroll
        for (int i = 0; i < (EL / 2); i += 2) own_pre.put(i, post.get(i), post.get(i + 1));
    }
    if (HAS_F) {
        post.load_or_ones(a.w_post, D, lane, size);
        gate.fill(1.0f);
    }
    float2 gpre[(EL / 2)], gpost[(EL / 2)], ggate[(EL / 2)];  // LONG: ggate holds A, gpost is in memory
#pragma unroll
    for (int i = 0; i < (EL / 2); ++i) gpost[i] = gpre[i] = ggate[i] = twice(0.0f);
    float *slots = partial + b * int64_t(kSlots) * D;
    auto each = [&](auto &&op) {  // op(pair, half, column) of this thread's columns
#pragma unroll
        for (int i = 0; i < (EL / 2); ++i) {
            if (R::inside(2 * i, D, lane, size)) op(i, 0, R::column(2 * i, lane, size));
            if (R::inside(2 * i + 1, D, lane, size)) op(i, 1, R::column(2 * i + 1, lane, size));
        }
    };
    auto half = [](float2 v, int h) { return h ? v.y : v.x; };
    auto load_gate = [&](int64_t g) {
        if (a.gate) gate.load(static_cast<const T *>(a.gate) + g * D, D, lane, size);
        if (LONG) {
            post.load_or_ones(a.w_post, D, lane, size);
            auto gp = [&](int i) { return __fmul2_rn(__fmul2_rn(gate.get(i), post.get(i)), twice(a.drop.scale)); };
#pragma unroll
            for (int i = 0; i < (EL / 2); i += 2) own_gp.put(i, gp(i), gp(i + 1));
        }
    };
    int64_t g = 0, g_end = r0;
    bool first_gate = true;
    for (int64_t r = r0; r < r1; ++r) {
        if (HAS_F && r >= g_end) {
            g = r / a.rows_per_gate;
            g_end = (g + 1) * a.rows_per_gate;
            load_gate(g);
        }
        const bool here = RING && ring.wait(r);
        const T *in[4] = {nullptr, nullptr, nullptr, nullptr};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (src[i]) in[i] = here ? ring.at(r, i) : src[i] + r * D;
        if (RING) ring.advance();
        auto row = [&](int i) { return in[i]; };
        R y, f, dh;
        if (HAS_H) {
            y.load(row(0), D, lane, size);
            dh.load(row(1), D, lane, size);
        }
        if (HAS_F) f.load(row(3), D, lane, size);
        // Read again from the ring in each phase: the sums take most of the registers, and
        // rows held over the barriers would spill.
        auto reload = [&](bool with_y) {
            if (!RING) return;
            asm volatile("" ::: "memory");
            if (HAS_H && with_y) {
                y.load(row(0), D, lane, size);
                dh.load(row(1), D, lane, size);
            }
            if (HAS_F) f.load(row(3), D, lane, size);
        };

        // Statistics of y and f, and the sums of dn = dh * w_pre that n'(y)^T needs. The layer
        // norm's mean square about the mean comes from sums about the row's first element, in
        // the same pass; where that element lies more than two deviations from the mean, and
        // the difference would lose digits, the sums are taken again about the mean.
        float2 y0 = twice(0.0f), f0 = twice(0.0f);  // minus what the sums are about
        float s[4], w[2];                           // sums: y, y^2, f, f^2; dn, dn y
        float2 q[6];
        auto sums = [&] {
#pragma unroll
            for (int i = 0; i < 6; ++i) q[i] = twice(0.0f);
            float2 pre[2];
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) {
                if (HAS_H) {
                    if (i % 2 == 0) own_pre.get(i, pre);
                    const float2 v = R::only_inside(__fadd2_rn(y.get(i), y0), i, D, lane, size);
                    const float2 dn = __fmul2_rn(dh.get(i), pre[i % 2]);
                    q[1] = __ffma2_rn(v, v, q[1]);
                    q[5] = __ffma2_rn(dn, v, q[5]);
                    if (a.layer) {
                        q[0] = __fadd2_rn(q[0], v);
                        q[4] = __fadd2_rn(q[4], dn);
                    }
                }
                if (HAS_F) {
                    const float2 v = R::only_inside(__fadd2_rn(f.get(i), f0), i, D, lane, size);
                    q[3] = __ffma2_rn(v, v, q[3]);
                    if (a.layer) q[2] = __fadd2_rn(q[2], v);
                }
            }
            if (a.layer) {
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = q[i].x + q[i].y;
                w[0] = q[4].x + q[4].y;
                w[1] = q[5].x + q[5].y;
                if (HAS_H && HAS_F) {
                    team.sum(s);
                    if (HAS_H) team.sum(w);
                } else if (HAS_H) {
                    float v[4] = {s[0], s[1], w[0], w[1]};
                    team.sum(v);
                    s[0] = v[0], s[1] = v[1], w[0] = v[2], w[1] = v[3];
                } else {
                    float v[2] = {s[2], s[3]};
                    team.sum(v);
                    s[2] = v[0], s[3] = v[1];
                }
            } else {
                float v[3] = {q[1].x + q[1].y, q[3].x + q[3].y, q[5].x + q[5].y};
                team.sum(v);
                s[0] = s[2] = w[0] = 0.0f;
                s[1] = v[0], s[3] = v[1], w[1] = v[2];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] *= inv;
            w[0] *= inv;
            w[1] *= inv;
        };
        if (a.layer) {
            if (HAS_H) y0 = twice(-to_float(*row(0)));
            if (HAS_F) f0 = twice(-to_float(*row(3)));
        }
        sums();
        if (a.layer && (s[0] * s[0] > 0.8f * s[1] || s[2] * s[2] > 0.8f * s[3])) {
            y0.x -= s[0], y0.y = y0.x;
            f0.x -= s[2], f0.y = f0.x;
            reload(true);
            sums();
        }
        if (RING) {  // past a barrier of this row, so every thread is done with the row before
            __syncwarp();
            if (lane == 0 && r > r0) ring.fetch_next();
        }
        const float yr1 = HAS_H ? rsqrtf(fmaxf(s[1] - s[0] * s[0], 0.0f) + a.eps) : 0.0f;
        const float fr1 = HAS_F ? rsqrtf(fmaxf(s[3] - s[2] * s[2], 0.0f) + a.eps) : 0.0f;
        // yhat = (y + ym) yr; n'(y)^T dn = yr (dn + dm + yhat proj)
        const float2 yr = twice(yr1), ym = twice(y0.x - s[0]), dm = twice(-w[0]);
        const float2 proj = twice(-(w[1] - s[0] * w[0]) * yr1);
        const float2 fr = twice(fr1), fm = twice(f0.x - s[2]);

        reload(true);
        float2 t[(EL / 2)];
        if (a.dy) {
            R dy;
            dy.load(row(2), D, lane, size);
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) t[i] = dy.get(i);
        } else {
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) t[i] = twice(0.0f);
        }
        float2 w2[2];
        if (HAS_H) {
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) {
                if (i % 2 == 0) own_pre.get(i, w2);
                const float2 yhat = __fmul2_rn(__fadd2_rn(y.get(i), ym), yr), d = dh.get(i);
                t[i] = __ffma2_rn(yr, __ffma2_rn(yhat, proj, __ffma2_rn(d, w2[i % 2], dm)), t[i]);
                gpre[i] = __ffma2_rn(d, yhat, gpre[i]);
            }
        }
        R o;
        const float2 alpha = twice(a.alpha);
#pragma unroll
        for (int i = 0; i < (EL / 2); ++i) o.set(i, __fmul2_rn(alpha, t[i]));
        o.store(static_cast<T *>(a.dx) + r * D, D, lane, size);
        if (!HAS_F) continue;

        drop_row<V, EL>(a.drop, t, r, D, lane, size);
        const float2 scale = twice(a.drop.scale);
        float2 s2[2] = {twice(0.0f), twice(0.0f)};
#pragma unroll
        for (int i = 0; i < (EL / 2); ++i) {
            const float2 fhat = __fmul2_rn(__fadd2_rn(f.get(i), fm), fr);
            float2 kt = R::only_inside(t[i], i, D, lane, size);
            if (LONG) {
                if (i % 2 == 0) own_gp.get(i, w2);
                t[i] = __fmul2_rn(kt, w2[i % 2]);
                ggate[i] = __ffma2_rn(kt, fhat, ggate[i]);
            } else {
                kt = __fmul2_rn(kt, scale);
                const float2 u = __fmul2_rn(kt, gate.get(i)), p = post.get(i);
                t[i] = __fmul2_rn(u, p);
                ggate[i] = __ffma2_rn(__fmul2_rn(kt, p), fhat, ggate[i]);
                gpost[i] = __ffma2_rn(u, fhat, gpost[i]);
            }
            s2[0] = __ffma2_rn(t[i], fhat, s2[0]);
            s2[1] = __fadd2_rn(s2[1], t[i]);
        }
        float v[2] = {s2[0].x + s2[0].y, s2[1].x + s2[1].y};
        team.sum(v);
        reload(false);
        const float2 fproj = twice(-(v[0] * inv)), fdm = twice(a.layer ? -(v[1] * inv) : 0.0f);
#pragma unroll
        for (int i = 0; i < (EL / 2); ++i) {
            const float2 fhat = __fmul2_rn(__fadd2_rn(f.get(i), fm), fr);
            o.set(i, __fmul2_rn(fr, __ffma2_rn(fhat, fproj, __fadd2_rn(t[i], fdm))));
        }
        o.store(static_cast<T *>(a.df) + r * D, D, lane, size);

        // the gate row ends here, or this run does
        const bool ends = r + 1 == g_end || r + 1 == a.rows;
        if (ends || r + 1 == r1) {
            if (LONG) {
                post.load_or_ones(a.w_post, D, lane, size);
                if (a.gate) gate.load(static_cast<const T *>(a.gate) + g * D, D, lane, size);
                if (a.dw_post)
                    each([&](int i, int h, int c) {
                        const float v = half(gate.get(i), h) * half(ggate[i], h) * a.drop.scale;
                        slots[c] = first_gate ? v : slots[c] + v;
                    });
                first_gate = false;
#pragma unroll
                for (int i = 0; i < (EL / 2); ++i)
                    ggate[i] = __fmul2_rn(__fmul2_rn(post.get(i), scale), ggate[i]);
            }
            if (a.dgate) {
                const int64_t g_start = g * a.rows_per_gate;
                if (ends && g_start >= r0) {
#pragma unroll
                    for (int i = 0; i < (EL / 2); ++i) o.set(i, ggate[i]);
                    o.store(static_cast<T *>(a.dgate) + g * D, D, lane, size);
                } else {
                    float *p = slots + (g_start < r0 ? 2 : 3) * int64_t(D);
                    each([&](int i, int h, int c) { p[c] = half(ggate[i], h); });
                }
            }
#pragma unroll
            for (int i = 0; i < (EL / 2); ++i) ggate[i] = twice(0.0f);
        }
    }
    if (HAS_F && !LONG && a.dw_post) each([&](int i, int h, int c) { slots[c] = half(gpost[i], h); });
    if (HAS_H && a.dw_pre) each([&](int i, int h, int c) { slots[D + c] = half(gpre[i], h); });
    if (RING && gave_up)  // a copy is late: it still writes this block's memory
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}

// The run that holds row r.
__device__ __forceinline__ int64_t run_of(int64_t rows, int64_t P, int64_t r)
{
    int64_t b = r * P / rows;
    while (b + 1 < P && run_start(rows, P, b + 1) <= r) ++b;
    while (b > 0 && run_start(rows, P, b) > r) --b;
    return b;
}

// Adds the runs' sums: block row 0 those of the weights, block row g + 1 those of gate row g if
// it lies in several runs. Thirty-two threads a column, each every thirty-second run in order.
constexpr int kFinishCols = 32, kFinishLanes = 32;
template <typename T>
__global__ void __launch_bounds__(kFinishCols *kFinishLanes)
norm_finish_kernel(NormArgs a, const float *partial, int64_t P)
{
    __shared__ float part[2][kFinishLanes][kFinishCols];
    const int tx = threadIdx.x, ty = threadIdx.y;
    const int64_t c = int64_t(blockIdx.x) * kFinishCols + tx, D = a.D;
    const int64_t stride = kSlots * D, g = int64_t(blockIdx.y) - 1;
    const bool in = c < D;
    float s0 = 0.0f, s1 = 0.0f;
    if (g < 0) {
        if (in) {
            if (a.dw_post)
#pragma unroll 16
                for (int64_t i = ty; i < P; i += kFinishLanes) s0 += partial[i * stride + c];
            if (a.dw_pre)
#pragma unroll 16
                for (int64_t i = ty; i < P; i += kFinishLanes) s1 += partial[i * stride + D + c];
        }
    } else {
        const int64_t start = g * a.rows_per_gate;
        const int64_t end = start + a.rows_per_gate < a.rows ? start + a.rows_per_gate : a.rows;
        const int64_t b0 = run_of(a.rows, P, start), b1 = run_of(a.rows, P, end - 1);
        if (b0 == b1) return;  // written by its run; the whole block
        // run b0 holds the gate's first rows: shared with the run after
        if (in)
#pragma unroll 8
            for (int64_t i = b0 + ty; i <= b1; i += kFinishLanes)
                s0 += partial[i * stride + (i == b0 ? 3 : 2) * D + c];
    }
    part[0][ty][tx] = s0;
    part[1][ty][tx] = s1;
    __syncthreads();
    if (ty > 1 || !in) return;
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kFinishLanes; ++i) v += part[ty][i][tx];
    if (g < 0) {
        float *out = ty == 0 ? a.dw_post : a.dw_pre;
        if (out) out[c] = v;
    } else if (ty == 0) {
        static_cast<T *>(a.dgate)[g * D + c] = from_float<T>(v);
    }
}

// Gate rows of a few runs each: a thread per column adds a gate row's runs one after another.
constexpr int kGateThreads = 256, kGateSpan = 24;
template <typename T>
__global__ void __launch_bounds__(kGateThreads) norm_gates_kernel(NormArgs a, const float *partial, int64_t P)
{
    const int64_t g = blockIdx.x, D = a.D, c = int64_t(blockIdx.y) * blockDim.x + threadIdx.x;
    const int64_t start = g * a.rows_per_gate;
    const int64_t end = start + a.rows_per_gate < a.rows ? start + a.rows_per_gate : a.rows;
    const int64_t b0 = run_of(a.rows, P, start), b1 = run_of(a.rows, P, end - 1);
    if (b0 == b1 || c >= D) return;
    float v = partial[(b0 * kSlots + 3) * D + c];
#pragma unroll 4
    for (int64_t i = b0 + 1; i <= b1; ++i) v += partial[(i * kSlots + 2) * D + c];
    static_cast<T *>(a.dgate)[g * D + c] = from_float<T>(v);
}

// With more gate rows than runs, a gate row lies in at most two: one block per run adds the
// row that it shares with the run before.
template <typename T>
__global__ void __launch_bounds__(128) norm_shared_gates_kernel(NormArgs a, const float *partial, int64_t P)
{
    const int64_t b = int64_t(blockIdx.x) + 1, rb = run_start(a.rows, P, b);
    const int64_t g = rb / a.rows_per_gate, D = a.D;
    if (g * a.rows_per_gate == rb) return;
    const float *before = partial + ((b - 1) * kSlots + 3) * D, *after = partial + (b * kSlots + 2) * D;
    for (int64_t c = threadIdx.x; c < D; c += blockDim.x)
        static_cast<T *>(a.dgate)[g * D + c] = from_float<T>(before[c] + after[c]);
}

// ------------------------------------------------------------------------------ host
inline int row_threads(int D, bool vec)
{
    const int el = elems_for(D, vec);
    return (D + el * 32 - 1) / (el * 32) * 32;
}

// Blocks an SM and slots of the ring: `threads` an SM as the registers allow, and the 224 KB
// of shared memory shared between them; no ring (0 slots) where it would hold fewer than two rows.
struct Plan {
    int size, blocks, stages;
    size_t smem;
};
inline Plan plan_for(int D, bool vec, int arrays, int bytes, int threads, int own)
{
    Plan p;
    const int size = row_threads(D, vec), el = elems_for(D, vec);
    const bool one_warp = size == 32 && el < kElems;
    p.size = size;
    p.blocks = one_warp ? 32 : threads / size < 1 ? 1 : threads / size;
    if (p.blocks > 32) p.blocks = 32;
    if (!one_warp && p.blocks > 16) p.blocks = 16;
    const size_t fixed = 2048 + size_t(own) * size * el * sizeof(float);
    const size_t row = size_t(arrays) * ((size_t(D) * bytes + 15) / 16 * 16 + 16), room = size_t(224) << 10;
    while (p.blocks > 1 && room / p.blocks < 2 * row + fixed) --p.blocks;
    const size_t slots = room / p.blocks > fixed ? (room / p.blocks - fixed) / row : 0;
    p.stages = int(slots < kMaxStages ? slots : kMaxStages);
    // wide rows take a ring on 16-byte boundaries and in blocks of up to 512 threads only
    if (p.stages < 2 || (D > kWideD && (!vec || size > 512))) p.stages = 0;
    p.smem = p.stages * row + fixed - 2048;
    return p;
}
constexpr int kSms = 152;  // a constant, so that a workspace query needs no device
constexpr int kForwardThreads = 768, kGradThreads = 512;  // an SM; up to 32 single warps

inline int64_t grad_runs(int dtype, int64_t rows, int D, bool vec)
{
    const int64_t most = int64_t(kSms) * plan_for(D, vec, 4, dtype_bytes(dtype), kGradThreads, kOwn).blocks;
    return rows < most ? rows : most;
}

template <typename T, int V, int FULL, bool RING, int MAXT, int EL>
cudaError_t norm_launch(const NormArgs &a, const Plan &p, cudaStream_t stream)
{
    const bool lg = a.rows_per_gate >= kLongGate;
    auto kernel = a.f && a.h ? lg ? norm_kernel<T, V, FULL, true, true, true, RING, MAXT, EL>
                                  : norm_kernel<T, V, FULL, true, true, false, RING, MAXT, EL>
                  : a.f      ? norm_kernel<T, V, FULL, true, false, false, RING, MAXT, EL>
                             : norm_kernel<T, V, FULL, false, true, false, RING, MAXT, EL>;
    static DeviceCache cache[4];
    int ready = 0;
    const cudaError_t e = cache[a.f && a.h ? lg : a.f ? 2 : 3].get(ready, [&](int &v) {
        v = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 << 10);
    });
    if (e != cudaSuccess) return e;
    const int64_t most = int64_t(kSms) * p.blocks;
    kernel<<<unsigned(a.rows < most ? a.rows : most), unsigned(p.size), p.smem, stream>>>(
        a, p.stages);
    return cudaGetLastError();
}

template <typename T, int V, int FULL, bool RING, int MAXT, int EL>
cudaError_t norm_grad_launch(const NormArgs &a, float *partial, int64_t P, const Plan &p,
                             cudaStream_t stream)
{
    const bool lg = a.rows_per_gate >= kLongGate;
    auto kernel = a.f && a.dh ? lg ? norm_grad_kernel<T, V, FULL, true, true, true, RING, MAXT, EL>
                                   : norm_grad_kernel<T, V, FULL, true, true, false, RING, MAXT, EL>
                  : a.f       ? norm_grad_kernel<T, V, FULL, true, false, false, RING, MAXT, EL>
                              : norm_grad_kernel<T, V, FULL, false, true, false, RING, MAXT, EL>;
    static DeviceCache cache[4];
    {
        int ready = 0;
        const cudaError_t e = cache[a.f && a.dh ? lg : a.f ? 2 : 3].get(ready, [&](int &v) {
            v = 1;
            return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 << 10);
        });
        if (e != cudaSuccess) return e;
    }
    kernel<<<unsigned(P), unsigned(p.size), p.smem, stream>>>(a, partial, p.stages);
    const int64_t gates = (a.rows + a.rows_per_gate - 1) / a.rows_per_gate;
    // how the gate rows that lie in several runs are added up
    const bool shared = a.dgate && P > 1 && a.rows_per_gate > 1, few = gates < P;
    const bool wide = shared && few && a.rows_per_gate * P / a.rows > kGateSpan;
    if (a.dw_post || a.dw_pre || wide) {
        const dim3 g(unsigned((a.D + kFinishCols - 1) / kFinishCols), 1u + unsigned(wide ? gates : 0));
        norm_finish_kernel<T><<<g, dim3(kFinishCols, kFinishLanes), 0, stream>>>(a, partial, P);
    }
    if (shared && few && !wide) {
        const int n = a.D < kGateThreads ? (a.D + 31) / 32 * 32 : kGateThreads;
        norm_gates_kernel<T><<<dim3(unsigned(gates), unsigned((a.D + n - 1) / n)), n, 0, stream>>>(a, partial, P);
    }
    if (shared && !few) norm_shared_gates_kernel<T><<<unsigned(P - 1), 128, 0, stream>>>(a, partial, P);
    return cudaGetLastError();
}

inline bool vectors_ok(int dtype, const NormArgs &a)
{
    if (a.D % (16 / dtype_bytes(dtype))) return false;
    const void *p[] = {a.x, a.f, a.gate, a.w_post, a.w_pre, a.y, a.h, a.dy, a.dh, a.dx, a.df, a.dgate};
    for (const void *q : p)
        if (!aligned16(q)) return false;
    return true;
}

// Rows of up to kWideD columns always leave room for a ring of two rows.
template <typename T>
cudaError_t forward(int dtype, const NormArgs &a, cudaStream_t stream)
{
    const bool vec = vectors_ok(dtype, a), full = a.D % (kElems * 32) == 0;
    const Plan p = plan_for(a.D, vec, 2, dtype_bytes(dtype), kForwardThreads, kOwn);
    constexpr int V = kVec<T>;
    if (a.D > kWideD && p.stages)
        return norm_launch<T, V, 0, true, 512, kElems>(a, p, stream);
    if (a.D > kWideD)
        return vec ? norm_launch<T, V, 0, false, 1024, kElems>(a, p, stream)
                   : norm_launch<T, 1, 0, false, 1024, kElems>(a, p, stream);
    if (a.D <= 128)
        return vec ? norm_launch<T, 4, 0, true, 32, 4>(a, p, stream) : norm_launch<T, 1, 0, true, 32, 4>(a, p, stream);
    if (a.D <= 256)
        return vec ? norm_launch<T, V, 0, true, 32, 8>(a, p, stream) : norm_launch<T, 1, 0, true, 32, 8>(a, p, stream);
    if (!vec)
        return a.D <= 2048 ? norm_launch<T, 1, 0, true, kNarrow, 8>(a, p, stream) : norm_launch<T, 1, 0, true, 512, 8>(a, p, stream);
    // Powers of two, whose strides are then constants: layer norm of 32,768 x 4,096 205 us against
    // 229, 32,768 x 1,024 with short gates 51 against 57; but rms with long gates 102 against 95 (x 2,048)
    // and 190 against 177 (x 4,096), where the sums are fewest.
    const bool fixed = a.layer || a.rows_per_gate < kLongGate || a.D < 2048;
    switch (fixed ? a.D : 0) {
        case 512: return norm_launch<T, V, 32, true, kNarrow, kElems>(a, p, stream);
        case 1024: return norm_launch<T, V, 64, true, kNarrow, kElems>(a, p, stream);
        case 2048: return norm_launch<T, V, 128, true, kNarrow, kElems>(a, p, stream);
        case 4096: return norm_launch<T, V, 256, true, kNarrow, kElems>(a, p, stream);
        default: break;
    }
    return full ? norm_launch<T, V, 1, true, kNarrow, kElems>(a, p, stream)
                : norm_launch<T, V, 0, true, kNarrow, kElems>(a, p, stream);
}

template <typename T>
cudaError_t gradient(int dtype, const NormArgs &a, float *partial, cudaStream_t stream)
{
    const bool vec = vectors_ok(dtype, a), full = a.D % (kElems * 32) == 0;
    const Plan p = plan_for(a.D, vec, 4, dtype_bytes(dtype), kGradThreads, kOwn);
    const int64_t P = grad_runs(dtype, a.rows, a.D, vec);
    constexpr int V = kVec<T>;
    if (a.D > kWideD && p.stages)
        return norm_grad_launch<T, V, 0, true, 512, kElems>(a, partial, P, p, stream);
    if (a.D > kWideD)
        return vec ? norm_grad_launch<T, V, 0, false, 1024, kElems>(a, partial, P, p, stream)
                   : norm_grad_launch<T, 1, 0, false, 1024, kElems>(a, partial, P, p, stream);
    if (a.D <= 128)
        return vec ? norm_grad_launch<T, 4, 0, true, 32, 4>(a, partial, P, p, stream) : norm_grad_launch<T, 1, 0, true, 32, 4>(a, partial, P, p, stream);
    if (a.D <= 256)
        return vec ? norm_grad_launch<T, V, 0, true, 32, 8>(a, partial, P, p, stream) : norm_grad_launch<T, 1, 0, true, 32, 8>(a, partial, P, p, stream);
    if (!vec)
        return a.D <= 2048 ? norm_grad_launch<T, 1, 0, true, kNarrow, 8>(a, partial, P, p, stream) : norm_grad_launch<T, 1, 0, true, 512, 8>(a, partial, P, p, stream);
    switch (a.D) {  // as in forward: 32,765 x 4,096 layer norm 369 us against 405
        case 512: return norm_grad_launch<T, V, 32, true, kNarrow, kElems>(a, partial, P, p, stream);
        case 1024: return norm_grad_launch<T, V, 64, true, kNarrow, kElems>(a, partial, P, p, stream);
        case 2048: return norm_grad_launch<T, V, 128, true, kNarrow, kElems>(a, partial, P, p, stream);
        case 4096: return norm_grad_launch<T, V, 256, true, kNarrow, kElems>(a, partial, P, p, stream);
        default: break;
    }
    return full ? norm_grad_launch<T, V, 1, true, kNarrow, kElems>(a, partial, P, p, stream)
                : norm_grad_launch<T, V, 0, true, kNarrow, kElems>(a, partial, P, p, stream);
}

}  // namespace norms
}  // namespace dc
