// The norm after a block, its gate, dropout and scaled residual, and the norm before the
// next block, in one pass over the rows; and the gradient of all of it.
//
// A team of threads (a warp, or the whole block) takes a row and keeps it in registers, 16
// elements a thread, so every row is read once and written once: two sums over the row
// for the root mean square norm, four for the layer norm, whose mean is taken first (sums
// of squares of centred values lose nothing to cancellation). The gradient computes the
// statistics again from the same rows. A team of the gradient takes a contiguous run of rows
// and adds up the gradients of the weights and gates in registers; what several runs share
// is written out per run and added in a fixed order by a second kernel.
#include "layers.cuh"

namespace dc {
namespace {

constexpr int kElems = 16;  // elements of a row per thread
// Rows above this take blocks of up to 1,024 threads, whose 64 registers each do not hold
// the gradient's sums: they spill, which narrower rows are spared.
constexpr int kWideD = 256 * kElems;

struct Team {
    int size;  // threads of a row
    int lane;  // this thread among them
    int warps;
    float *buf;  // [2][4][32] shared, one block one team (size > 32)
    int phase;

    // Sums of n values over the team, to every thread.
    template <int N>
    __device__ __forceinline__ void sum(float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        if (warps == 1) return;
        float *b = buf + phase * (4 * 32);
        phase ^= 1;
        const int w = lane >> 5, l = lane & 31;
        if (l == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) b[i * 32 + w] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = l < warps ? b[i * 32 + l] : 0.0f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        }
    }
};

template <typename T, int V>
struct Row {
    static constexpr int kItems = kElems / V;
    Vec<T, V> e[kItems];

    __device__ __forceinline__ void load(const T *p, int D, int lane, int size)
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int c = (i * size + lane) * V;
            if (c < D)
                e[i] = *reinterpret_cast<const Vec<T, V> *>(p + c);
            else
#pragma unroll
                for (int j = 0; j < V; ++j) e[i].e[j] = from_float<T>(0.0f);
        }
    }
    __device__ __forceinline__ void ones()
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) e[i].e[j] = from_float<T>(1.0f);
    }
    __device__ __forceinline__ float get(int k) const { return to_float(e[k / V].e[k % V]); }
    __device__ __forceinline__ void set(int k, float v) { e[k / V].e[k % V] = from_float<T>(v); }
    __device__ __forceinline__ void store(T *p, int D, int lane, int size) const
    {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int c = (i * size + lane) * V;
            if (c < D) *reinterpret_cast<Vec<T, V> *>(p + c) = e[i];
        }
    }
};

// Bit k: this thread's element k is kept.
template <int V>
__device__ __forceinline__ uint32_t keep_bits(const DropRule &d, int64_t row, int D, int lane,
                                              int size)
{
    if (d.threshold == 0) return 0xffffffffu;
    const int64_t base = d.offset + row * ((D + 3) / 4);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kElems / V; ++i) {
        const int c = (i * size + lane) * V;
        if (V >= 4) {
#pragma unroll
            for (int q = 0; q < (V >= 4 ? V / 4 : 1); ++q) {
                const uint64_t draw = splitmix(d.seed, uint64_t(base + c / 4 + q));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (kept(d, draw, j)) m |= 1u << (i * V + q * 4 + j);
            }
        } else {
            const uint64_t draw = splitmix(d.seed, uint64_t(base + c / 4));
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (kept(d, draw, (c + j) & 3)) m |= 1u << (i * V + j);
        }
    }
    return m;
}

// Columns past D of a thread's slice (their values must not enter centred sums).
template <int V>
__device__ __forceinline__ bool inside(int k, int D, int lane, int size)
{
    return ((k / V) * size + lane) * V + k % V < D;
}

template <typename T, int V, bool HAS_F, bool HAS_H, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_kernel(NormArgs a)
{
    __shared__ float buf[2 * 4 * 32];
    const int size = blockDim.x, D = a.D;
    Team team{size, int(threadIdx.x), size / 32, buf, 0};
    const int lane = team.lane;
    const float inv = 1.0f / float(D);
    const T *xp = static_cast<const T *>(a.x);
    const T *fp = static_cast<const T *>(a.f);
    const T *gp = static_cast<const T *>(a.gate);
    Row<T, V> post, pre;
    if (a.w_post) post.load(static_cast<const T *>(a.w_post), D, lane, size); else post.ones();
    if (a.w_pre) pre.load(static_cast<const T *>(a.w_pre), D, lane, size); else pre.ones();
    const int64_t first = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
    const int64_t step = int64_t(gridDim.x) * blockDim.y;
    for (int64_t r = first; r < a.rows; r += step) {
        Row<T, V> x;
        x.load(xp + r * D, D, lane, size);
        float y[kElems];
        if (HAS_F) {
            Row<T, V> f, gate;
            f.load(fp + r * D, D, lane, size);
            if (gp) gate.load(gp + (r / a.rows_per_gate) * D, D, lane, size); else gate.ones();
            const uint32_t keep = keep_bits<V>(a.drop, r, D, lane, size);
            float mean = 0.0f, s[1];
            if (a.layer) {
                s[0] = 0.0f;
#pragma unroll
                for (int k = 0; k < kElems; ++k) s[0] += f.get(k);
                team.sum(s);
                mean = s[0] * inv;
            }
            s[0] = 0.0f;
#pragma unroll
            for (int k = 0; k < kElems; ++k) {
                const float v = f.get(k) - mean;
                if (inside<V>(k, D, lane, size)) s[0] += v * v;
            }
            team.sum(s);
            const float rstd = rsqrtf(s[0] * inv + a.eps);
#pragma unroll
            for (int k = 0; k < kElems; ++k) {
                const float z = (f.get(k) - mean) * rstd * post.get(k) * a.drop.scale;
                y[k] = a.alpha * x.get(k) + gate.get(k) * (keep >> k & 1 ? z : 0.0f);
            }
            Row<T, V> o;
#pragma unroll
            for (int k = 0; k < kElems; ++k) o.set(k, y[k]);
            o.store(static_cast<T *>(a.y) + r * D, D, lane, size);
        } else {
#pragma unroll
            for (int k = 0; k < kElems; ++k) y[k] = x.get(k);
        }
        if (HAS_H) {
            float mean = 0.0f, s[1];
            if (a.layer) {
                s[0] = 0.0f;
#pragma unroll
                for (int k = 0; k < kElems; ++k)
                    if (inside<V>(k, D, lane, size)) s[0] += y[k];
                team.sum(s);
                mean = s[0] * inv;
            }
            s[0] = 0.0f;
#pragma unroll
            for (int k = 0; k < kElems; ++k) {
                const float v = y[k] - mean;
                if (inside<V>(k, D, lane, size)) s[0] += v * v;
            }
            team.sum(s);
            const float rstd = rsqrtf(s[0] * inv + a.eps);
            Row<T, V> o;
#pragma unroll
            for (int k = 0; k < kElems; ++k) o.set(k, (y[k] - mean) * rstd * pre.get(k));
            o.store(static_cast<T *>(a.h) + r * D, D, lane, size);
        }
    }
}

// ------------------------------------------------------------------------ gradient
// Run b of P holds rows [rows b / P, rows (b+1) / P).
__host__ __device__ inline int64_t run_start(int64_t rows, int64_t P, int64_t b)
{
    return rows * b / P;
}

// Per run: sums for w_post, w_pre, the gate row shared with the run before, the gate row
// shared with the run after.
constexpr int kSlots = 4;

template <typename T, int V, bool HAS_F, bool HAS_H, int MAXT>
__global__ void __launch_bounds__(MAXT) norm_grad_kernel(NormArgs a, float *partial, int64_t P)
{
    __shared__ float buf[2 * 4 * 32];
    const int size = blockDim.x, D = a.D;
    Team team{size, int(threadIdx.x), size / 32, buf, 0};
    const int lane = team.lane;
    const float inv = 1.0f / float(D);
    const int64_t b = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
    if (b >= P) return;  // a whole team; teams smaller than the block use no barrier
    const int64_t r0 = run_start(a.rows, P, b), r1 = run_start(a.rows, P, b + 1);
    const T *gp = static_cast<const T *>(a.gate);
    Row<T, V> post, pre, gate;
    if (HAS_F) {
        if (a.w_post) post.load(static_cast<const T *>(a.w_post), D, lane, size); else post.ones();
        gate.ones();
    }
    if (HAS_H) {
        if (a.w_pre) pre.load(static_cast<const T *>(a.w_pre), D, lane, size); else pre.ones();
    }
    float gpost[kElems], gpre[kElems], ggate[kElems];
#pragma unroll
    for (int k = 0; k < kElems; ++k) gpost[k] = gpre[k] = ggate[k] = 0.0f;
    auto put = [&](float *p, const float (&v)[kElems]) {
#pragma unroll
        for (int k = 0; k < kElems; ++k) {
            const int c = ((k / V) * size + lane) * V + k % V;
            if (c < D) p[c] = v[k];
        }
    };
    float *slot = partial + b * int64_t(kSlots) * D;
    int64_t g = -1, g_end = 0;
    for (int64_t r = r0; r < r1; ++r) {
        if (HAS_F && (g < 0 || r == g_end)) {
            g = r / a.rows_per_gate;
            g_end = (g + 1) * a.rows_per_gate;
            if (gp) gate.load(gp + g * D, D, lane, size);
        }
        Row<T, V> y, f, dy, dh;
        if (HAS_H) {
            y.load(static_cast<const T *>(a.x) + r * D, D, lane, size);
            dh.load(static_cast<const T *>(a.dh) + r * D, D, lane, size);
        }
        if (HAS_F) f.load(static_cast<const T *>(a.f) + r * D, D, lane, size);
        const bool has_dy = a.dy != nullptr;
        if (has_dy) dy.load(static_cast<const T *>(a.dy) + r * D, D, lane, size);
        uint32_t keep = 0xffffffffu;
        if (HAS_F) keep = keep_bits<V>(a.drop, r, D, lane, size);

        // statistics of y and f, and the sums of dn = dh * w_pre that n'(y)^T needs
        float ym = 0.0f, fm = 0.0f, dm = 0.0f;
        float s[3];
        if (a.layer) {
            s[0] = s[1] = s[2] = 0.0f;
#pragma unroll
            for (int k = 0; k < kElems; ++k) {
                if (HAS_H) {
                    s[0] += y.get(k);
                    s[2] += dh.get(k) * pre.get(k);
                }
                if (HAS_F) s[1] += f.get(k);
            }
            team.sum(s);
            ym = s[0] * inv;
            fm = s[1] * inv;
            dm = s[2] * inv;
        }
        s[0] = s[1] = s[2] = 0.0f;
#pragma unroll
        for (int k = 0; k < kElems; ++k) {
            if (!inside<V>(k, D, lane, size)) continue;
            if (HAS_H) {
                const float v = y.get(k) - ym;
                s[0] += v * v;
                s[2] += dh.get(k) * pre.get(k) * v;
            }
            if (HAS_F) {
                const float v = f.get(k) - fm;
                s[1] += v * v;
            }
        }
        team.sum(s);
        const float yr = HAS_H ? rsqrtf(s[0] * inv + a.eps) : 0.0f;
        const float fr = HAS_F ? rsqrtf(s[1] * inv + a.eps) : 0.0f;
        const float proj = s[2] * inv * yr;  // mean of dn * yhat

        float t[kElems];
#pragma unroll
        for (int k = 0; k < kElems; ++k) {
            t[k] = has_dy ? dy.get(k) : 0.0f;
            if (HAS_H) {
                const float yhat = (y.get(k) - ym) * yr;
                const float d = dh.get(k);
                t[k] += yr * (d * pre.get(k) - dm - yhat * proj);
                gpre[k] += d * yhat;
            }
        }
        Row<T, V> o;
#pragma unroll
        for (int k = 0; k < kElems; ++k) o.set(k, a.alpha * t[k]);
        o.store(static_cast<T *>(a.dx) + r * D, D, lane, size);
        if (!HAS_F) continue;

        float s2[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kElems; ++k) {
            const float fhat = (f.get(k) - fm) * fr;
            const float kt = keep >> k & 1 ? t[k] * a.drop.scale : 0.0f;
            const float u = kt * gate.get(k), p = post.get(k);
            if (inside<V>(k, D, lane, size)) {
                ggate[k] += kt * p * fhat;
                gpost[k] += u * fhat;
                s2[0] += u * p * fhat;
                s2[1] += u * p;
            }
            t[k] = u * p;
        }
        team.sum(s2);
        const float fproj = s2[0] * inv, fdm = a.layer ? s2[1] * inv : 0.0f;
#pragma unroll
        for (int k = 0; k < kElems; ++k)
            o.set(k, fr * (t[k] - fdm - (f.get(k) - fm) * fr * fproj));
        o.store(static_cast<T *>(a.df) + r * D, D, lane, size);

        // the gate row ends here, or this run does
        const bool ends = r + 1 == g_end || r + 1 == a.rows;
        if (a.dgate && (ends || r + 1 == r1)) {
            const int64_t g_start = g * a.rows_per_gate;
            if (ends && g_start >= r0) {
#pragma unroll
                for (int k = 0; k < kElems; ++k) o.set(k, ggate[k]);
                o.store(static_cast<T *>(a.dgate) + g * D, D, lane, size);
            } else {
                put(slot + (g_start < r0 ? 2 : 3) * int64_t(D), ggate);
            }
#pragma unroll
            for (int k = 0; k < kElems; ++k) ggate[k] = 0.0f;
        }
    }
    if (HAS_F && a.dw_post) put(slot, gpost);
    if (HAS_H && a.dw_pre) put(slot + D, gpre);
}

// Adds the runs' sums: block row 0 those of the weights, block row b > 0 those of the
// gate row that runs b - 1 and b share, if b - 1 is where it starts. Four threads a
// column, each a quarter of the runs in order.
constexpr int kFinishCols = 64;
template <typename T>
__global__ void __launch_bounds__(4 * kFinishCols)
norm_finish_kernel(NormArgs a, const float *partial, int64_t P)
{
    __shared__ float part[2][4][kFinishCols];
    const int tx = threadIdx.x, ty = threadIdx.y;
    const int64_t c = int64_t(blockIdx.x) * kFinishCols + tx, D = a.D;
    const int64_t stride = kSlots * D;
    const bool in = c < D;
    float s0 = 0.0f, s1 = 0.0f;
    const int64_t b = blockIdx.y;
    if (b == 0) {
        if (in)
            for (int64_t i = ty; i < P; i += 4) {
                if (a.dw_post) s0 += partial[i * stride + c];
                if (a.dw_pre) s1 += partial[i * stride + D + c];
            }
    } else {
        const int64_t rb = run_start(a.rows, P, b);
        const int64_t g = rb / a.rows_per_gate, gs = g * a.rows_per_gate;
        if (!a.dgate || gs == rb || gs < run_start(a.rows, P, b - 1)) return;  // the whole block
        const int64_t ge = gs + a.rows_per_gate < a.rows ? gs + a.rows_per_gate : a.rows;
        if (in) {
            if (ty == 0) s0 = partial[(b - 1) * stride + 3 * D + c];
            for (int64_t i = b + ty; i < P && run_start(a.rows, P, i) < ge; i += 4)
                s0 += partial[i * stride + 2 * D + c];
        }
    }
    part[0][ty][tx] = s0;
    part[1][ty][tx] = s1;
    __syncthreads();
    if (ty != 0 || !in) return;
    s0 = (part[0][0][tx] + part[0][1][tx]) + (part[0][2][tx] + part[0][3][tx]);
    s1 = (part[1][0][tx] + part[1][1][tx]) + (part[1][2][tx] + part[1][3][tx]);
    if (b == 0) {
        if (a.dw_post) a.dw_post[c] = s0;
        if (a.dw_pre) a.dw_pre[c] = s1;
    } else {
        const int64_t g = run_start(a.rows, P, b) / a.rows_per_gate;
        static_cast<T *>(a.dgate)[g * D + c] = from_float<T>(s0);
    }
}

// Threads of a row, and rows of a block: a warp per row up to 512 columns, four rows a
// block; above, a block per row.
dim3 team_block(int D)
{
    const int size = (D + kElems * 32 - 1) / (kElems * 32) * 32;
    return dim3(unsigned(size), size == 32 ? 4u : 1u);
}

// Runs of the gradient: enough for every SM, and at least 16 rows each where there are
// many rows (a run writes four rows of sums).
int64_t grad_runs(int64_t rows, int D)
{
    const dim3 blk = team_block(D);
    const int64_t teams = int64_t(152) * (blk.y > 1 ? 16 : D <= 4096 ? 2 : 1);
    int64_t P = (rows + 15) / 16;
    if (P < 152) P = rows < 152 ? rows : 152;
    return P < teams ? P : teams;
}

template <typename T, int V, int MAXT>
cudaError_t norm_typed(const NormArgs &a, cudaStream_t stream)
{
    const dim3 blk = team_block(a.D);
    int sms = 0;
    cudaError_t e = sm_count(sms);
    if (e != cudaSuccess) return e;
    int64_t grid = (a.rows + blk.y - 1) / blk.y;
    const int64_t most = int64_t(sms) * (2048 / int(blk.x * blk.y) < 16 ? 2048 / int(blk.x * blk.y) : 16);
    if (grid > most) grid = most;
    if (a.f && a.h)
        norm_kernel<T, V, true, true, MAXT><<<unsigned(grid), blk, 0, stream>>>(a);
    else if (a.f)
        norm_kernel<T, V, true, false, MAXT><<<unsigned(grid), blk, 0, stream>>>(a);
    else
        norm_kernel<T, V, false, true, MAXT><<<unsigned(grid), blk, 0, stream>>>(a);
    return cudaGetLastError();
}

template <typename T, int V, int MAXT>
cudaError_t norm_grad_typed(const NormArgs &a, float *partial, cudaStream_t stream)
{
    const dim3 blk = team_block(a.D);
    const int64_t P = grad_runs(a.rows, a.D);
    const unsigned grid = unsigned((P + blk.y - 1) / blk.y);
    if (a.f && a.dh)
        norm_grad_kernel<T, V, true, true, MAXT><<<grid, blk, 0, stream>>>(a, partial, P);
    else if (a.f)
        norm_grad_kernel<T, V, true, false, MAXT><<<grid, blk, 0, stream>>>(a, partial, P);
    else
        norm_grad_kernel<T, V, false, true, MAXT><<<grid, blk, 0, stream>>>(a, partial, P);
    const bool shared_gates = a.dgate && P > 1;
    if (a.dw_post || a.dw_pre || shared_gates) {
        const dim3 g(unsigned((a.D + kFinishCols - 1) / kFinishCols),
                     shared_gates ? unsigned(P) : 1u);
        norm_finish_kernel<T><<<g, dim3(kFinishCols, 4), 0, stream>>>(a, partial, P);
    }
    return cudaGetLastError();
}

bool vectors_ok(int dtype, const NormArgs &a)
{
    if (a.D % (16 / dtype_bytes(dtype))) return false;
    const void *p[] = {a.x, a.f, a.gate, a.w_post, a.w_pre, a.y, a.h, a.dy, a.dh, a.dx, a.df, a.dgate};
    for (const void *q : p)
        if (!aligned16(q)) return false;
    return true;
}

}  // namespace

cudaError_t launch_norm(int dtype, const NormArgs &a, cudaStream_t stream)
{
    const bool vec = vectors_ok(dtype, a);
    DC_DTYPE_SWITCH(dtype, T, {
        if (a.D <= kWideD)
            return vec ? norm_typed<T, kVec<T>, 256>(a, stream) : norm_typed<T, 1, 256>(a, stream);
        return vec ? norm_typed<T, kVec<T>, 1024>(a, stream) : norm_typed<T, 1, 1024>(a, stream);
    })
}

size_t norm_grad_workspace(int, int64_t rows, int D)
{
    return size_t(grad_runs(rows, D)) * kSlots * size_t(D) * sizeof(float);
}

cudaError_t launch_norm_grad(int dtype, const NormArgs &a, float *partial, cudaStream_t stream)
{
    const bool vec = vectors_ok(dtype, a);
    DC_DTYPE_SWITCH(dtype, T, {
        if (a.D <= kWideD)
            return vec ? norm_grad_typed<T, kVec<T>, 256>(a, partial, stream)
                       : norm_grad_typed<T, 1, 256>(a, partial, stream);
        return vec ? norm_grad_typed<T, kVec<T>, 1024>(a, partial, stream)
                   : norm_grad_typed<T, 1, 1024>(a, partial, stream);
    })
}

}  // namespace dc
