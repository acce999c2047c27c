// Dropout from the counter-based generator and the gated unit with its gradient.
//
// All three move each byte once and are bound by memory: 16-byte accesses, several in
// flight per thread. A thread takes one group of columns and U rows, so that no index is
// divided; narrow rows share a block. Measured (bfloat16, one GB300): dropout of 32,768 x 4,096
// 79 us, 6.8 TB/s; the gated unit 16,384 x 2,048 32 us, 6.2 TB/s, and its gradient 65,536 x 2,048
// 190 us, 7.1 TB/s. Rows whose columns do not fill 16-byte accesses go element by element:
// 30,000 x 1,001 3.8 TB/s (gradient 4.3), dropout of 30,000 x 2,002 2.4.
#include "layers.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256;

// Threads x cover the column groups of a row, threads y and blocks x the rows.
struct RowGrid {
    dim3 grid, block;
};
template <int U>
RowGrid row_grid(int64_t rows, int64_t groups)
{
    int bx = 1;
    while (bx < kThreads && bx < groups) bx *= 2;
    const int by = kThreads / bx;
    RowGrid g;
    g.block = dim3(unsigned(bx), unsigned(by));
    g.grid = dim3(unsigned((rows + int64_t(by) * U - 1) / (int64_t(by) * U)),
                  unsigned((groups + bx - 1) / bx));
    return g;
}

// U rows a thread where that still leaves blocks for every SM
bool many_rows(int64_t rows, int64_t groups) { return rows * groups >= int64_t(152) * 4 * 4 * kThreads; }

// ------------------------------------------------------------------------- dropout
// Contiguous arrays whose columns are a multiple of four: element i uses field i % 4 of
// draw offset + i / 4, whatever its row.
template <typename T, bool RES, int U>
__global__ void __launch_bounds__(kThreads)
dropout_flat_kernel(const T *x, const T *res, T *y, int64_t vectors, DropRule d)
{
    constexpr int V = kVec<T>;
    const int64_t i0 = int64_t(blockIdx.x) * (kThreads * U) + threadIdx.x;
    Vec<T, V> a[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * kThreads;
        if (i < vectors) {
            a[u] = reinterpret_cast<const Vec<T, V> *>(x)[i];
            if (RES) b[u] = reinterpret_cast<const Vec<T, V> *>(res)[i];
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t i = i0 + u * kThreads;
        if (i >= vectors) break;
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const uint64_t draw = splitmix(d.seed, uint64_t(d.offset + i * (V / 4) + q));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = q * 4 + j;
                float v = kept(d, draw, j) ? to_float(a[u].e[k]) * d.scale : 0.0f;
                if (RES) v += to_float(b[u].e[k]);
                a[u].e[k] = from_float<T>(v);
            }
        }
        reinterpret_cast<Vec<T, V> *>(y)[i] = a[u];
    }
}

// Any strides and columns: one draw, four columns of a row, per thread.
template <typename T, bool RES>
__global__ void __launch_bounds__(kThreads)
dropout_rows_kernel(const T *x, int64_t ldx, const T *res, int64_t ldr, T *y, int64_t ldy,
                    int64_t rows, int cols, DropRule d)
{
    const int64_t r = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
    const int words = (cols + 3) / 4;
    const int w = blockIdx.y * blockDim.x + threadIdx.x;
    if (r >= rows || w >= words) return;
    const uint64_t draw = splitmix(d.seed, uint64_t(d.offset + r * words + w));
    T a[4], b[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = w * 4 + j;
        if (c < cols) {
            a[j] = x[r * ldx + c];
            if (RES) b[j] = res[r * ldr + c];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = w * 4 + j;
        if (c >= cols) break;
        float v = kept(d, draw, j) ? to_float(a[j]) * d.scale : 0.0f;
        if (RES) v += to_float(b[j]);
        y[r * ldy + c] = from_float<T>(v);
    }
}

template <typename T, bool RES>
cudaError_t dropout_typed(int64_t rows, int cols, const T *x, int64_t ldx, const T *res,
                          int64_t ldr, T *y, int64_t ldy, const DropRule &d, cudaStream_t stream)
{
    constexpr int V = kVec<T>;
    const bool flat = rows == 1 || (ldx == cols && ldy == cols && (!RES || ldr == cols));
    const int64_t n = rows * int64_t(cols);
    if (flat && (cols % 4 == 0 || rows == 1) && n % V == 0 && aligned16(x) && aligned16(y) &&
        aligned16(res)) {
        const int64_t vectors = n / V;
        if (many_rows(vectors, 1)) {
            constexpr int U = 4;
            dropout_flat_kernel<T, RES, U>
                <<<unsigned((vectors + kThreads * U - 1) / (kThreads * U)), kThreads, 0, stream>>>(
                    x, res, y, vectors, d);
        } else {
            dropout_flat_kernel<T, RES, 1>
                <<<unsigned((vectors + kThreads - 1) / kThreads), kThreads, 0, stream>>>(
                    x, res, y, vectors, d);
        }
    } else {
        const RowGrid g = row_grid<1>(rows, (cols + 3) / 4);
        dropout_rows_kernel<T, RES>
            <<<g.grid, g.block, 0, stream>>>(x, ldx, res, ldr, y, ldy, rows, cols, d);
    }
    return cudaGetLastError();
}

// ---------------------------------------------------------------------- gated unit
// The normal distribution at -|g|, as e^(-g^2/2) s P(s) with s = 1 / (|g| / sqrt 2 + 2): e^(z^2)
// erfc(z) is smooth in 1 / (z + k) over all z >= 0 (the variable of Shepherd and Laframboise,
// Math. Comp. 36, 1981, for the same function). P, of degree 8 in 4 s - 1, was fitted to the
// least largest relative error, 4.4e-8; in 32 bits it stays within 3 2^-23, so that the tail
// keeps its digits where 1/2 (1 + erf) loses them, at two special-function operations an
// element. The gradient of 65,536 x 2,048 took 358 us with normcdff and takes 190 with this.
__device__ __forceinline__ float2 normal_tail(float2 g, float2 &e)
{
    const float2 h = __fmul2_rn(__fmul2_rn(g, g), twice(-0.72134752044448170f));  // -log2(e) / 2
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(h.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(h.y));
    const float2 s = make_float2(__fdividef(1.0f, fabsf(g.x) * 0.70710678f + 2.0f),
                                 __fdividef(1.0f, fabsf(g.y) * 0.70710678f + 2.0f));
    const float2 t = __ffma2_rn(s, twice(4.0f), twice(-1.0f));
    float2 q = twice(-0.000231977624935098f);
    q = __ffma2_rn(q, t, twice(0.0003795158118009567f));
    q = __ffma2_rn(q, t, twice(0.0014894097112119198f));
    q = __ffma2_rn(q, t, twice(-0.0032200065907090902f));
    q = __ffma2_rn(q, t, twice(-0.01074141450226307f));
    q = __ffma2_rn(q, t, twice(0.018217826262116432f));
    q = __ffma2_rn(q, t, twice(0.13973475992679596f));
    q = __ffma2_rn(q, t, twice(0.3435804843902588f));
    q = __ffma2_rn(q, t, twice(0.5107913613319397f));
    return __fmul2_rn(__fmul2_rn(q, s), e);
}

template <int ACT>
__device__ __forceinline__ void act_and_slope(float2 g, float2 &a, float2 &slope)
{
    if (ACT == DC_ACT_SILU) {
        const float2 s = make_float2(__fdividef(1.0f, 1.0f + __expf(-g.x)), __fdividef(1.0f, 1.0f + __expf(-g.y)));
        a = __fmul2_rn(g, s);
        slope = __fmul2_rn(s, __ffma2_rn(g, make_float2(1.0f - s.x, 1.0f - s.y), twice(1.0f)));
    } else {
        float2 e;
        const float2 q = normal_tail(g, e);
        const float2 cdf = make_float2(g.x > 0.0f ? 1.0f - q.x : q.x, g.y > 0.0f ? 1.0f - q.y : q.y);
        a = __fmul2_rn(g, cdf);
        slope = __ffma2_rn(__fmul2_rn(g, e), twice(0.3989422804014327f), cdf);
    }
}

// pairs of a thread's V elements; V = 1 works on one
template <typename T, int V>
__device__ __forceinline__ float2 pair_in(const Vec<T, V> &v, int j)
{
    if (V == 1) return make_float2(to_float(v.e[0]), 0.0f);
    return pair_of(&v.e[V == 1 ? 0 : j]);
}
template <typename T, int V>
__device__ __forceinline__ void pair_out(Vec<T, V> &v, int j, float2 x)
{
    if (V == 1)
        v.e[0] = from_float<T>(x.x);
    else
        put_pair(&v.e[V == 1 ? 0 : j], x);
}

template <typename T, int ACT, int V, int U>
__global__ void __launch_bounds__(kThreads)
gated_kernel(const T *h, int64_t ldh, T *out, int64_t lda, int64_t rows, int F)
{
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
    if (c >= F) return;
    const int64_t r0 = int64_t(blockIdx.x) * (blockDim.y * U) + threadIdx.y;
    Vec<T, V> g[U], m[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * blockDim.y;
        if (r < rows) {
            g[u] = *reinterpret_cast<const Vec<T, V> *>(h + r * ldh + c);
            m[u] = *reinterpret_cast<const Vec<T, V> *>(h + r * ldh + F + c);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * blockDim.y;
        if (r >= rows) break;
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            float2 a, slope;
            act_and_slope<ACT>(pair_in(g[u], j), a, slope);
            pair_out(g[u], j, __fmul2_rn(a, pair_in(m[u], j)));
        }
        *reinterpret_cast<Vec<T, V> *>(out + r * lda + c) = g[u];
    }
}

template <typename T, int ACT, int V, int U>
__global__ void __launch_bounds__(kThreads)
gated_grad_kernel(const T *da, int64_t ldda, const T *h, int64_t ldh, T *dh, int64_t lddh,
                  int64_t rows, int F)
{
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
    if (c >= F) return;
    const int64_t r0 = int64_t(blockIdx.x) * (blockDim.y * U) + threadIdx.y;
    Vec<T, V> g[U], m[U], d[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * blockDim.y;
        if (r < rows) {
            g[u] = *reinterpret_cast<const Vec<T, V> *>(h + r * ldh + c);
            m[u] = *reinterpret_cast<const Vec<T, V> *>(h + r * ldh + F + c);
            d[u] = *reinterpret_cast<const Vec<T, V> *>(da + r * ldda + c);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int64_t r = r0 + u * blockDim.y;
        if (r >= rows) break;
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            float2 a, slope;
            act_and_slope<ACT>(pair_in(g[u], j), a, slope);
            const float2 dj = pair_in(d[u], j);
            pair_out(g[u], j, __fmul2_rn(__fmul2_rn(dj, pair_in(m[u], j)), slope));
            pair_out(m[u], j, __fmul2_rn(dj, a));
        }
        *reinterpret_cast<Vec<T, V> *>(dh + r * lddh + c) = g[u];
        *reinterpret_cast<Vec<T, V> *>(dh + r * lddh + F + c) = m[u];
    }
}

template <typename T, int ACT, int V, int U>
void gated_launch(int64_t rows, int F, const T *h, int64_t ldh, T *a, int64_t lda,
                  cudaStream_t stream)
{
    const RowGrid g = row_grid<U>(rows, F / V);
    gated_kernel<T, ACT, V, U><<<g.grid, g.block, 0, stream>>>(h, ldh, a, lda, rows, F);
}

template <typename T, int ACT, int V, int U>
void gated_grad_launch(int64_t rows, int F, const T *da, int64_t ldda, const T *h, int64_t ldh,
                       T *dh, int64_t lddh, cudaStream_t stream)
{
    const RowGrid g = row_grid<U>(rows, F / V);
    gated_grad_kernel<T, ACT, V, U>
        <<<g.grid, g.block, 0, stream>>>(da, ldda, h, ldh, dh, lddh, rows, F);
}

template <typename T, int ACT>
cudaError_t gated_typed(int64_t rows, int F, const T *h, int64_t ldh, T *a, int64_t lda,
                        cudaStream_t stream)
{
    constexpr int V = kVec<T>;
    if (F % V == 0 && ldh % V == 0 && lda % V == 0 && aligned16(h) && aligned16(a)) {
        if (many_rows(rows, F / V))
            gated_launch<T, ACT, V, 4>(rows, F, h, ldh, a, lda, stream);
        else
            gated_launch<T, ACT, V, 1>(rows, F, h, ldh, a, lda, stream);
    } else {
        gated_launch<T, ACT, 1, 4>(rows, F, h, ldh, a, lda, stream);
    }
    return cudaGetLastError();
}

template <typename T, int ACT>
cudaError_t gated_grad_typed(int64_t rows, int F, const T *da, int64_t ldda, const T *h,
                             int64_t ldh, T *dh, int64_t lddh, cudaStream_t stream)
{
    constexpr int V = kVec<T>;
    if (F % V == 0 && ldh % V == 0 && ldda % V == 0 && lddh % V == 0 && aligned16(h) &&
        aligned16(da) && aligned16(dh)) {
        if (many_rows(rows, F / V))
            gated_grad_launch<T, ACT, V, 2>(rows, F, da, ldda, h, ldh, dh, lddh, stream);
        else
            gated_grad_launch<T, ACT, V, 1>(rows, F, da, ldda, h, ldh, dh, lddh, stream);
    } else {
        gated_grad_launch<T, ACT, 1, 4>(rows, F, da, ldda, h, ldh, dh, lddh, stream);
    }
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_dropout(int dtype, int64_t rows, int cols, const void *x, int64_t ldx,
                           const void *res, int64_t ldr, void *y, int64_t ldy, const DropRule &d,
                           cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, {
        if (res)
            return dropout_typed<T, true>(rows, cols, static_cast<const T *>(x), ldx,
                                          static_cast<const T *>(res), ldr, static_cast<T *>(y),
                                          ldy, d, stream);
        return dropout_typed<T, false>(rows, cols, static_cast<const T *>(x), ldx, nullptr, 0,
                                       static_cast<T *>(y), ldy, d, stream);
    })
}

cudaError_t launch_gated(int dtype, int act, int64_t rows, int F, const void *h, int64_t ldh,
                         void *a, int64_t lda, cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, {
        const T *hp = static_cast<const T *>(h);
        T *ap = static_cast<T *>(a);
        return act == DC_ACT_SILU
                   ? gated_typed<T, DC_ACT_SILU>(rows, F, hp, ldh, ap, lda, stream)
                   : gated_typed<T, DC_ACT_GELU>(rows, F, hp, ldh, ap, lda, stream);
    })
}

cudaError_t launch_gated_grad(int dtype, int act, int64_t rows, int F, const void *da,
                              int64_t ldda, const void *h, int64_t ldh, void *dh, int64_t lddh,
                              cudaStream_t stream)
{
    DC_DTYPE_SWITCH(dtype, T, {
        const T *dp = static_cast<const T *>(da);
        const T *hp = static_cast<const T *>(h);
        T *op = static_cast<T *>(dh);
        return act == DC_ACT_SILU
                   ? gated_grad_typed<T, DC_ACT_SILU>(rows, F, dp, ldda, hp, ldh, op, lddh, stream)
                   : gated_grad_typed<T, DC_ACT_GELU>(rows, F, dp, ldda, hp, ldh, op, lddh, stream);
    })
}

}  // namespace dc
