// Dropout from the counter-based generator and the gated unit with its gradient.
//
// All three move each byte once and are bound by memory: 16-byte accesses, several in
// flight per thread. A thread takes one group of columns and U rows, so that no index is
// divided; narrow rows share a block.
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
template <typename T, int ACT>
__device__ __forceinline__ void act_and_slope(float g, float &a, float &slope)
{
    if (ACT == DC_ACT_SILU) {
        const float s = __fdividef(1.0f, 1.0f + __expf(-g));
        a = g * s;
        slope = s * (1.0f + g * (1.0f - s));
    } else {
        const float cdf = normcdff(g);
        a = g * cdf;
        slope = cdf + g * 0.3989422804014327f * __expf(-0.5f * g * g);
    }
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
        for (int j = 0; j < V; ++j) {
            float a, slope;
            act_and_slope<T, ACT>(to_float(g[u].e[j]), a, slope);
            g[u].e[j] = from_float<T>(a * to_float(m[u].e[j]));
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
        for (int j = 0; j < V; ++j) {
            float a, slope;
            act_and_slope<T, ACT>(to_float(g[u].e[j]), a, slope);
            const float dj = to_float(d[u].e[j]);
            g[u].e[j] = from_float<T>(dj * to_float(m[u].e[j]) * slope);
            m[u].e[j] = from_float<T>(dj * a);
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
