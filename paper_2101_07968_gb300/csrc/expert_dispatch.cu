// Which kernel takes an expert product, and the copies of operands that the tensor cores'
// tile copies cannot read: those need rows that start on 16-byte boundaries.
#include "layers.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256;

// Rows [y][x] of z matrices, x contiguous, to rows padded with zeros to `pad` elements. A
// thread writes eight elements; its eight loads hit the lines that its neighbours' do.
__global__ void __launch_bounds__(kThreads)
align_rows_kernel(const uint16_t *src, uint16_t *dst, int64_t rows, int32_t y, int32_t x, int32_t pad,
                  int64_t stride_z, int64_t stride_y)
{
    const int groups = pad / 8;
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * 8;
    const int64_t r = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
    if (c >= groups * 8 || r >= rows) return;
    const uint16_t *p = src + (r / y) * stride_z + (r % y) * stride_y;
    Vec<uint16_t, 8> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v.e[j] = c + j < x ? p[c + j] : uint16_t(0);
    *reinterpret_cast<Vec<uint16_t, 8> *>(dst + r * pad + c) = v;
}

struct Matrix {
    const void *p;
    int64_t z, y, x;  // extents, x contiguous
    int64_t stride_z, stride_y;
};

bool aligned(const Matrix &m)
{
    return aligned16(m.p) && m.stride_y % 8 == 0 && (m.z == 1 || m.stride_z % 8 == 0);
}
int64_t padded(int64_t x) { return (x + 7) / 8 * 8; }
size_t copy_bytes(const Matrix &m)
{
    return aligned(m) ? 0 : (size_t(m.z) * m.y * padded(m.x) * 2 + 255) / 256 * 256;
}

cudaError_t align_rows(Matrix &m, unsigned char *&workspace, cudaStream_t stream)
{
    const size_t bytes = copy_bytes(m);
    if (!bytes) return cudaSuccess;
    const int64_t pad = padded(m.x), rows = m.z * m.y;
    int bx = 1;
    while (bx < 64 && bx < pad / 8) bx *= 2;
    const int by = kThreads / bx;
    const dim3 grid(unsigned((rows + by - 1) / by), unsigned((pad / 8 + bx - 1) / bx));
    align_rows_kernel<<<grid, dim3(unsigned(bx), unsigned(by)), 0, stream>>>(
        static_cast<const uint16_t *>(m.p), reinterpret_cast<uint16_t *>(workspace), rows, int32_t(m.y),
        int32_t(m.x), int32_t(pad), m.stride_z, m.stride_y);
    m.p = workspace;
    m.stride_y = pad;
    m.stride_z = pad * m.y;
    workspace += bytes;
    return cudaGetLastError();
}

// the two operands with their contiguous axes innermost
void operands(const ExpertArgs &g, bool weights, Matrix &a, Matrix &b)
{
    if (weights) {
        a = {g.a, 1, g.rows, g.m, 0, g.a_r};
        b = {g.b, 1, g.rows, g.n, 0, g.b_r};
    } else {
        const bool k_major = g.b_r == 1;
        a = {g.a, 1, g.rows, g.r, 0, g.a_m};
        b = {g.b, g.experts, k_major ? g.n : g.r, k_major ? g.r : g.n, g.b_e, k_major ? g.b_n : g.b_r};
    }
}

bool few(const ExpertArgs &g, bool weights) { return !weights && g.rows <= DC_FEW_ROWS; }

}  // namespace

size_t expert_workspace(int dtype, const ExpertArgs &g, bool weights)
{
    if (dtype == DC_FP32 || few(g, weights)) return 0;
    Matrix a, b;
    operands(g, weights, a, b);
    return copy_bytes(a) + copy_bytes(b);
}

cudaError_t launch_expert_rows(int dtype, const ExpertArgs &g, void *workspace, cudaStream_t stream)
{
    if (few(g, false)) return expert_few_rows(dtype, g, stream);
    if (dtype == DC_FP32) return expert_simt_rows(g, stream);
    Matrix a, b;
    operands(g, false, a, b);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    cudaError_t e = align_rows(a, ws, stream);
    if (e == cudaSuccess) e = align_rows(b, ws, stream);
    if (e != cudaSuccess) return e;
    ExpertArgs h = g;
    h.a = a.p;
    h.a_m = a.stride_y;
    h.b = b.p;
    h.b_e = b.stride_z;
    (g.b_r == 1 ? h.b_n : h.b_r) = b.stride_y;
    return expert_mma_rows(dtype == DC_BF16, h, stream);
}

cudaError_t launch_expert_weights(int dtype, const ExpertArgs &g, void *workspace,
                                  cudaStream_t stream)
{
    if (g.rows == 0 || dtype == DC_FP32) {
        if (dtype == DC_FP32) return expert_simt_weights(g, stream);
        // no rows: every dW is zero, and there is nothing to read
        for (int e = 0; e < g.experts; ++e) {
            char *p = static_cast<char *>(g.c) + e * g.c_e * 2;
            const cudaError_t r = cudaMemset2DAsync(p, size_t(g.c_m) * 2, 0, size_t(g.n) * 2, size_t(g.m), stream);
            if (r != cudaSuccess) return r;
        }
        return cudaSuccess;
    }
    Matrix a, b;
    operands(g, true, a, b);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    cudaError_t e = align_rows(a, ws, stream);
    if (e == cudaSuccess) e = align_rows(b, ws, stream);
    if (e != cudaSuccess) return e;
    ExpertArgs h = g;
    h.a = a.p;
    h.a_r = a.stride_y;
    h.b = b.p;
    h.b_r = b.stride_y;
    return expert_mma_weights(dtype == DC_BF16, h, stream);
}

}  // namespace dc
