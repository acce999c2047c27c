// Which kernel takes an expert product, and the copies of operands that the tensor cores
// cannot take as they are: tile copies need rows that start on 16-byte boundaries, and floats
// go in parts.
//
// Floats on the tensor cores: x = hi + lo with hi and lo of the 11 significant bits that tf32
// holds, and x w = hi hi + hi lo + lo hi: three products of operands that hold both parts.
// What is left out (lo lo, and the bits of x past lo) is below 3 2^-22 |x w| a product, and 7e-8
// of it in the root mean square. With the sums as expert_mma.cu takes them, products of at least
// kPartDepth summed elements come out nearer than a 32-bit sum of one product after another (operands
// of one sign: from 96 on; at 64 they are 1.3e-7 off against 1.15). The CUDA cores take shorter ones.
// Weight gradients go in parts from kPartLeast rows of an expert on: 9e-8 off against 6 at 8 rows, 1.3e-7
// against 1.1 at 32, less from 48 on; the CUDA cores would need several times as long.
// 16,384 rows over 8 experts x 2,048 x 2,048: 576 us, 238 TFLOP/s with the copies (a library product of
// floats 2.3 ms), and 2e-7 off in the root mean square.
#include "expert_rows.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256;

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

// One matrix of a copy: rows [z][y][x], x contiguous, to rows padded with zeros to `pad`
// elements. A block takes (kThreads >> wide) rows by (1 << wide) groups of eight elements.
struct Copy {
    const uint16_t *src;
    uint16_t *dst;
    int64_t rows, stride_z, stride_y;
    int32_t y, x, pad, wide;
    int64_t blocks_x, blocks;
};

Copy copy_of(const Matrix &m, void *dst)
{
    Copy c = {static_cast<const uint16_t *>(m.p), static_cast<uint16_t *>(dst), m.z * m.y, m.stride_z, m.stride_y,
              int32_t(m.y), int32_t(m.x), int32_t(padded(m.x)), 0, 0, 0};
    while ((1 << c.wide) < 64 && (1 << c.wide) < c.pad / 8) ++c.wide;
    const int by = kThreads >> c.wide, bx = 1 << c.wide;
    c.blocks_x = (c.pad / 8 + bx - 1) / bx;
    c.blocks = c.blocks_x * ((c.rows + by - 1) / by);
    return c;
}

// Both operands' copies in one launch (a launch costs what a small copy does): the first
// a.blocks blocks are a's, the others b's. A thread writes eight elements; its eight loads
// hit the lines that its neighbours' do.
__global__ void __launch_bounds__(kThreads) align_rows_kernel(Copy a, Copy b)
{
    const bool second = blockIdx.x >= a.blocks;
    const Copy &m = second ? b : a;
    const int64_t block = blockIdx.x - (second ? a.blocks : 0);
    const int64_t r = block / m.blocks_x * (kThreads >> m.wide) + (threadIdx.x >> m.wide);
    const int c = int(block % m.blocks_x << m.wide | (threadIdx.x & ((1 << m.wide) - 1))) * 8;
    if (c >= m.pad || r >= m.rows) return;
    const uint16_t *p = m.src + (r / m.y) * m.stride_z + (r % m.y) * m.stride_y;
    Vec<uint16_t, 8> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v.e[j] = c + j < m.x ? p[c + j] : uint16_t(0);
    *reinterpret_cast<Vec<uint16_t, 8> *>(m.dst + r * m.pad + c) = v;
}

// Copies of a and b that need them; a and b then are the copies.
cudaError_t align_rows(Matrix &a, Matrix &b, void *workspace, cudaStream_t stream)
{
    Copy c[2] = {};
    unsigned char *at = static_cast<unsigned char *>(workspace);
    Matrix *m[2] = {&a, &b};
    for (int i = 0; i < 2; ++i) {
        const size_t bytes = copy_bytes(*m[i]);
        if (!bytes) continue;
        c[i] = copy_of(*m[i], at);
        m[i]->p = at;
        m[i]->stride_y = c[i].pad;
        m[i]->stride_z = int64_t(c[i].pad) * m[i]->y;
        at += bytes;
    }
    const int64_t blocks = c[0].blocks + c[1].blocks;
    if (!blocks) return cudaSuccess;
    align_rows_kernel<<<unsigned(blocks), kThreads, 0, stream>>>(c[0], c[1]);
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

// Two rows, two experts x 4,096 x 2,048: 8.3 us, by tiles 12.2; eight rows 12.5 against 12.1;
// sixteen rows of as many experts x 2,048 x 2,048 36 against 26.8. Floats go that way up to 64 rows:
// their parts would cost twice the weights' bytes to write (30 rows over 4 experts x
// 2,048 x 2,048: 29 us in a graph, in parts 108).
bool few(int dtype, const ExpertArgs &g, bool weights)
{
    return !weights && g.rows <= (dtype == DC_FP32 ? 16 * DC_FEW_ROWS : DC_FEW_ROWS);
}

// ----------------------------------------------------------------- floats in parts
constexpr int kPartDepth = 64, kPartLeast = 8;

__device__ __forceinline__ void parts_of(const float x, float &hi, float &lo)
{
    uint32_t h;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(h) : "f"(x));
    hi = __uint_as_float(h & 0xffffe000u);
    // rounded past the largest float (or infinite): cut off instead, without a second part
    if (isinf(hi)) hi = __uint_as_float(__float_as_uint(x) & 0xffffe000u);
    lo = isinf(hi) ? 0.0f : x - hi;
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(h) : "f"(lo));
    lo = __uint_as_float(h & 0xffffe000u);
}

// A row's high parts, then its low ones.
__device__ __forceinline__ void put_parts(float *row, int64_t half, int64_t at, float x)
{
    float hi, lo;
    parts_of(x, hi, lo);
    row[at] = hi;
    row[half + at] = lo;
}

// Rows [z][y][x], x contiguous and summed; a thread takes four elements. wide: rows start on
// 16-byte boundaries.
__global__ void __launch_bounds__(kThreads)
split_rows_kernel(const float *src, float *dst, int64_t rows, int32_t y, int32_t x, int32_t pad,
                  int64_t stride_z, int64_t stride_y, bool wide)
{
    const int c = (blockIdx.y * blockDim.x + threadIdx.x) * 4;
    const int64_t r = int64_t(blockIdx.x) * blockDim.y + threadIdx.y;
    if (c >= pad || r >= rows) return;
    const float *p = src + (r / y) * stride_z + (r % y) * stride_y;
    Vec<float, 4> v, lo;
    if (wide && c + 4 <= x) {
        v = *reinterpret_cast<const Vec<float, 4> *>(p + c);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) v.e[j] = c + j < x ? p[c + j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) parts_of(v.e[j], v.e[j], lo.e[j]);
    float *q = dst + r * 2 * pad + c;
    *reinterpret_cast<Vec<float, 4> *>(q) = v;
    *reinterpret_cast<Vec<float, 4> *>(q + pad) = lo;
}

// The transposing copies: a block brings 32 summed lines of kAcross columns into shared memory
// and writes them as parts, 32 neighbours of a column at a time.
constexpr int kAcross = 128;
struct Across {
    float at[32][kAcross + 1];
};
__device__ __forceinline__ void load_across(Across &t, const float *p, int64_t stride, int64_t lines, int columns)
{
    const int tx = threadIdx.x % 32, ty = threadIdx.x / 32;
#pragma unroll
    for (int i = 0; i < 32; i += kThreads / 32)
#pragma unroll
        for (int c = 0; c < kAcross; c += 32)
            t.at[i + ty][c + tx] = i + ty < lines && c + tx < columns ? p[(i + ty) * stride + c + tx] : 0.0f;
    __syncthreads();
}
__device__ __forceinline__ void put_across(const Across &t, float *rows, int64_t pitch, int64_t half, int columns)
{
    const int tx = threadIdx.x % 32;
#pragma unroll 4
    for (int c = threadIdx.x / 32; c < columns; c += kThreads / 32) put_parts(rows + c * pitch, half, tx, t.at[tx][c]);
}

// [z][x][y], y contiguous and x summed, to rows [z][y].
__global__ void __launch_bounds__(kThreads)
split_columns_kernel(const float *src, float *dst, int32_t y, int32_t x, int32_t pad, int64_t stride_z,
                     int64_t stride_x)
{
    __shared__ Across tile;
    const int x0 = blockIdx.x * 32, y0 = blockIdx.y * kAcross, columns = min(kAcross, y - y0);
    load_across(tile, src + blockIdx.z * stride_z + x0 * stride_x + y0, stride_x, x - x0, columns);
    put_across(tile, dst + (int64_t(blockIdx.z) * y + y0) * 2 * pad + x0, 2 * int64_t(pad), pad, columns);
}

// The rows of the batch [rows][y], summed expert by expert, to rows [y]: each segment's rows are
// rounded up to kPartRows with zeros, and its two parts lie side by side.
__global__ void __launch_bounds__(kThreads)
split_segments_kernel(const float *src, float *dst, const int64_t *offsets, int64_t rows, int32_t experts,
                      int32_t y, int64_t stride, int64_t pitch)
{
    extern __shared__ int32_t dyn[];
    __shared__ Across tile;
    const Segments seg = segments_at(dyn, experts);
    if (threadIdx.x < 32) build_segments<false>(seg, offsets, rows, experts, kPartRows, 1);
    __syncthreads();
    const int t = blockIdx.x;
    if (t >= seg.tile[seg.count]) return;
    const int s = find_segment(seg.tile, seg.count, t), first = seg.tile[s];
    const int64_t r0 = seg.start[s] + int64_t(t - first) * kPartRows;
    const int64_t half = int64_t(seg.tile[s + 1] - first) * kPartRows;
    for (int y0 = blockIdx.y * kAcross; y0 < y; y0 += gridDim.y * kAcross) {
        const int columns = min(kAcross, y - y0);
        load_across(tile, src + r0 * stride + y0, stride, seg.start[s + 1] - r0, columns);
        put_across(tile, dst + y0 * pitch + int64_t(first) * 2 * kPartRows + int64_t(t - first) * kPartRows, pitch, half,
                   columns);
        __syncthreads();
    }
}

int64_t part_pad(int64_t r) { return (r + 31) / 32 * 32; }
// the longest that the segments' rounded rows can be
int64_t part_rows(const ExpertArgs &g) { return (g.rows / kPartRows + g.experts + 3) * kPartRows; }
size_t part_bytes(int64_t rows, int64_t length) { return (size_t(rows) * 2 * length * 4 + 255) / 256 * 256; }

// Shorter sums and smaller batches stay on the CUDA cores, where the bounds above hold and the
// copies would take longer than the products (200 rows over 8 experts x 512 x 512 take 27-32 us
// in parts, most of it copies and launches).
bool use_parts(const ExpertArgs &g, bool weights)
{
    if (2 * part_rows(g) >= int64_t(1) << 31) return false;
    return weights ? g.rows >= 64 && g.rows >= 2 * kPartLeast * int64_t(g.experts)
                   : g.r >= kPartDepth;
}

cudaError_t split_rows(const Matrix &m, float *dst, cudaStream_t stream)
{
    const int64_t pad = part_pad(m.x), rows = m.z * m.y;
    int bx = 8;
    while (bx < 64 && bx < pad / 4) bx *= 2;
    const int by = kThreads / bx;
    const dim3 grid(unsigned((rows + by - 1) / by), unsigned((pad / 4 + bx - 1) / bx));
    const bool wide = aligned16(m.p) && m.stride_y % 4 == 0 && (m.z == 1 || m.stride_z % 4 == 0);
    split_rows_kernel<<<grid, dim3(unsigned(bx), unsigned(by)), 0, stream>>>(
        static_cast<const float *>(m.p), dst, rows, int32_t(m.y), int32_t(m.x), int32_t(pad), m.stride_z, m.stride_y, wide);
    return cudaGetLastError();
}

cudaError_t float_rows(const ExpertArgs &g, void *workspace, cudaStream_t stream)
{
    const int64_t pad = part_pad(g.r);
    float *a = static_cast<float *>(workspace);
    float *b = reinterpret_cast<float *>(static_cast<char *>(workspace) + part_bytes(g.rows, pad));
    cudaError_t e = split_rows({g.a, 1, g.rows, g.r, 0, g.a_m}, a, stream);
    if (e != cudaSuccess) return e;
    if (g.b_r == 1) {
        e = split_rows({g.b, g.experts, g.n, g.r, g.b_e, g.b_n}, b, stream);
    } else {
        const dim3 grid(unsigned(pad / 32), unsigned((g.n + kAcross - 1) / kAcross), unsigned(g.experts));
        split_columns_kernel<<<grid, kThreads, 0, stream>>>(static_cast<const float *>(g.b), b, g.n, g.r,
                                                                   int32_t(pad), g.b_e, g.b_r);
        e = cudaGetLastError();
    }
    if (e != cudaSuccess) return e;
    ExpertArgs h = g;
    h.a = a;
    h.a_m = 2 * pad;
    h.b = b;
    h.b_r = 1;
    h.b_n = 2 * pad;
    h.b_e = 2 * pad * g.n;
    h.r = int32_t(pad);
    return expert_mma_rows(DC_FP32, h, nullptr, stream);
}

cudaError_t float_weights(const ExpertArgs &g, void *workspace, cudaStream_t stream)
{
    const int64_t length = part_rows(g);
    float *a = static_cast<float *>(workspace);
    float *b = reinterpret_cast<float *>(static_cast<char *>(workspace) + part_bytes(g.m, length));
    const unsigned tiles = unsigned(length / kPartRows);
    // a block finds its segment once, for up to four slices of columns
    auto slices = [](int n) { return unsigned((n + 4 * kAcross - 1) / (4 * kAcross)); };
    split_segments_kernel<<<dim3(tiles, slices(g.m)), kThreads, segments_bytes(g.experts), stream>>>(
        static_cast<const float *>(g.a), a, g.offsets, g.rows, g.experts, g.m, g.a_r, 2 * length);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    split_segments_kernel<<<dim3(tiles, slices(g.n)), kThreads, segments_bytes(g.experts), stream>>>(
        static_cast<const float *>(g.b), b, g.offsets, g.rows, g.experts, g.n, g.b_r, 2 * length);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    ExpertArgs h = g;
    h.a = a;
    h.a_r = 2 * length;
    h.b = b;
    h.b_r = 2 * length;
    e = expert_mma_weights(DC_FP32, h, kPartLeast, nullptr, stream);
    return e != cudaSuccess ? e : expert_simt_weights(g, kPartLeast - 1, stream);
}

}  // namespace

size_t expert_workspace(int dtype, const ExpertArgs &g, bool weights)
{
    if (few(dtype, g, weights)) return 0;
    if (dtype == DC_FP32) {
        if (!use_parts(g, weights)) return 0;
        return weights ? part_bytes(g.m, part_rows(g)) + part_bytes(g.n, part_rows(g))
                       : part_bytes(g.rows, part_pad(g.r)) + part_bytes(int64_t(g.experts) * g.n, part_pad(g.r));
    }
    Matrix a, b;
    operands(g, weights, a, b);
    return copy_bytes(a) + copy_bytes(b) + expert_mma_sum_bytes(dtype, g, weights);
}

// After the copies: the sums of long products, NULL for others.
static float *sums_at(int dtype, const ExpertArgs &g, bool weights, void *workspace, size_t copies)
{
    return expert_mma_sum_bytes(dtype, g, weights)
               ? reinterpret_cast<float *>(static_cast<char *>(workspace) + copies) : nullptr;
}

cudaError_t launch_expert_rows(int dtype, const ExpertArgs &g, void *workspace, cudaStream_t stream)
{
    if (few(dtype, g, false)) return expert_few_rows(dtype, g, stream);
    if (dtype == DC_FP32) return use_parts(g, false) ? float_rows(g, workspace, stream) : expert_simt_rows(g, stream);
    Matrix a, b;
    operands(g, false, a, b);
    float *sums = sums_at(dtype, g, false, workspace, copy_bytes(a) + copy_bytes(b));
    const cudaError_t e = align_rows(a, b, workspace, stream);
    if (e != cudaSuccess) return e;
    ExpertArgs h = g;
    h.a = a.p;
    h.a_m = a.stride_y;
    h.b = b.p;
    h.b_e = b.stride_z;
    (g.b_r == 1 ? h.b_n : h.b_r) = b.stride_y;
    return expert_mma_rows(dtype, h, sums, stream);
}

cudaError_t launch_expert_weights(int dtype, const ExpertArgs &g, void *workspace,
                                  cudaStream_t stream)
{
    if (dtype == DC_FP32)
        return g.rows > 0 && use_parts(g, true) ? float_weights(g, workspace, stream)
                                                : expert_simt_weights(g, g.rows, stream);
    if (g.rows == 0) {  // every dW is zero, and there is nothing to read
        for (int e = 0; e < g.experts; ++e) {
            char *p = static_cast<char *>(g.c) + e * g.c_e * 2;
            const cudaError_t r = cudaMemset2DAsync(p, size_t(g.c_m) * 2, 0, size_t(g.n) * 2, size_t(g.m), stream);
            if (r != cudaSuccess) return r;
        }
        return cudaSuccess;
    }
    Matrix a, b;
    operands(g, true, a, b);
    float *sums = sums_at(dtype, g, true, workspace, copy_bytes(a) + copy_bytes(b));
    const cudaError_t e = align_rows(a, b, workspace, stream);
    if (e != cudaSuccess) return e;
    ExpertArgs h = g;
    h.a = a.p;
    h.a_r = a.stride_y;
    h.b = b.p;
    h.b_r = b.stride_y;
    return expert_mma_weights(dtype, h, 0, sums, stream);
}

}  // namespace dc
