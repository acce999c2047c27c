// Small products of floats on the CUDA cores: any stride and alignment. Tiles of
// 64 x 64, staged in shared memory as floats, 4 x 4 sums per thread (19 TFLOP/s on large ones,
// which go to the tensor cores; what comes here is bound by the launch and its latency).
#include "expert_rows.cuh"

namespace dc {
namespace {

constexpr int kTile = 64, kDepth = 16, kThreads = 256;

// Stages [kTile rows][kDepth] of a strided matrix, transposed: s[depth][row].
__device__ __forceinline__ void stage(float (&s)[kDepth][kTile + 1], const float *p, int64_t s_row,
                                      int64_t s_dep, int rows, int depth, bool depth_first)
{
    for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
        const int row = depth_first ? i / kDepth : i % kTile;
        const int dep = depth_first ? i % kDepth : i / kTile;
        s[dep][row] = row < rows && dep < depth ? p[row * s_row + dep * s_dep] : 0.0f;
    }
}

// WEIGHTS false: the block's tile of rows times the expert's matrix. true: the expert's
// rows are what is summed over.
template <bool WEIGHTS>
__global__ void __launch_bounds__(kThreads) expert_simt_kernel(ExpertArgs g, int64_t most)
{
    extern __shared__ int32_t dyn[];
    __shared__ float sa[kDepth][kTile + 1], sb[kDepth][kTile + 1];
    const Segments seg = segments_at(dyn, g.experts);
    if (threadIdx.x < 32) build_segments<false>(seg, g.offsets, g.rows, g.experts, kTile, 1);
    __syncthreads();
    int e, rows;
    int64_t depth;
    const float *a = static_cast<const float *>(g.a), *b = static_cast<const float *>(g.b);
    float *c = static_cast<float *>(g.c);
    const int n0 = blockIdx.x * kTile;
    if (WEIGHTS) {
        e = blockIdx.z;
        const int64_t r0 = seg.start[e + 1];
        depth = seg.start[e + 2] - r0;
        if (depth > most) return;
        const int m0 = blockIdx.y * kTile;
        rows = min(kTile, g.m - m0);
        a += m0 * g.a_m + r0 * g.a_r;
        b += n0 * g.b_n + r0 * g.b_r;
        c += e * g.c_e + m0 * g.c_m + n0;
    } else {
        const int64_t t = blockIdx.y + int64_t(blockIdx.z) * gridDim.y;
        if (t >= seg.tile[seg.count]) return;
        const int s = find_segment(seg.tile, seg.count, int(t));
        const int64_t r0 = seg.start[s] + int64_t(t - seg.tile[s]) * kTile;
        rows = int(min(int64_t(kTile), seg.start[s + 1] - r0));
        const bool none = s == 0 || s == seg.count - 1;
        depth = none ? 0 : g.r;
        a += r0 * g.a_m;
        b += (none ? 0 : s - 1) * g.b_e + n0 * g.b_n;
        c += r0 * g.c_m + n0;
    }
    const int cols = min(kTile, g.n - n0);
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    float acc[4][4] = {};
    for (int64_t d0 = 0; d0 < depth; d0 += kDepth) {
        const int dd = int(min(int64_t(kDepth), depth - d0));
        stage(sa, a + d0 * g.a_r, g.a_m, g.a_r, rows, dd, g.a_r == 1);
        stage(sb, b + d0 * g.b_r, g.b_n, g.b_r, cols, dd, g.b_r == 1);
        __syncthreads();
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            float x[4], w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = sa[d][ty + 16 * i], w[i] = sb[d][tx + 16 * i];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += x[i] * w[j];
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = ty + 16 * i, col = tx + 16 * j;
            if (row < rows && col < cols) c[row * g.c_m + col] = acc[i][j];
        }
}

}  // namespace

cudaError_t expert_simt_rows(const ExpertArgs &a, cudaStream_t stream)
{
    // at most one short tile per segment
    const int64_t tiles = a.rows / kTile + a.experts + 2;
    const unsigned ty = unsigned(tiles < 32768 ? tiles : 32768);
    const dim3 grid(unsigned((a.n + kTile - 1) / kTile), ty, unsigned((tiles + ty - 1) / ty));
    expert_simt_kernel<false><<<grid, kThreads, segments_bytes(a.experts), stream>>>(a, 0);
    return cudaGetLastError();
}

cudaError_t expert_simt_weights(const ExpertArgs &a, int64_t most, cudaStream_t stream)
{
    const dim3 grid(unsigned((a.n + kTile - 1) / kTile), unsigned((a.m + kTile - 1) / kTile),
                    unsigned(a.experts));
    expert_simt_kernel<true><<<grid, kThreads, segments_bytes(a.experts), stream>>>(a, most);
    return cudaGetLastError();
}

}  // namespace dc
