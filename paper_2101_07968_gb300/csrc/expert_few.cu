// Expert products of a few rows: matrix-vector products that stream each expert's weights
// once over every SM, where tiles would leave most of them idle. Bound by memory: the
// weights of the experts that have rows.
//
// A block takes one group of up to kGroup rows of one expert and a slice of features.
// Weights with the summed axis contiguous: a warp per two features, lanes along the axis,
// eight 16-byte loads a lane in flight. Weights with the features contiguous: a lane holds
// several features and the block's lanes split the summed axis. The sums are added in a
// fixed order. Two rows of two experts x 4,096 x 2,048 (bfloat16): 7.8 us in a graph, 4.3 TB/s; the
// offsets' latency and then the weights' are what is left; with the features contiguous 9.8 us.
#include "layers.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kGroup = 4;  // rows that share a pass over the weights

struct Group {
    int expert;  // -1: rows of no expert
    int64_t row;
    int rows;    // 0: another block's
};

// The group that starts at row `r`, if one does: groups are cut from each segment's start.
__device__ __forceinline__ Group group_at(const ExpertArgs &g, int64_t r)
{
    __shared__ int64_t found[3];
    if (threadIdx.x < 32) {
        // the running maximum of the clamped offsets gives the segments; the last one that
        // starts at or before r holds it
        const int lane = threadIdx.x;
        int64_t top = 0, start = 0, end = g.rows;
        int expert = -1;
        for (int e0 = 0; e0 <= g.experts; e0 += 32) {
            const int e = e0 + lane;
            int64_t v = e <= g.experts ? g.offsets[e] : g.rows;
            v = v < 0 ? 0 : v > g.rows ? g.rows : v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o && u > v) v = u;
            }
            if (v < top) v = top;
            const uint32_t below = __ballot_sync(0xffffffffu, e <= g.experts && v <= r);
            const int n = __popc(below);  // starts are in order, so these are the first n lanes
            if (n) {
                expert = e0 + n - 1;
                start = __shfl_sync(0xffffffffu, v, n - 1);
            }
            const int64_t after = __shfl_sync(0xffffffffu, v, n < 32 ? n : 31);
            if (n < 32) {
                end = e0 + n <= g.experts ? after : g.rows;
                break;
            }
            top = __shfl_sync(0xffffffffu, v, 31);
        }
        if (expert >= g.experts) {  // after the last expert
            expert = -1;
            end = g.rows;
        }
        if (lane == 0) {
            found[0] = expert;
            found[1] = start;
            found[2] = end;
        }
    }
    __syncthreads();
    Group q;
    q.expert = int(found[0]);
    q.row = r;
    const int64_t left = found[2] - r;
    q.rows = (r - found[1]) % kGroup ? 0 : int(left < kGroup ? left : kGroup);
    return q;
}

// Weights with the summed axis contiguous: kFeatures features of a warp at once, so that two
// tokens' 8,192 products of 2,048 elements are all in flight in one round of blocks.
constexpr int kFeatures = 2;
template <typename T, int V, int ROWS>
__device__ __forceinline__ void dot_rows(const ExpertArgs &g, const Group &q, int n)
{
    constexpr int U = V > 1 ? 4 : 8;  // loads of a feature in flight
    const int lane = threadIdx.x & 31;
    const T *w[kFeatures];
#pragma unroll
    for (int f = 0; f < kFeatures; ++f)  // the last feature again past the end
        w[f] = static_cast<const T *>(g.b) + q.expert * g.b_e + int64_t(min(n + f, g.n - 1)) * g.b_n;
    const T *x = static_cast<const T *>(g.a) + q.row * g.a_m;
    float acc[kFeatures][ROWS];
#pragma unroll
    for (int f = 0; f < kFeatures; ++f)
#pragma unroll
        for (int i = 0; i < ROWS; ++i) acc[f][i] = 0.0f;
    for (int64_t k0 = lane * V; k0 < g.r; k0 += 32 * V * U) {
        Vec<T, V> b[kFeatures][U];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int f = 0; f < kFeatures; ++f) {
                const int64_t k = k0 + u * 32 * V;
                if (k < g.r) b[f][u] = *reinterpret_cast<const Vec<T, V> *>(w[f] + k);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = k0 + u * 32 * V;
            if (k >= g.r) break;
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const Vec<T, V> a = *reinterpret_cast<const Vec<T, V> *>(x + i * g.a_m + k);
#pragma unroll
                for (int f = 0; f < kFeatures; ++f)
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[f][i] += to_float(a.e[j]) * to_float(b[f][u].e[j]);
            }
        }
    }
#pragma unroll
    for (int f = 0; f < kFeatures; ++f)
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            float v = acc[f][i];
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == 0 && n + f < g.n) static_cast<T *>(g.c)[(q.row + i) * g.c_m + n + f] = from_float<T>(v);
        }
}

template <typename T, int V>
__global__ void __launch_bounds__(kThreads, 2) few_dot_kernel(ExpertArgs g)
{
    const Group q = group_at(g, blockIdx.y);
    if (q.rows == 0) return;
    const int n = (blockIdx.x * kWarps + threadIdx.x / 32) * kFeatures;
    if (n >= g.n) return;
    if (q.expert < 0) {
        const int i = (threadIdx.x & 31) / kFeatures, f = threadIdx.x % kFeatures;
        if (i < q.rows && n + f < g.n) static_cast<T *>(g.c)[(q.row + i) * g.c_m + n + f] = from_float<T>(0.0f);
    } else if (q.rows == 1) {
        dot_rows<T, V, 1>(g, q, n);
    } else if (q.rows == 2) {
        dot_rows<T, V, 2>(g, q, n);
    } else if (q.rows == 3) {
        dot_rows<T, V, 3>(g, q, n);
    } else {
        dot_rows<T, V, 4>(g, q, n);
    }
}

// Weights with the features contiguous: a block takes kCols of them, kCols / V lanes wide, and
// its other lanes split the summed axis.
constexpr int kCols = 32, kColumnThreads = 512, kColumnWarps = kColumnThreads / 32;
template <typename T, int V, int ROWS>
__device__ __forceinline__ void column_rows(const ExpertArgs &g, const Group &q, int n0,
                                            float (&part)[kColumnWarps][kGroup][kCols])
{
    constexpr int kWide = kCols / V, kSplit = kColumnThreads / kWide, U = 8;
    const int f = threadIdx.x % kWide * V, s = threadIdx.x / kWide;
    const int n = n0 + f, lane = threadIdx.x & 31;
    const T *w = static_cast<const T *>(g.b) + q.expert * g.b_e + n;
    const T *x = static_cast<const T *>(g.a) + q.row * g.a_m;
    float acc[ROWS][V];
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) acc[i][j] = 0.0f;
    if (n < g.n) {
        for (int64_t k0 = s; k0 < g.r; k0 += kSplit * U) {
            Vec<T, V> b[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = k0 + u * kSplit;
                if (k < g.r) b[u] = *reinterpret_cast<const Vec<T, V> *>(w + k * g.b_r);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t k = k0 + u * kSplit;
                if (k >= g.r) break;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) {
                    const float a = to_float(x[i * g.a_m + k]);
#pragma unroll
                    for (int j = 0; j < V; ++j) acc[i][j] += a * to_float(b[u].e[j]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) {
#pragma unroll
            for (int o = 16; o >= kWide; o >>= 1) acc[i][j] += __shfl_xor_sync(0xffffffffu, acc[i][j], o);
            if (lane < kWide) part[threadIdx.x / 32][i][f + j] = acc[i][j];
        }
    __syncthreads();
    for (int t = threadIdx.x; t < ROWS * kCols; t += kColumnThreads) {
        const int i = t / kCols, c = t % kCols;
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < kColumnWarps; ++k) v += part[k][i][c];
        if (n0 + c < g.n) static_cast<T *>(g.c)[(q.row + i) * g.c_m + n0 + c] = from_float<T>(v);
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kColumnThreads) few_column_kernel(ExpertArgs g)
{
    __shared__ float part[kColumnWarps][kGroup][kCols];
    const Group q = group_at(g, blockIdx.y);
    const int n0 = blockIdx.x * kCols;
    if (q.rows == 0) return;
    if (q.expert < 0) {
        const int i = threadIdx.x / kCols, c = n0 + threadIdx.x % kCols;
        if (i < q.rows && c < g.n) static_cast<T *>(g.c)[(q.row + i) * g.c_m + c] = from_float<T>(0.0f);
    } else if (q.rows == 1) {
        column_rows<T, V, 1>(g, q, n0, part);
    } else if (q.rows == 2) {
        column_rows<T, V, 2>(g, q, n0, part);
    } else if (q.rows == 3) {
        column_rows<T, V, 3>(g, q, n0, part);
    } else {
        column_rows<T, V, 4>(g, q, n0, part);
    }
}

}  // namespace

cudaError_t expert_few_rows(int dtype, const ExpertArgs &g, cudaStream_t stream)
{
    const int bytes = dtype_bytes(dtype), v = 16 / bytes;
    const bool dot = g.b_r == 1;
    const int64_t stride = dot ? g.b_n : g.b_r;
    bool wide = aligned16(g.b) && stride % v == 0 && (g.experts == 1 || g.b_e % v == 0);
    if (dot) wide = wide && aligned16(g.a) && g.r % v == 0 && (g.rows == 1 || g.a_m % v == 0);
    else wide = wide && g.n % v == 0;
    const dim3 grid(unsigned(dot ? (g.n + kWarps * kFeatures - 1) / (kWarps * kFeatures) : (g.n + kCols - 1) / kCols),
                    unsigned(g.rows));
    DC_DTYPE_SWITCH(dtype, T, {
        constexpr int V = kVec<T>;
        if (dot) {
            if (wide) few_dot_kernel<T, V><<<grid, kThreads, 0, stream>>>(g);
            else few_dot_kernel<T, 1><<<grid, kThreads, 0, stream>>>(g);
        } else {
            if (wide) few_column_kernel<T, V><<<grid, kColumnThreads, 0, stream>>>(g);
            else few_column_kernel<T, 1><<<grid, kColumnThreads, 0, stream>>>(g);
        }
        return cudaGetLastError();
    })
}

}  // namespace dc
