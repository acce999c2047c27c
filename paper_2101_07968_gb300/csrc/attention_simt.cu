// Attention of floats, on the CUDA cores.
//
// Forward, a block per tile of 64 rows and head: keys 64 at a time; scores S = scale q k^T, the
// running maximum m and sum l of each row, and y = sum e^(S - m) v / l, kept in registers.
// Gradient, with P = e^(S - lse) and dS = P (dy v^T - delta):
//   rows     a tile of 64 rows and a head, over the keys up to it: dq = scale dS k
//   columns  a tile of 64 keys and a key head, over its group's heads and the rows from it on:
//            dv = P^T dy, dk = scale dS^T q
// Each sum has one owner and one order: no atomics. Where tiles and key heads are few, a group's heads are
// dealt to several blocks, whose sums are joined afterwards (attention_plan.cu). What a mask leaves out is skipped, not
// multiplied by zero, so that whatever stands there is without effect.
//
// 256 threads, 4 x 4 scores a thread. Rows of operands lie in shared memory four floats apart from
// whole banks' multiples, so that threads read four neighbouring elements of 16 rows without
// conflicts: eight such reads feed 64 products. The next block's operands come by asynchronous copies
// as soon as the last product with this one's is done. 2,000 tokens in 3 sequences x 8 heads on 2 x 64: 112 us forward,
// rows 149, columns 193, bound by the longest item's 16 blocks one after another.
#include "attention.cuh"

namespace dc {
namespace {

constexpr int kThreads = 256, kTile = kSimtRows;
constexpr int kScorePitch = kTile + 4;

template <int DP>
constexpr int kPitch = DP + 4;

// Rows 0 .. rows of x [token][D] to shared memory; zeros beyond rows and D. `wide`: four elements a copy. The
// copies are one group of the thread's (copies_wait).
template <int DP>
__device__ __forceinline__ void bring(float *to, const float *x, int64_t stride, int rows, int D, bool wide)
{
    if (wide) {
#pragma unroll
        for (int i = threadIdx.x * 4; i < kTile * DP; i += kThreads * 4) {
            const int r = i / DP, d = i % DP;
            const bool there = r < rows && d < D;
            const uint32_t at = uint32_t(__cvta_generic_to_shared(to + r * kPitch<DP> + d));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(there ? x + r * stride + d : x),
                         "r"(there ? 16 : 0)
                         : "memory");
        }
    } else {
        for (int i = threadIdx.x; i < kTile * DP; i += kThreads) {
            const int r = i / DP, d = i % DP;
            to[r * kPitch<DP> + d] = r < rows && d < D ? x[r * stride + d] : 0.0f;
        }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}
// All but the last N groups have arrived, of every thread.
template <int N>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncthreads();
}
inline bool runs_of_four(const void *p, int64_t token, int64_t head, int D)
{
    return D % 4 == 0 && aligned16(p) && token % 4 == 0 && head % 4 == 0;
}

// s[i][j] = sum over d of x[ty + 16 i][d] z[tx + 16 j][d]
template <int DP>
__device__ __forceinline__ void scores(const float *x, const float *z, float (&s)[4][4])
{
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
#pragma unroll 2
    for (int d = 0; d < DP; d += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = *reinterpret_cast<const float4 *>(x + (ty + 16 * i) * kPitch<DP> + d);
            b[i] = *reinterpret_cast<const float4 *>(z + (tx + 16 * i) * kPitch<DP> + d);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                s[i][j] += a[i].x * b[j].x + a[i].y * b[j].y + a[i].z * b[j].z + a[i].w * b[j].w;
    }
}

// acc[i][4 m + e] += sum over columns c of p[ty + 16 i][c] z[c][4 tx + 64 m + e]; MASKED: only over the columns
// that the row's mask lets through, from lo(i) up to hi(i).
template <int DP, bool MASKED, typename Lo, typename Hi>
__device__ __forceinline__ void add_product(const float *p, const float *z, float (&acc)[4][DP / 16], Lo lo, Hi hi)
{
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll 2
    for (int c0 = 0; c0 < kTile; c0 += 4) {
        float4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const float4 *>(p + (ty + 16 * i) * kScorePitch + c0);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int m = 0; m < DP / 64; ++m) {
                const float4 b = *reinterpret_cast<const float4 *>(z + (c0 + k) * kPitch<DP> + 4 * tx + 64 * m);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (MASKED && (c0 + k < lo(i) || c0 + k >= hi(i))) continue;
                    const float x = k == 0 ? w[i].x : k == 1 ? w[i].y : k == 2 ? w[i].z : w[i].w;
                    acc[i][4 * m] += x * b.x;
                    acc[i][4 * m + 1] += x * b.y;
                    acc[i][4 * m + 2] += x * b.z;
                    acc[i][4 * m + 3] += x * b.w;
                }
            }
    }
}

// Rows of a tile to [token][heads][D]
template <typename T, int DP>
__device__ __forceinline__ void put(T *y, int64_t stride, int rows, int D, const float (&acc)[4][DP / 16],
                                    const float (&by)[4])
{
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty + 16 * i;
        if (r >= rows) continue;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) {
            const int d = 4 * tx + 64 * (j / 4) + j % 4;
            if (d < D) y[r * stride + d] = from_float<T>(acc[i][j] * by[i]);
        }
    }
}

template <typename T>
__device__ __forceinline__ void put_zeros(T *y, int64_t stride, int rows, int D)
{
    for (int i = threadIdx.x; i < rows * D; i += kThreads) y[i / D * stride + i % D] = from_float<T>(0.0f);
}

template <int DP>
__global__ void __launch_bounds__(kThreads) attention_simt_kernel(const AttentionArgs a, const bool wide)
{
    extern __shared__ __align__(16) float dyn[];
    constexpr int kSize = kTile * kPitch<DP>;
    float *q = dyn, *k = q + kSize, *v = k + kSize, *p = v + kSize;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int64_t items = int64_t(a.plan->tiles) * a.heads;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const AttentionTile t = plan_tiles(a.plan)[item / a.heads];
        const int h = int(item % a.heads), g = h / a.group;
        const int64_t out = int64_t(a.heads) * a.D;
        float *y = static_cast<float *>(a.y) + t.row0 * out + int64_t(h) * a.D;
        if (t.first < 0) {
            put_zeros(y, out, t.rows, a.D);
            for (int r = threadIdx.x; r < t.rows; r += kThreads) a.lse[h * a.tokens + t.row0 + r] = 0.0f;
            continue;
        }
        const int hi = t.row0 + t.rows;
        auto keys = [&](int c0) {
            bring<DP>(k, static_cast<const float *>(a.k) + c0 * a.k_token + g * a.k_head, a.k_token, min(kTile, hi - c0), a.D, wide);
        };
        auto values = [&](int c0) {
            bring<DP>(v, static_cast<const float *>(a.v) + c0 * a.v_token + g * a.v_head, a.v_token, min(kTile, hi - c0), a.D, wide);
        };
        __syncthreads();
        bring<DP>(q, static_cast<const float *>(a.q) + t.row0 * a.q_token + h * a.q_head, a.q_token, t.rows, a.D, wide);
        keys(t.first);
        values(t.first);
        float m[4], l[4] = {}, acc[4][DP / 16] = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = -INFINITY;
        for (int c0 = t.first; c0 < hi; c0 += kTile) {
            const bool last = c0 + kTile >= hi;
            copies_wait<1>();  // this block's keys
            float s[4][4];
            scores<DP>(q, k, s);
            __syncthreads();
            if (!last) keys(c0 + kTile);
            const int n = hi - c0;
            auto end = [&](int i) { return min(n, t.row0 + ty + 16 * i - c0 + 1); };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s[i][j] = !last || tx + 16 * j < end(i) ? s[i][j] * a.scale : -INFINITY;
                    top = fmaxf(top, s[i][j]);
                }
#pragma unroll
                for (int o = 8; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float next = fmaxf(m[i], top);
                // nothing but -inf so far: any finite reference will do
                const float from = next == -INFINITY ? 0.0f : next;
                const float old = expf(m[i] - from);
                float sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = !last || tx + 16 * j < end(i) ? expf(s[i][j] - from) : 0.0f;
                    sum += e;
                    p[(ty + 16 * i) * kScorePitch + tx + 16 * j] = e;
                }
#pragma unroll
                for (int o = 8; o > 0; o /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                l[i] = l[i] * old + sum;
                m[i] = next;
#pragma unroll
                for (int j = 0; j < DP / 16; ++j) acc[i][j] *= old;
            }
            if (last) {
                copies_wait<0>();
                add_product<DP, true>(p, v, acc, [](int) { return 0; }, end);
            } else {
                copies_wait<1>();  // this block's values
                add_product<DP, false>(p, v, acc, [](int) { return 0; }, end);
                __syncthreads();
                values(c0 + kTile);
            }
        }
        float by[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            by[i] = 1.0f / l[i];
            if (tx == 0 && ty + 16 * i < t.rows) a.lse[h * a.tokens + t.row0 + ty + 16 * i] = m[i] + logf(l[i]);
        }
        put<float, DP>(y, out, t.rows, a.D, acc, by);
    }
}

// One pair of tiles of the gradient: x0, x1 (64 stationary rows: q and dy, or k and v), z0, z1 (64
// moving ones: k and v, or q and dy; z0 twice, since its last product ends a step).
template <int DP, bool COLUMNS>
__global__ void __launch_bounds__(kThreads) attention_grad_simt_kernel(const AttentionArgs a, const bool wide)
{
    extern __shared__ __align__(16) float dyn[];
    constexpr int kSize = kTile * kPitch<DP>;
    float *x0 = dyn, *x1 = x0 + kSize, *z1 = x1 + kSize, *z0s = z1 + kSize, *p = z0s + 2 * kSize;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int outer = COLUMNS ? a.kv_heads * a.split : a.heads;
    const int64_t items = int64_t(a.plan->tiles) * outer;
    const float *q = static_cast<const float *>(a.q), *k = static_cast<const float *>(a.k), *v = static_cast<const float *>(a.v);
    const float *dy = static_cast<const float *>(a.dy);
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        AttentionTile t = plan_tiles(a.plan)[item / outer];
        const int part = COLUMNS ? int(item % outer) / a.kv_heads : 0;
        const int o = COLUMNS ? int(item % outer) % a.kv_heads : int(item % outer), g = COLUMNS ? o : o / a.group;
        const int64_t out = int64_t(COLUMNS ? a.kv_heads : a.heads) * a.D;
        if (COLUMNS && t.first >= 0) {  // tile i from the end has the work of tile i from the start
            const int n = (t.end - t.first + kTile - 1) / kTile, i = n - 1 - (t.row0 - t.first) / kTile;
            t.row0 = t.first + i * kTile;
            t.rows = min(kTile, t.end - t.row0);
        }
        const int64_t at = t.row0 * out + int64_t(o) * a.D, all = a.tokens * out;
        // a part's sums, or the gradients themselves
        float *const d0 = !COLUMNS ? static_cast<float *>(a.dq) + at
                          : a.split > 1 ? a.partial + part * all + at
                                        : static_cast<float *>(a.dk) + at;
        float *const d1 = !COLUMNS ? nullptr
                          : a.split > 1 ? a.partial + (a.split + part) * all + at
                                        : static_cast<float *>(a.dv) + at;
        if (t.first < 0) {
            put_zeros(d0, out, t.rows, a.D);
            if (COLUMNS) put_zeros(d1, out, t.rows, a.D);
            continue;
        }
        const int h0 = COLUMNS ? g * a.group + part * a.group / a.split : o;
        const int h1 = COLUMNS ? g * a.group + (part + 1) * a.group / a.split : o + 1;
        const int lo = COLUMNS ? t.row0 : t.first, hi = COLUMNS ? t.end : t.row0 + t.rows;
        const int per = (hi - lo + kTile - 1) / kTile, steps = per * (h1 - h0);
        auto first_of = [&](int i, float *to) {
            const int h = h0 + i / per, c0 = lo + i % per * kTile, n = min(kTile, hi - c0);
            if (COLUMNS)
                bring<DP>(to, q + c0 * a.q_token + h * a.q_head, a.q_token, n, a.D, wide);
            else
                bring<DP>(to, k + c0 * a.k_token + g * a.k_head, a.k_token, n, a.D, wide);
        };
        auto second_of = [&](int i) {
            const int h = h0 + i / per, c0 = lo + i % per * kTile, n = min(kTile, hi - c0);
            if (COLUMNS)
                bring<DP>(z1, dy + c0 * a.dy_token + h * a.dy_head, a.dy_token, n, a.D, wide);
            else
                bring<DP>(z1, v + c0 * a.v_token + g * a.v_head, a.v_token, n, a.D, wide);
        };
        __syncthreads();
        float acc0[4][DP / 16] = {}, acc1[4][COLUMNS ? DP / 16 : 1] = {};
        if (COLUMNS) {
            bring<DP>(x0, k + t.row0 * a.k_token + g * a.k_head, a.k_token, t.rows, a.D, wide);
            bring<DP>(x1, v + t.row0 * a.v_token + g * a.v_head, a.v_token, t.rows, a.D, wide);
        } else {
            bring<DP>(x0, q + t.row0 * a.q_token + o * a.q_head, a.q_token, t.rows, a.D, wide);
            bring<DP>(x1, dy + t.row0 * a.dy_token + o * a.dy_head, a.dy_token, t.rows, a.D, wide);
        }
        first_of(0, z0s);
        second_of(0);
        for (int step = 0; step < steps; ++step) {
            const int h = h0 + step / per, c0 = lo + step % per * kTile, n = min(kTile, hi - c0);
            float *const z0 = z0s + (step & 1) * kSize;
            copies_wait<0>();
            if (step + 1 < steps) first_of(step + 1, z0s + (~step & 1) * kSize);
            float s[4][4], ds[4][4];
            scores<DP>(x0, z0, s);
            scores<DP>(x1, z1, ds);
            // columns of row i that count: keys up to it, or rows from the key on
            auto from = [&](int i) { return COLUMNS ? t.row0 + ty + 16 * i - c0 : 0; };
            auto end = [&](int i) { return COLUMNS ? n : min(n, t.row0 + ty + 16 * i - c0 + 1); };
            const bool cut = COLUMNS ? c0 == t.row0 || n < kTile : c0 + kTile > t.row0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = tx + 16 * j, r = ty + 16 * i;
                    const int64_t row = h * a.tokens + (COLUMNS ? c0 + c : t.row0 + r);
                    if (c >= from(i) && c < end(i) && r < t.rows) {
                        s[i][j] = expf(s[i][j] * a.scale - a.lse[row]);
                        ds[i][j] = s[i][j] * (ds[i][j] - a.delta[row]);
                    } else {
                        s[i][j] = ds[i][j] = 0.0f;
                    }
                    if (COLUMNS) p[r * kScorePitch + c] = s[i][j];
                }
            if constexpr (COLUMNS) {
                __syncthreads();
                if (cut) add_product<DP, true>(p, z1, acc1, from, end);
                else add_product<DP, false>(p, z1, acc1, from, end);
            }
            __syncthreads();  // z1 and P have been read
            if (step + 1 < steps) second_of(step + 1);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) p[(ty + 16 * i) * kScorePitch + tx + 16 * j] = ds[i][j];
            __syncthreads();
            if (cut) add_product<DP, true>(p, z0, acc0, from, end);
            else add_product<DP, false>(p, z0, acc0, from, end);
        }
        const float by0[4] = {a.scale, a.scale, a.scale, a.scale}, by1[4] = {1.0f, 1.0f, 1.0f, 1.0f};
        put<float, DP>(d0, out, t.rows, a.D, acc0, by0);
        if constexpr (COLUMNS) put<float, DP>(d1, out, t.rows, a.D, acc1, by1);
    }
}

template <int DP, typename K>
cudaError_t go(K kernel, DeviceCache &cache, int tiles, const AttentionArgs &a, int64_t items, bool wide, cudaStream_t stream)
{
    const int smem = int(sizeof(float)) * (tiles * kTile * kPitch<DP> + kTile * kScorePitch);
    int ready = 0;
    const cudaError_t e = cache.get(ready, [&](int &v) {
        v = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    });
    if (e != cudaSuccess) return e;
    const int64_t limit = int64_t(1) << 20;
    kernel<<<unsigned(items < limit ? items : limit), kThreads, smem, stream>>>(a, wide);
    return cudaGetLastError();
}

bool all_wide(const AttentionArgs &a, bool grad)
{
    return runs_of_four(a.q, a.q_token, a.q_head, a.D) && runs_of_four(a.k, a.k_token, a.k_head, a.D) &&
           runs_of_four(a.v, a.v_token, a.v_head, a.D) && (!grad || runs_of_four(a.dy, a.dy_token, a.dy_head, a.D));
}

template <int DP>
cudaError_t forward(const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    static DeviceCache cache;
    return go<DP>(attention_simt_kernel<DP>, cache, 3, a, most * a.heads, all_wide(a, false), stream);
}

template <int DP, bool COLUMNS>
cudaError_t backward(const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    static DeviceCache cache;
    return go<DP>(attention_grad_simt_kernel<DP, COLUMNS>, cache, 5, a, most * (COLUMNS ? a.kv_heads * a.split : a.heads),
                  all_wide(a, true), stream);
}

}  // namespace

cudaError_t launch_attention_simt(const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    return a.D <= 64 ? forward<64>(a, most, stream) : forward<128>(a, most, stream);
}

cudaError_t launch_attention_grad_simt(const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    cudaError_t e = a.D <= 64 ? backward<64, true>(a, most, stream) : backward<128, true>(a, most, stream);
    if (e == cudaSuccess)
        e = a.D <= 64 ? backward<64, false>(a, most, stream) : backward<128, false>(a, most, stream);
    return e;
}

}  // namespace dc
