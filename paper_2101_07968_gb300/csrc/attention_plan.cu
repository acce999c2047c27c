// Attention: the list of tiles, the row sums of the gradient, and which kernels run.
#include "attention.cuh"

namespace dc {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kBuckets = 512;  // of work: the order within one is of no account

// inclusive scans of a block, by sum or by maximum
template <bool MAX>
__device__ __forceinline__ int scan(int v, int *warps)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto join = [](int x, int y) { return MAX ? max(x, y) : x + y; };
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const int t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v = join(v, t);
    }
    __syncthreads();  // the last scan's reads
    if (lane == 31) warps[warp] = v;
    __syncthreads();
    if (warp == 0) {
        int t = warps[lane];
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int s = __shfl_up_sync(0xffffffffu, t, o);
            if (lane >= o) t = join(t, s);
        }
        warps[lane] = t;
    }
    __syncthreads();
    return warp ? join(v, warps[warp - 1]) : v;
}

// One block. first [sequences + 3] tiles before each segment, start [sequences + 3] its first row:
// segment 0 are the rows before the first sequence, segment sequences + 1 those after the last.
// An offset outside [0, tokens], or below an earlier one, counts as the nearest valid value.
// Tiles come in order of falling work, which is a tile's number in its sequence.
__global__ void __launch_bounds__(kPlanThreads)
attention_plan_kernel(const int64_t *offsets, int32_t sequences, int64_t tokens, int32_t rows, AttentionPlan *plan,
                      int32_t *first, int32_t *start)
{
    __shared__ int warps[32], count[kBuckets], carry[2];
    const int segments = sequences + 2;
    if (threadIdx.x < 2) carry[threadIdx.x] = 0;
    if (threadIdx.x < kBuckets) count[threadIdx.x] = 0;
    __syncthreads();
    // start[i] for i = 0 .. segments: 0, the offsets, tokens
    int longest = 0;
    for (int i0 = 0; i0 <= segments; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        int64_t v = i == 0 ? 0 : i <= sequences + 1 ? offsets[i - 1] : tokens;
        v = min(max(v, int64_t(0)), tokens);
        const int at = max(scan<true>(int(v), warps), carry[0]);
        if (i <= segments) start[i] = at;
        __syncthreads();
        if (threadIdx.x == kPlanThreads - 1) carry[0] = at;
        __syncthreads();
    }
    for (int i0 = 0; i0 < segments; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        const int n = i < segments ? (start[i + 1] - start[i] + rows - 1) / rows : 0;
        if (i > 0 && i < segments - 1) longest = max(longest, n);
        const int sum = scan<false>(n, warps) + carry[1];
        if (i < segments) first[i + 1] = sum;
        if (i == 0) first[0] = 0;
        __syncthreads();
        if (threadIdx.x == kPlanThreads - 1) carry[1] = sum;
        __syncthreads();
    }
    const int tiles = carry[1];
    longest = scan<true>(longest, warps);
    __syncthreads();
    if (threadIdx.x == kPlanThreads - 1) carry[0] = longest;
    __syncthreads();
    longest = max(carry[0], 1);
    AttentionTile *list = reinterpret_cast<AttentionTile *>(plan + 1);
    // twice over the tiles: how many of each bucket, then where they go
    for (int pass = 0; pass < 2; ++pass) {
        for (int t = threadIdx.x; t < tiles; t += kPlanThreads) {
            int lo = 0, hi = segments;  // first[lo] <= t < first[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if (first[mid] <= t) lo = mid;
                else hi = mid;
            }
            const int i = t - first[lo];
            const bool none = lo == 0 || lo == segments - 1;
            const int work = none ? 0 : i + 1;
            const int bucket = int(int64_t(longest - min(work, longest)) * (kBuckets - 1) / longest);
            const int at = atomicAdd(&count[bucket], 1);
            if (pass) {
                AttentionTile q;
                q.row0 = start[lo] + i * rows;
                q.rows = min(rows, start[lo + 1] - q.row0);
                q.first = none ? -1 : start[lo];
                q.end = start[lo + 1];
                list[at] = q;
            }
        }
        __syncthreads();
        if (pass == 0) {
            const int mine = threadIdx.x < kBuckets ? count[threadIdx.x] : 0;
            const int up_to = scan<false>(mine, warps);
            if (threadIdx.x < kBuckets) count[threadIdx.x] = up_to - mine;
            __syncthreads();
        }
    }
    if (threadIdx.x == 0) plan->tiles = tiles;
}

// delta[h][t] = sum over d of dy y, a warp per row.
template <typename T>
__global__ void __launch_bounds__(256) attention_delta_kernel(const AttentionArgs a)
{
    const int64_t i = int64_t(blockIdx.x) * 8 + threadIdx.x / 32;
    if (i >= a.tokens * a.heads) return;
    const int64_t t = i / a.heads;
    const int h = int(i - t * a.heads), lane = threadIdx.x % 32;
    const T *y = static_cast<const T *>(a.y) + i * a.D;
    const T *dy = static_cast<const T *>(a.dy) + t * a.dy_token + h * a.dy_head;
    float s = 0.0f;
    for (int d = lane; d < a.D; d += 32) s += to_float(y[d]) * to_float(dy[d]);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) a.delta[h * a.tokens + t] = s;
}

// The tensor cores' copies need heads that start on 16-byte boundaries: others are copied to rows of
// whole 16 bytes first, eight elements a thread.
struct Heads {
    const void *p;
    int64_t token, head;
    int32_t heads;
};
int64_t padded(int32_t D) { return (int64_t(D) + 7) / 8 * 8; }
bool aligned(const Heads &h, int64_t tokens)
{
    return aligned16(h.p) && (tokens == 1 || h.token % 8 == 0) && (h.heads == 1 || h.head % 8 == 0);
}
__global__ void __launch_bounds__(256)
align_heads_kernel(const uint16_t *x, uint16_t *to, int64_t units, int32_t heads, int32_t D, int32_t per, int64_t token,
                   int64_t head)
{
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= units) return;
    const int64_t row = i / per, t = row / heads;
    const int d = int(i - row * per) * 8;
    const uint16_t *p = x + t * token + (row - t * heads) * head + d;
    Vec<uint16_t, 8> v;
#pragma unroll
    for (int j = 0; j < 8; ++j) v.e[j] = d + j < D ? p[j] : uint16_t(0);
    *reinterpret_cast<Vec<uint16_t, 8> *>(to + i * 8) = v;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

Heads operand(const AttentionArgs &a, int i)
{
    switch (i) {
        case 0: return {a.q, a.q_token, a.q_head, a.heads};
        case 1: return {a.k, a.k_token, a.k_head, a.kv_heads};
        case 2: return {a.v, a.v_token, a.v_head, a.kv_heads};
        default: return {a.dy, a.dy_token, a.dy_head, a.heads};
    }
}

// Parts of the workspace; copy[i]: of operand i, where it needs one.
struct Layout {
    int rows;  // of a tile
    size_t first, start, delta, copy[4], total;
    bool copied[4];
};
Layout layout(int dtype, const AttentionArgs &a, int32_t sequences, bool grad)
{
    Layout l = {};
    l.rows = dtype == DC_FP32 || grad ? kSimtRows : attention_mma_rows(a);
    size_t at = round256(sizeof(AttentionPlan) +
                         sizeof(AttentionTile) * size_t(attention_most_tiles(a.tokens, sequences, l.rows)));
    l.first = at;
    at += round256(sizeof(int32_t) * (size_t(sequences) + 3));
    l.start = at;
    at += round256(sizeof(int32_t) * (size_t(sequences) + 3));
    l.delta = at;
    if (grad) at += round256(sizeof(float) * size_t(a.heads) * size_t(a.tokens));
    for (int i = 0; i < (grad ? 4 : 3) && dtype != DC_FP32; ++i) {
        const Heads h = operand(a, i);
        l.copied[i] = !aligned(h, a.tokens);
        l.copy[i] = at;
        if (l.copied[i]) at += round256(size_t(a.tokens) * h.heads * padded(a.D) * 2);
    }
    l.total = at;
    return l;
}

cudaError_t align_operands(AttentionArgs &a, const Layout &l, unsigned char *ws, cudaStream_t stream)
{
    for (int i = 0; i < 4; ++i) {
        if (!l.copied[i]) continue;
        const Heads h = operand(a, i);
        const int64_t pad = padded(a.D), units = a.tokens * h.heads * (pad / 8), blocks = (units + 255) / 256;
        if (blocks > (int64_t(1) << 31) - 1) return cudaErrorInvalidValue;
        uint16_t *to = reinterpret_cast<uint16_t *>(ws + l.copy[i]);
        align_heads_kernel<<<unsigned(blocks), 256, 0, stream>>>(static_cast<const uint16_t *>(h.p), to, units, h.heads, a.D,
                                                                 int(pad / 8), h.token, h.head);
        const void **p[4] = {&a.q, &a.k, &a.v, &a.dy};
        int64_t *token[4] = {&a.q_token, &a.k_token, &a.v_token, &a.dy_token};
        int64_t *head[4] = {&a.q_head, &a.k_head, &a.v_head, &a.dy_head};
        *p[i] = to;
        *token[i] = h.heads * pad;
        *head[i] = pad;
    }
    return cudaSuccess;
}

}  // namespace

size_t attention_workspace(int dtype, const AttentionArgs &a, int32_t sequences, bool grad)
{
    return layout(dtype, a, sequences, grad).total;
}

cudaError_t launch_attention(int dtype, AttentionArgs a, int32_t sequences, const int64_t *offsets, bool grad,
                             void *workspace, cudaStream_t stream)
{
    const Layout l = layout(dtype, a, sequences, grad);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    AttentionPlan *plan = reinterpret_cast<AttentionPlan *>(ws);
    attention_plan_kernel<<<1, kPlanThreads, 0, stream>>>(offsets, sequences, a.tokens, l.rows, plan,
                                                          reinterpret_cast<int32_t *>(ws + l.first),
                                                          reinterpret_cast<int32_t *>(ws + l.start));
    a.plan = plan;
    const int64_t most = attention_most_tiles(a.tokens, sequences, l.rows);
    if (!grad) {
        if (dtype == DC_FP32) return launch_attention_simt(dtype, a, most, stream);
        const cudaError_t e = align_operands(a, l, ws, stream);
        return e == cudaSuccess ? launch_attention_mma(dtype, a, most, stream) : e;
    }
    a.delta = reinterpret_cast<float *>(ws + l.delta);
    const int64_t blocks = (a.tokens * a.heads + 7) / 8;
    if (blocks > (int64_t(1) << 31) - 1) return cudaErrorInvalidValue;
    switch (dtype) {
        case DC_BF16: attention_delta_kernel<__nv_bfloat16><<<unsigned(blocks), 256, 0, stream>>>(a); break;
        case DC_FP16: attention_delta_kernel<__half><<<unsigned(blocks), 256, 0, stream>>>(a); break;
        default: attention_delta_kernel<float><<<unsigned(blocks), 256, 0, stream>>>(a);
    }
    return launch_attention_grad_simt(dtype, a, most, stream);
}

}  // namespace dc
