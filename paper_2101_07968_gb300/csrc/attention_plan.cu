// Attention: the list of tiles, the row sums of the gradient, and which kernels run.
#include <type_traits>

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
    pdl_trigger();  // a kernel after this one gets ready while the list is made
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

// The powers of two that dS of halves is held in, one of each row (of a head) and of each key (of a key head): a lane's
// scale leaves with its sums. They follow from bounds of what that output may see, and of nothing else, so that
// whatever stands in other sequences, other heads or behind the mask does not change a bit:
//   |dS_ij| <= |dy_i| |v_j| + r_i,  r_i = |dy_i . y_i| + |dy_i| (2^-8 |y_i| + 2^-20)
// with lengths of heads; r_i covers delta_i with y's rounding taken back. A row takes the largest |v_j| of the keys
// up to it, a key the largest |dy_i| and r_i of the rows from it on, of its group's heads. Both are maxima over
// a part of a sequence: of rows of 128 tokens (chunks) where they are whole, of single ones at its ends.
constexpr int kChunk = 128;
struct GradSizes {
    float *dy_norm, *row_bound;               // [heads][tokens]: |dy_i|, r_i
    float *v_norm;                            // [kv_heads][tokens]
    uint32_t *top_v, *top_dy, *top_row;       // their largest of a chunk (and a group's heads), float bits: [kv_heads][chunks]
    int8_t *row_power, *key_power;
    int32_t chunks;
};
// Magnitudes' bits are in the order of their values; NaN above all.
__device__ __forceinline__ uint32_t most_of_group(const AttentionArgs &a, const float *of, int g, int64_t t)
{
    uint32_t m = 0;
    for (int h = g * a.group; h < (g + 1) * a.group; ++h) m = max(m, __float_as_uint(of[h * a.tokens + t]));
    return m;
}
__device__ __forceinline__ uint32_t most_of_block(uint32_t v, uint32_t *warps)
{
    v = __reduce_max_sync(0xffffffffu, v);
    __syncthreads();  // the last one's reads
    if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = v;
    __syncthreads();
    return max(max(warps[0], warps[1]), max(warps[2], warps[3]));
}
__global__ void __launch_bounds__(kChunk)
attention_chunks_kernel(const AttentionArgs a, const GradSizes z, const int32_t *start, int32_t sequences)
{
    __shared__ uint32_t warps[4];
    pdl_trigger();
    pdl_wait();  // delta's kernel: the lengths
    const int64_t lo = start[1], hi = start[sequences + 1], items = int64_t(z.chunks) * a.kv_heads;
    for (int64_t i = blockIdx.x; i < items; i += gridDim.x) {
        const int g = int(i / z.chunks);
        const int64_t t = (i - int64_t(g) * z.chunks) * kChunk + threadIdx.x;
        const bool counts = t >= lo && t < hi;
        const uint32_t v = most_of_block(counts ? __float_as_uint(z.v_norm[g * a.tokens + t]) : 0, warps);
        const uint32_t dy = most_of_block(counts ? most_of_group(a, z.dy_norm, g, t) : 0, warps);
        const uint32_t row = most_of_block(counts ? most_of_group(a, z.row_bound, g, t) : 0, warps);
        if (threadIdx.x == 0) {
            z.top_v[i] = v;
            z.top_dy[i] = dy;
            z.top_row[i] = row;
        }
    }
}
// 2^15 is above bound times it: half of what halves reach, for the rounding of all that the bound is made of
__device__ __forceinline__ int8_t power_for(float bound)
{
    return bound > 0.0f && bound < INFINITY ? int8_t(min(max(14 - ilogbf(bound), -96), 96)) : int8_t(0);
}
// A tile of 128 rows and a key head, a thread a token.
__global__ void __launch_bounds__(kChunk) attention_powers_kernel(const AttentionArgs a, const GradSizes z)
{
    __shared__ uint32_t warps[4];
    pdl_wait();  // the chunks
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // the largest of tokens [lo, hi), by the whole block
    auto most = [&](int lo, int hi, auto of, const uint32_t *chunks) {
        uint32_t m = 0;
        const int c0 = (lo + kChunk - 1) / kChunk, c1 = hi / kChunk;
        const int end = c0 < c1 ? c0 * kChunk : hi;
        for (int t = lo + threadIdx.x; t < end; t += kChunk) m = max(m, of(t));
        if (c0 < c1) {
            for (int c = c0 + threadIdx.x; c < c1; c += kChunk) m = max(m, chunks[c]);
            for (int t = c1 * kChunk + threadIdx.x; t < hi; t += kChunk) m = max(m, of(t));
        }
        return most_of_block(m, warps);
    };
    // of this thread's value and those before it, or behind it
    auto scan = [&](uint32_t v, bool behind) {
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const uint32_t t = behind ? __shfl_down_sync(0xffffffffu, v, o) : __shfl_up_sync(0xffffffffu, v, o);
            if (behind ? lane + o < 32 : lane >= o) v = max(v, t);
        }
        __syncthreads();
        if (lane == (behind ? 0 : 31)) warps[warp] = v;
        __syncthreads();
        for (int w = 0; w < 4; ++w)
            if (behind ? w > warp : w < warp) v = max(v, warps[w]);
        return v;
    };
    const int64_t items = int64_t(a.plan->tiles) * a.kv_heads;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const AttentionTile q = plan_tiles(a.plan)[item / a.kv_heads];
        if (q.first < 0) continue;
        const int g = int(item % a.kv_heads), t = q.row0 + threadIdx.x;
        const int64_t at = g * a.tokens, chunk = int64_t(g) * z.chunks;
        const bool there = int(threadIdx.x) < q.rows;
        auto value = [&](int64_t i) { return __float_as_uint(z.v_norm[at + i]); };
        auto gradient = [&](int64_t i) { return most_of_group(a, z.dy_norm, g, i); };
        auto row = [&](int64_t i) { return most_of_group(a, z.row_bound, g, i); };
        const uint32_t mine = there ? value(t) : 0;
        uint32_t v = most(q.first, q.row0, value, z.top_v + chunk);
        v = max(v, scan(mine, false));
        uint32_t dy = most(q.row0 + q.rows, q.end, gradient, z.top_dy + chunk);
        dy = max(dy, scan(there ? gradient(t) : 0, true));
        uint32_t r = most(q.row0 + q.rows, q.end, row, z.top_row + chunk);
        r = max(r, scan(there ? row(t) : 0, true));
        if (!there) continue;
        z.key_power[at + t] = power_for(__uint_as_float(dy) * __uint_as_float(mine) + __uint_as_float(r));
        for (int h = g * a.group; h < (g + 1) * a.group; ++h) {
            const int64_t i = h * a.tokens + t;
            z.row_power[i] = power_for(z.dy_norm[i] * __uint_as_float(v) + z.row_bound[i]);
        }
    }
}

// delta[h][t] = sum over d of dy y: LANES lanes a row of a head, sixteen bytes a lane at a time (32,768 tokens x 32
// heads x 128: 104 us, 5.2 TB/s; two or four rows on their way at once, or neighbouring tokens a block: no less). Eight
// lanes where they hold a row, else sixteen. Halves: also the lengths and bounds that dS's powers of two follow from.
template <typename T, bool WIDE, int LANES>
__global__ void __launch_bounds__(256) attention_delta_kernel(const AttentionArgs a, const GradSizes z, const int32_t *start,
                                                              int32_t sequences)
{
    constexpr bool kHalf = std::is_same<T, __half>::value;
    constexpr int V = kVec<T>;
    // the same elements to a lane whether they come in one access or not: the same bits
    auto bring = [&](const T *p, int left) {
        if (WIDE) return *reinterpret_cast<const Vec<T, V> *>(p);
        Vec<T, V> v;
#pragma unroll
        for (int j = 0; j < V; ++j) v.e[j] = j < left ? p[j] : from_float<T>(0.0f);
        return v;
    };
    constexpr int kRows = 256 / LANES;  // of a block at a time
    const int64_t rows = a.tokens * a.heads, step = int64_t(gridDim.x) * kRows;
    const int l = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const uint32_t lanes = ((1u << LANES) - 1) << (threadIdx.x % 32 / LANES * LANES);
    auto sum = [&](float s) {  // over the row's lanes
#pragma unroll
        for (int o = LANES / 2; o > 0; o /= 2) s += __shfl_xor_sync(lanes, s, o);
        return s;
    };
    for (int64_t i = int64_t(blockIdx.x) * kRows + group; i < rows; i += step) {
        const int64_t t = rows < (int64_t(1) << 31) ? int64_t(uint32_t(i) / uint32_t(a.heads)) : i / a.heads;
        const T *y = static_cast<const T *>(a.y) + i * a.D;
        const T *dy = static_cast<const T *>(a.dy) + t * a.dy_token + (i - t * a.heads) * a.dy_head;
        float s = 0.0f, s_dy = 0.0f, s_y = 0.0f;
        for (int d = l * V; d < a.D; d += LANES * V) {
            const Vec<T, V> p = bring(y + d, a.D - d), q = bring(dy + d, a.D - d);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float e = to_float(p.e[j]), g = to_float(q.e[j]);
                s += e * g;
                if (kHalf) {
                    s_dy += g * g;
                    s_y += e * e;
                }
            }
        }
        s = sum(s);
        const int64_t at = (i - t * a.heads) * a.tokens + t;
        if (l == 0) a.delta[at] = s;
        if constexpr (kHalf) {
            const float dy_norm = sqrtf(sum(s_dy)), y_norm = sqrtf(sum(s_y));
            if (l == 0) {
                z.dy_norm[at] = dy_norm;
                z.row_bound[at] = fabsf(s) + dy_norm * (0x1p-8f * y_norm + 0x1p-20f);
            }
        }
    }
    if constexpr (kHalf) {
        const int64_t first = int64_t(start[1]) * a.kv_heads, end = int64_t(start[sequences + 1]) * a.kv_heads;
        for (int64_t i = first + int64_t(blockIdx.x) * kRows + group; i < end; i += step) {
            const int64_t t = i / a.kv_heads;
            const T *v = static_cast<const T *>(a.v) + t * a.v_token + (i - t * a.kv_heads) * a.v_head;
            float s = 0.0f;
            for (int d = l * V; d < a.D; d += LANES * V) {
                const Vec<T, V> p = bring(v + d, a.D - d);
#pragma unroll
                for (int j = 0; j < V; ++j) s += to_float(p.e[j]) * to_float(p.e[j]);
            }
            s = sum(s);
            if (l == 0) z.v_norm[(i - t * a.kv_heads) * a.tokens + t] = sqrtf(s);
        }
    }
}

// The tensor cores' copies need heads that start on 16-byte boundaries: others are copied to rows of
// whole 16 bytes first, eight elements a thread. The forward kernel compares scores before it scales them, by a
// positive factor: where the scale is negative (or zero), q is copied too, negated (or as zeros).
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
struct HeadsCopy {
    const void *x;
    void *to;
    int64_t units, token, head;
    int32_t heads, per;
    float factor;
};
struct HeadsCopies {
    HeadsCopy of[4];
    int32_t D;
};
template <typename T>
__global__ void __launch_bounds__(256) align_heads_kernel(const HeadsCopies c)
{
    const HeadsCopy &m = c.of[blockIdx.y];
    const int64_t step = int64_t(gridDim.x) * 256;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < m.units; i += step) {
        const int64_t row = i / m.per, t = row / m.heads;
        const int d = int(i - row * m.per) * 8;
        const T *p = static_cast<const T *>(m.x) + t * m.token + (row - t * m.heads) * m.head + d;
        Vec<T, 8> v;
#pragma unroll
        for (int j = 0; j < 8; ++j) v.e[j] = from_float<T>(d + j < c.D ? to_float(p[j]) * m.factor : 0.0f);
        *reinterpret_cast<Vec<T, 8> *>(static_cast<T *>(m.to) + i * 8) = v;
    }
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

// dk and dv of a group's heads from `split` parts, in order.
template <typename T>
__global__ void __launch_bounds__(256) join_parts_kernel(const AttentionArgs a)
{
    const int64_t n = a.tokens * a.kv_heads * a.D, step = int64_t(gridDim.x) * 256;
    T *const out = static_cast<T *>(blockIdx.y ? a.dv : a.dk);
    const float *const parts = a.partial + blockIdx.y * a.split * n;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < n; i += step) {
        float t = 0.0f;
        for (int p = 0; p < a.split; ++p) t += parts[p * n + i];
        out[i] = from_float<T>(t);
    }
}

// How many parts a group's heads are dealt to. With an item an SM or more, one: the parts' sums cost a pass over
// memory (8,192 tokens x 8 heads on 4 x 128, 256 items: 335 us in one part, 373 in two). With fewer, enough for two
// items an SM, if there are as many heads: a pass lasts as long as its longest item (2,000 floats in 3 sequences x 8
// heads on 2 x 64, 70 items: 1,123 us in one part, 592 in four).
int32_t parts_of(const AttentionArgs &a, int32_t sequences, int rows, int sms)
{
    const int64_t items = (a.tokens / rows + (sequences < a.tokens ? sequences : a.tokens) + 1) * a.kv_heads;
    if (items >= sms) return 1;
    const int64_t wanted = (2 * int64_t(sms) + items - 1) / items;
    return int32_t(wanted < a.group ? wanted : a.group);
}

// Where what dS's powers of two follow from lies in the workspace, from `at` on.
struct SizesAt {
    size_t dy_norm, row_bound, v_norm, top[3], row_power, key_power, end;
    int32_t chunks;
};
SizesAt grad_sizes(const AttentionArgs &a, size_t at)
{
    const size_t rows = size_t(a.heads) * size_t(a.tokens), keys = size_t(a.kv_heads) * size_t(a.tokens);
    SizesAt s;
    s.chunks = int32_t((a.tokens + kChunk - 1) / kChunk);
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += round256(bytes);
        return here;
    };
    s.dy_norm = take(sizeof(float) * rows);
    s.row_bound = take(sizeof(float) * rows);
    s.v_norm = take(sizeof(float) * keys);
    for (size_t &t : s.top) t = take(sizeof(uint32_t) * a.kv_heads * size_t(s.chunks));
    s.row_power = take(rows);
    s.key_power = take(keys);
    s.end = at;
    return s;
}

// Parts of the workspace; copy[i]: of operand i, where it needs one.
struct Layout {
    int rows;  // of a tile
    int32_t split;
    size_t first, start, delta, sizes, partial, copy[4], total;
    bool copied[4];
};
constexpr int kMostSms = 160;  // (a workspace is asked for before the device is)
Layout layout(int dtype, const AttentionArgs &a, int32_t sequences, bool grad)
{
    Layout l = {};
    l.rows = dtype == DC_FP32 ? kSimtRows : grad ? kMmaRows : attention_mma_rows(a);
    size_t at = round256(sizeof(AttentionPlan) +
                         sizeof(AttentionTile) * size_t(attention_most_tiles(a.tokens, sequences, l.rows)));
    l.first = at;
    at += round256(sizeof(int32_t) * (size_t(sequences) + 3));
    l.start = at;
    at += round256(sizeof(int32_t) * (size_t(sequences) + 3));
    l.delta = at;
    if (grad) at += round256(sizeof(float) * size_t(a.heads) * size_t(a.tokens));
    l.sizes = at;
    if (grad && dtype == DC_FP16) at = grad_sizes(a, at).end;
    l.split = grad ? parts_of(a, sequences, l.rows, kMostSms) : 1;
    l.partial = at;
    if (l.split > 1) at += round256(sizeof(float) * 2 * l.split * size_t(a.tokens) * a.kv_heads * a.D);
    for (int i = 0; i < (grad ? 4 : 3) && dtype != DC_FP32; ++i) {
        const Heads h = operand(a, i);
        l.copied[i] = !aligned(h, a.tokens) || (i == 0 && !grad && a.scale <= 0.0f);
        l.copy[i] = at;
        if (l.copied[i]) at += round256(size_t(a.tokens) * h.heads * padded(a.D) * 2);
    }
    l.total = at;
    return l;
}

template <typename T>
cudaError_t align_operands(AttentionArgs &a, const Layout &l, bool grad, unsigned char *ws, cudaStream_t stream)
{
    float factor = 1.0f;
    if (!grad && a.scale <= 0.0f) {
        factor = a.scale < 0.0f ? -1.0f : 0.0f;
        a.scale = a.scale < 0.0f ? -a.scale : 1.0f;
    }
    HeadsCopies c = {};
    c.D = a.D;
    int n = 0;
    int64_t most = 0;
    const int64_t pad = padded(a.D);
    for (int i = 0; i < 4; ++i) {
        if (!l.copied[i]) continue;
        const Heads h = operand(a, i);
        void *const to = ws + l.copy[i];
        c.of[n] = {h.p, to, a.tokens * h.heads * (pad / 8), h.token, h.head, h.heads, int32_t(pad / 8), i == 0 ? factor : 1.0f};
        if (c.of[n].units > most) most = c.of[n].units;
        ++n;
        const void **p[4] = {&a.q, &a.k, &a.v, &a.dy};
        int64_t *token[4] = {&a.q_token, &a.k_token, &a.v_token, &a.dy_token};
        int64_t *head[4] = {&a.q_head, &a.k_head, &a.v_head, &a.dy_head};
        *p[i] = to;
        *token[i] = h.heads * pad;
        *head[i] = pad;
    }
    if (n == 0) return cudaSuccess;
    const int64_t blocks = (most + 255) / 256, limit = 8192;
    align_heads_kernel<T><<<dim3(unsigned(blocks < limit ? blocks : limit), n), 256, 0, stream>>>(c);
    return cudaGetLastError();
}

template <typename T>
cudaError_t gradient(int dtype, AttentionArgs a, int32_t sequences, unsigned char *ws, const Layout &l, int64_t most,
                     cudaStream_t stream)
{
    int sms = 0;
    cudaError_t e = sm_count(sms);
    if (e == cudaSuccess) e = align_operands<T>(a, l, true, ws, stream);
    if (e != cudaSuccess) return e;
    const bool eight = a.D <= 8 * kVec<T>;  // lanes of a row
    const int64_t blocks = (a.tokens * a.heads + 15) / 16, limit = int64_t(sms) * 16;
    const unsigned grid = unsigned(blocks < limit ? blocks : limit);
    const int32_t *start = reinterpret_cast<const int32_t *>(ws + l.start);
    // operands of 16 bits are aligned by now; y is the caller's
    const int unit = 16 / int(sizeof(T));
    const bool wide = a.D % unit == 0 && aligned16(a.y) && aligned16(a.dy) && aligned16(a.v) && a.dy_token % unit == 0 &&
                      a.dy_head % unit == 0 && (a.tokens == 1 || a.v_token % unit == 0) &&
                      (a.kv_heads == 1 || a.v_head % unit == 0);
    GradSizes z = {};
    if (dtype == DC_FP16) {
        const SizesAt s = grad_sizes(a, l.sizes);
        z.dy_norm = reinterpret_cast<float *>(ws + s.dy_norm);
        z.row_bound = reinterpret_cast<float *>(ws + s.row_bound);
        z.v_norm = reinterpret_cast<float *>(ws + s.v_norm);
        z.top_v = reinterpret_cast<uint32_t *>(ws + s.top[0]);
        z.top_dy = reinterpret_cast<uint32_t *>(ws + s.top[1]);
        z.top_row = reinterpret_cast<uint32_t *>(ws + s.top[2]);
        a.row_power = z.row_power = reinterpret_cast<int8_t *>(ws + s.row_power);
        a.key_power = z.key_power = reinterpret_cast<int8_t *>(ws + s.key_power);
        z.chunks = s.chunks;
    }
    auto delta = wide ? eight ? attention_delta_kernel<T, true, 8> : attention_delta_kernel<T, true, 16>
                      : eight ? attention_delta_kernel<T, false, 8> : attention_delta_kernel<T, false, 16>;
    delta<<<grid, 256, 0, stream>>>(a, z, start, sequences);
    if (dtype == DC_FP16) {
        const int64_t chunks = int64_t(z.chunks) * a.kv_heads, tiles = most * a.kv_heads;
        e = launch_early(attention_chunks_kernel, chunks < limit ? chunks : limit, kChunk, 0, stream, a, z, start, sequences);
        if (e == cudaSuccess)
            e = launch_early(attention_powers_kernel, tiles < limit ? tiles : limit, kChunk, 0, stream, a, z);
        if (e != cudaSuccess) return e;
    }
    a.split = l.split;
    a.partial = reinterpret_cast<float *>(ws + l.partial);
    e = sizeof(T) == 2 ? launch_attention_grad_mma(dtype, a, most, stream) : launch_attention_grad_simt(a, most, stream);
    if (e != cudaSuccess || a.split == 1) return e;
    const int64_t join = (a.tokens * a.kv_heads * a.D + 255) / 256;
    join_parts_kernel<T><<<dim3(unsigned(join < limit ? join : limit), 2), 256, 0, stream>>>(a);
    return cudaGetLastError();
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
        if (dtype == DC_FP32) return launch_attention_simt(a, most, stream);
        const cudaError_t e = dtype == DC_BF16 ? align_operands<__nv_bfloat16>(a, l, false, ws, stream)
                                               : align_operands<__half>(a, l, false, ws, stream);
        return e == cudaSuccess ? launch_attention_mma(dtype, a, most, stream) : e;
    }
    a.delta = reinterpret_cast<float *>(ws + l.delta);
    switch (dtype) {
        case DC_BF16: return gradient<__nv_bfloat16>(dtype, a, sequences, ws, l, most, stream);
        case DC_FP16: return gradient<__half>(dtype, a, sequences, ws, l, most, stream);
        default: return gradient<float>(dtype, a, sequences, ws, l, most, stream);
    }
}

}  // namespace dc
