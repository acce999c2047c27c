// Shared device and host helpers of the layer operators (expert products, block
// norms, dropout, gated units).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "gen_device.cuh"

namespace dc {

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <>
__device__ __forceinline__ float to_float(float v) { return v; }

// the one rounding of an output
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
template <>
__device__ __forceinline__ float from_float(float v) { return v; }

// Two neighbours at once: the sums and products of pairs are single instructions.
__device__ __forceinline__ float2 pair_of(const __nv_bfloat16 *e) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(e)); }
__device__ __forceinline__ float2 pair_of(const __half *e) { return __half22float2(*reinterpret_cast<const __half2 *>(e)); }
__device__ __forceinline__ float2 pair_of(const float *e) { return *reinterpret_cast<const float2 *>(e); }
__device__ __forceinline__ void put_pair(__nv_bfloat16 *e, float2 v) { *reinterpret_cast<__nv_bfloat162 *>(e) = __float22bfloat162_rn(v); }
__device__ __forceinline__ void put_pair(__half *e, float2 v) { *reinterpret_cast<__half2 *>(e) = __float22half2_rn(v); }
__device__ __forceinline__ void put_pair(float *e, float2 v) { *reinterpret_cast<float2 *>(e) = v; }
__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// V consecutive elements, moved by one load or store of V * sizeof(T) bytes
template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T e[V];
};

template <typename T>
constexpr int kVec = 16 / int(sizeof(T));  // elements of a 16-byte access

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline bool dtype_ok(int dtype) { return dtype >= DC_BF16 && dtype <= DC_FP32; }
inline int dtype_bytes(int dtype) { return dtype == DC_FP32 ? 4 : 2; }

// Dropout: elements whose 16-bit field is at least `threshold` are kept and multiplied by
// `scale` = 65536 / (65536 - threshold). Sixteen bits an element let one SplitMix64 draw
// serve four: two 64-bit multiplications are what the mask costs, and one per element
// would bound the pass by integer issue instead of memory.
struct DropRule {
    uint64_t seed;
    int64_t offset;
    uint32_t threshold;  // 0: everything is kept, no draws
    float scale;
};

// SplitMix64 in two parts, for kernels that step the state themselves: splitmix(seed, n) is
// splitmix_output(seed + (n + 1) kGamma).
constexpr uint64_t kGamma = 0x9e3779b97f4a7c15ull;
__device__ __forceinline__ uint64_t splitmix_output(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xbf58476d1ce4e5b9ull;
    z = (z ^ (z >> 27)) * 0x94d049bb133111ebull;
    return z ^ (z >> 31);
}

inline DropRule drop_rule(double p, uint64_t seed, int64_t offset)
{
    DropRule d;
    d.seed = seed;
    d.offset = offset;
    d.threshold = uint32_t(p * 65536.0 + 0.5);
    d.scale = d.threshold < 65536u ? float(65536.0 / double(65536u - d.threshold)) : 0.0f;
    return d;
}

// A field is at least `threshold` (1 .. 65536) when the word with that field on top is above
// threshold 2^16 - 1 (the largest word for 65536, which drops all).
__device__ __forceinline__ bool kept(const DropRule &d, uint64_t draw, int field)
{
    const uint32_t w = uint32_t(draw >> (field & 2 ? 32 : 0));
    return d.threshold == 0 || (field & 1 ? w : w << 16) > (d.threshold << 16) - 1u;
}

// Runs body with T bound to the element type of `dtype`.
#define DC_DTYPE_SWITCH(dtype, T, ...)                \
    switch (dtype) {                                  \
        case DC_BF16: {                               \
            using T = __nv_bfloat16;                  \
            __VA_ARGS__                               \
        }                                             \
        case DC_FP16: {                               \
            using T = __half;                         \
            __VA_ARGS__                               \
        }                                             \
        default: {                                    \
            using T = float;                          \
            __VA_ARGS__                               \
        }                                             \
    }

cudaError_t sm_count(int &n);  // of the current device (layers_abi.cu)

// launchers of the layer operators
struct NormArgs {
    const void *x, *f, *gate, *w_post, *w_pre;  // forward; x is y in the gradient
    void *y, *h;
    const void *dy, *dh;
    void *dx, *df, *dgate;
    float *dw_post, *dw_pre;
    int64_t rows, rows_per_gate;
    int32_t D;
    bool layer;
    float alpha, eps;
    DropRule drop;
};
cudaError_t launch_dropout(int dtype, int64_t rows, int cols, const void *x, int64_t ldx,
                           const void *res, int64_t ldr, void *y, int64_t ldy, const DropRule &d,
                           cudaStream_t stream);
cudaError_t launch_gated(int dtype, int act, int64_t rows, int F, const void *h, int64_t ldh,
                         void *a, int64_t lda, cudaStream_t stream);
cudaError_t launch_gated_grad(int dtype, int act, int64_t rows, int F, const void *da,
                              int64_t ldda, const void *h, int64_t ldh, void *dh, int64_t lddh,
                              cudaStream_t stream);
cudaError_t launch_norm(int dtype, const NormArgs &a, cudaStream_t stream);
size_t norm_grad_workspace(int dtype, int64_t rows, int D);
cudaError_t launch_norm_grad(int dtype, const NormArgs &a, float *partial, cudaStream_t stream);

// One product grouped by expert: C[m][n] = sum_r A[m][r] B[n][r], as strided arrays.
// Rows (y, dx): m is a row, n a feature, B the expert's weights. Weights (dW): m, n index
// the expert's matrix and r runs over its rows.
struct ExpertArgs {
    const void *a, *b;
    void *c;
    int64_t a_m, a_r;       // strides of A
    int64_t b_e, b_n, b_r;  // strides of B (b_e between experts; 0 for weights)
    int64_t c_e, c_m;       // strides of C (c_e between experts; 0 for rows); c_n is 1
    const int64_t *offsets;
    int64_t rows;
    int32_t experts, m, n, r;  // rows: m unused; weights: r unused
    int32_t *status;
};
size_t expert_workspace(int dtype, const ExpertArgs &a, bool weights);
cudaError_t launch_expert_rows(int dtype, const ExpertArgs &a, void *workspace, cudaStream_t stream);
cudaError_t launch_expert_weights(int dtype, const ExpertArgs &a, void *workspace,
                                  cudaStream_t stream);
// The kernels behind them: the tensor cores (expert_mma.cu) for 16-bit operands on 16-byte
// boundaries and floats in tf32 parts, few rows of any type (expert_few.cu), the CUDA cores
// for small float products (expert_simt.cu; experts of `most` rows or fewer).
// sums: expert_mma_sum_bytes for sums too long to stay in the tensor cores.
size_t expert_mma_sum_bytes(int dtype, const ExpertArgs &a, bool weights);
cudaError_t expert_mma_rows(int dtype, const ExpertArgs &a, float *sums, cudaStream_t stream);
cudaError_t expert_mma_weights(int dtype, const ExpertArgs &a, int least, float *sums, cudaStream_t stream);
cudaError_t expert_few_rows(int dtype, const ExpertArgs &a, cudaStream_t stream);
cudaError_t expert_simt_rows(const ExpertArgs &a, cudaStream_t stream);
cudaError_t expert_simt_weights(const ExpertArgs &a, int64_t most, cudaStream_t stream);

// Norms and rotation of queries (0) and keys (1).
struct HeadNormArgs {
    const void *x[2], *dy[2], *w[2];  // dy: the gradient's, contiguous
    void *y[2];                       // outputs (dx), contiguous
    float *dw[2];
    int64_t token[2], head[2];  // strides of x
    int32_t heads[2];
    const int64_t *positions;
    int64_t tokens;
    int32_t D, rotary;
    bool interleaved, norm;
    float eps;
    float *partial;           // gradient of the weights: the blocks' sums (nullable)
    int32_t parts[2], per_part[2], blocks[2];  // of a token's heads, the heads of one, the grid (set by the launcher)
};
// Of pair i per position: in 2^-64 of a turn, and what is below, in 2^-128. A kernel's parameters hold those of the heads
// that it takes and no more: one token in a graph took 6.1 us with 2 KB of them, 4.3 with 1 KB.
template <int N>
struct Turns {
    uint64_t upper[N], below[N];
};
using AllTurns = Turns<DC_HEAD_NORM_DIM_MAX / 2>;
template <int N>
inline Turns<N> first_turns(const AllTurns &t)
{
    Turns<N> f;
    for (int i = 0; i < N; ++i) {
        f.upper[i] = t.upper[i];
        f.below[i] = t.below[i];
    }
    return f;
}
// Few tokens: a token's heads are dealt to `parts` groups, `per_part` each (the last part's fewer, but one at least:
// copies start at a part's first head), as finely as tokens * parts >= wanted needs, but not finer than `least` heads
// a part.
struct HeadParts {
    int32_t parts, per_part;
};
inline HeadParts head_parts(int64_t tokens, int32_t heads, int64_t wanted, int32_t least)
{
    int32_t parts = 1;
    while (tokens * parts < wanted && heads > parts * least) parts *= 2;
    const int32_t per = (heads + parts - 1) / parts;
    return {(heads + per - 1) / per, per};  // rounded up, the last parts would begin past the last head
}
size_t head_norm_workspace(int D);
cudaError_t launch_head_norm(int dtype, const HeadNormArgs &a, const AllTurns &turns, cudaStream_t stream);
cudaError_t launch_head_norm_grad(int dtype, const HeadNormArgs &a, const AllTurns &turns, cudaStream_t stream);

// attention_plan.cu
struct AttentionArgs;
size_t attention_workspace(int dtype, const AttentionArgs &a, int32_t sequences, bool grad);
cudaError_t launch_attention(int dtype, AttentionArgs a, int32_t sequences, const int64_t *offsets, bool grad,
                             void *workspace, cudaStream_t stream);

}  // namespace dc
