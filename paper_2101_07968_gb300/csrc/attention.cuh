// Causal attention of packed sequences: what its kernels share. Rows are cut into tiles that never
// cross a sequence's end; a list of them, those with the most work first, is made on the device
// (attention_plan.cu), since the sequences' offsets are device data.
#pragma once

#include "layers.cuh"

namespace dc {

// `rows` rows from row0 on, of a sequence that starts at row `first` and ends before `end`. first < 0: rows of no
// sequence, whose outputs are zeros.
struct AttentionTile {
    int32_t row0, rows, first, end;
};

// The plan's head in the workspace, then its tiles.
struct AttentionPlan {
    int32_t tiles;
    int32_t pad[15];
};
__host__ __device__ inline const AttentionTile *plan_tiles(const AttentionPlan *p)
{
    return reinterpret_cast<const AttentionTile *>(p + 1);
}

struct AttentionArgs {
    const void *q, *k, *v, *dy;      // dy: the gradient of y, [tokens][heads][D]
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, dy_token, dy_head;  // strides
    void *y, *dq, *dk, *dv;          // contiguous
    float *lse;                      // [heads][tokens]
    float *delta;                    // [heads][tokens]: sum of dy y
    // gradient of halves, the powers of two that dS is held in: [heads][tokens] of a row's dq, [kv_heads][tokens] of a
    // key's dk
    const int8_t *row_power, *key_power;
    const AttentionPlan *plan;
    int64_t tokens;
    int32_t heads, kv_heads, group, D;
    float scale;
    int32_t *status;
    // gradient: a group's heads may be dealt to `split` blocks, whose sums of dk and dv, floats [2][split][tokens]
    // [kv_heads][D], are then added up in order (1: none)
    int32_t split;
    float *partial;
};

// The most tiles of `rows` rows that a plan can have: a short one for each sequence, and the rows
// before the first and after the last.
inline int64_t attention_most_tiles(int64_t tokens, int32_t sequences, int rows)
{
    return tokens / rows + sequences + 2;
}

// Item `round` of a block, of items in order of falling work: every other round is dealt backwards,
// so that the sums are even. -1: none left.
__device__ __forceinline__ int64_t dealt(int64_t round, int64_t items)
{
    const int64_t at = round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x, i = round * gridDim.x + at;
    return i < items ? i : -1;
}

// csrc/attention_mma.cu, csrc/attention_grad_mma.cu: 16-bit types on the tensor cores, operands on 16-byte boundaries
// with strides of whole 16 bytes.
constexpr int kMmaRows = 128;
int attention_mma_rows(const AttentionArgs &a);  // of a tile of the forward pass
cudaError_t launch_attention_mma(int dtype, const AttentionArgs &a, int64_t most_tiles, cudaStream_t stream);
cudaError_t launch_attention_grad_mma(int dtype, const AttentionArgs &a, int64_t most_tiles, cudaStream_t stream);

// csrc/attention_simt.cu: floats, on the CUDA cores
constexpr int kSimtRows = 64;
cudaError_t launch_attention_simt(const AttentionArgs &a, int64_t most_tiles, cudaStream_t stream);
cudaError_t launch_attention_grad_simt(const AttentionArgs &a, int64_t most_tiles, cudaStream_t stream);

}  // namespace dc
