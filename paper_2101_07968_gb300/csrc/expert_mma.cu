// Expert products on the tensor cores (tcgen05): 16-bit operands, and floats as tf32 parts.
//
// The feature axis is the M of a product and the rows of the batch its N, so that ragged
// experts cost little: a tile's N is its rows rounded up to 16 (32 for a pair), where a tile
// whose M is the rows would do 128 at a time. D[feature][row] = sum_r A[feature][r] B[row][r]:
//   y   A = W_e (r = k contiguous)            B = x
//   dx  A = W_e^T (features contiguous)       B = dy
//   dW  A = dy^T, B = x^T (both with the summed axis, an expert's rows, outermost)
// The hardware reads either order of an operand, so nothing is transposed.
// Floats come as two parts that tf32 holds (expert_dispatch.cu), side by side along the summed
// axis, which is innermost and padded. A stage takes both parts of both operands and feeds three
// products: hi hi to one set of sums, hi lo and lo hi to another.
//
// A persistent pair of CTAs, one tile of 256 features between them, takes every grid-th tile.
// Warp 4 copies operand blocks of 128 bytes along the summed axis into a ring of stages by TMA;
// a thread of warp 5 issues the products; warps 0-3 store the finished tile from one half of
// the tensor memory while the next accumulates in the other. Rows of other experts that a copy
// brings along end in columns that are not stored; for dW, where they would be summed, warp 6
// overwrites those of an expert's last block with zeros between the copy's arrival and the
// product. Every wait ends after a number of tries, and the kernel then reports it in status.
//
// Measured (bfloat16, one GB300, short runs): 16,384 rows over 16 even experts x 4,096 x 2,048, 154-160 us
// each (1,720-1,780 TFLOP/s; ragged experts, whose last tiles are short, 173); 65,536 rows over 32 experts x
// 2,048 x 4,096, 567-580 us (1,900-1,940 TFLOP/s against a library product's 1,902). Long runs lower the
// clock to 1,450-1,500 of 2,070 MHz: 176 us, ragged 192, 726 a product of the larger. The tensor cores are busy 85 % of
// the time; a block's products take 512 cycles and its copies, read by every pair through the
// L2, some 630 (15 TB/s). A product takes some 100 cycles to issue whatever its columns, so
// tiles narrower than 256 do not run at the tensor cores' rate. With one or a few experts' rows
// the weights' bytes bound it: 128 rows over 24 of 32 experts x 2,048 x 2,048 38 us (5.3 TB/s).
#include <cuda.h>

#include <cmath>
#include <type_traits>

#include "blackwell.cuh"
#include "expert_rows.cuh"

namespace dc {
namespace {

constexpr int kBKBytes = 128;            // summed axis per stage: a line
constexpr int kPair = 2;                 // CTAs that share a tile
constexpr int kBM = 128;                 // features per CTA
constexpr int kThreads = 7 * 32;
constexpr uint32_t kABytes = kBM * kBKBytes;
constexpr uint32_t kBoxBytes = 64 * kBKBytes;  // a box of 64 lines

enum { kRowsK, kRowsMN, kWeights, kWeightsK };  // rows with A K-major or MN-major; weights MN- or K-major

struct MmaArgs {
    void *c;
    int64_t c_e, c_m;   // weights: expert and row strides of dW; rows: c_m is a row's stride
    const int64_t *offsets;
    int64_t rows;
    int32_t experts;
    int32_t m, n, r;    // M extent; weights: N extent; rows: summed extent
    int32_t *status;
    bool wide;          // weights: 16-byte stores; rows: 4-byte stores
    int32_t least;      // weights: experts of fewer rows are left to another kernel
    float *sums;        // long sums: a CTA's tile of the rounds so far (expert_mma_sum_bytes)
};

// Blocks summed in the tensor cores at a time. They cut a sum off at every step where a float
// would round, always toward zero: 1e-7 of it a step where the terms share a sign.
// 16-bit operands: 512 steps lose 5e-5, a tenth of half's rounding, and a million rows in one
// go 7e-3. So after 128 blocks (8,192 summed elements) a round's sums are added to those before it
// in floats, rounded: in memory that stays in the L2, since no registers are left at 256 columns,
// and while the next round is summed. One expert of 65,536 rows x 2,048 x 4,096, dW: 676-698 us against 631-686 in one go.
// Shorter sums are one round. It bounds the wait for a finished round, too.
constexpr int kRound16 = 128;
constexpr int64_t kLongSum = int64_t(kRound16) * kBKBytes / 2;
constexpr int kMostPairs = 80;  // of CTAs whose sums a workspace has room for

struct Tile {
    int32_t e;      // expert
    int32_t m0;     // first feature of the pair's or CTA's tile
    int32_t n0;     // first row (rows) or column (weights)
    int32_t cols;   // of them
    int32_t r0, r;  // summed axis: start (weights) and extent
};

template <int MODE, int BN>
__device__ __forceinline__ Tile tile_at(const MmaArgs &a, const Segments &seg, int t)
{
    Tile q;
    if (MODE == kWeights || MODE == kWeightsK) {
        const int nm = (a.m + kBM * kPair - 1) / (kBM * kPair), nn = (a.n + BN - 1) / BN;
        q.e = t / (nm * nn);
        const int i = t - q.e * (nm * nn);
        q.m0 = (i % nm) * (kBM * kPair);
        q.n0 = (i / nm) * BN;
        q.cols = min(BN, a.n - q.n0);
        q.r0 = seg.start[q.e + 1];
        q.r = seg.start[q.e + 2] - q.r0;
        if (MODE == kWeightsK) {  // the padded rows' high parts, then their low ones
            if (q.r < a.least) q.cols = 0;
            q.r0 = 2 * kPartRows * seg.tile[q.e + 1];
            q.r = kPartRows * (seg.tile[q.e + 2] - seg.tile[q.e + 1]);
        }
    } else {
        const int nm = (a.m + kBM * kPair - 1) / (kBM * kPair);
        const int whole = seg.tile[seg.count];
        const int s = find_segment(t < whole ? seg.tile : seg.part, seg.count, t);
        const int size = seg.start[s + 1] - seg.start[s];
        // the last rows' tiles follow the whole ones
        const int i = t < whole ? t - seg.tile[s] : t - seg.part[s] + size / BN * nm;
        const bool none = s == 0 || s == seg.count - 1;
        q.e = none ? 0 : s - 1;
        q.m0 = (i % nm) * (kBM * kPair);
        q.n0 = seg.start[s] + (i / nm) * BN;
        q.cols = min(BN, seg.start[s + 1] - q.n0);
        q.r0 = 0;
        q.r = none ? 0 : a.r;
    }
    return q;
}

// Rows (MN-major: columns, in whole lines) of B that a CTA's stage holds.
template <int MODE, int BN>
constexpr int kStageRows = MODE == kWeights && BN / kPair < 64 ? 64 : BN / kPair;

template <int MODE, int BN>
__device__ __forceinline__ int tile_count(const MmaArgs &a, const Segments &seg)
{
    if (MODE == kWeights || MODE == kWeightsK)
        return a.experts * ((a.m + kBM * kPair - 1) / (kBM * kPair)) * ((a.n + BN - 1) / BN);
    return seg.part[seg.count];
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi, __half)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}

// 32 finished columns (rows of the batch) of a lane's feature.
template <typename T>
__device__ __forceinline__ void store_rows(const MmaArgs &a, const Tile &q, int feature, int c0,
                                           const float (&v)[32])
{
    const int lane = threadIdx.x & 31;
    const int n = q.cols - c0;
    T *p = static_cast<T *>(a.c) + (int64_t(q.n0) + c0) * a.c_m + feature;
    if constexpr (sizeof(T) == 2) if (a.wide) {
        // Lanes in pairs exchange a value, so that each stores two features of one row: the
        // even lane those of row j, the odd one those of row j + 1.
        const bool odd = lane & 1;
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            const float other = __shfl_xor_sync(0xffffffffu, odd ? v[j] : v[j + 1], 1);
            const uint32_t w = odd ? pack2(other, v[j + 1], T()) : pack2(v[j], other, T());
            const int row = j + odd;
            if (row < n && feature < a.m)
                *reinterpret_cast<uint32_t *>(p + row * a.c_m - odd) = w;
        }
        return;
    }
    if (feature >= a.m) return;
#pragma unroll
    for (int j = 0; j < 32; ++j)
        if (j < n) p[j * a.c_m] = from_float<T>(v[j]);
}

// Rows of dW: a lane holds a row's neighbours, so 128 bytes a row go through shared memory
// (16-byte units, swizzled by the row) and leave as whole lines. Straight from the lanes, an
// instruction wrote 16 bytes to each of 32 rows: 2.8 TB/s where the output is the bound.
struct Lines {
    uint4 u[32][8];
};
template <typename T>
__device__ __forceinline__ void stage_columns(Lines &s, int unit, const float (&v)[32])
{
    const int lane = threadIdx.x & 31;
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
        for (int j = 0; j < 32; j += 4, ++unit)
            *reinterpret_cast<float4 *>(&s.u[lane][unit ^ (lane & 7)]) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
        return;
    } else
#pragma unroll
    for (int j = 0; j < 32; j += 8, ++unit)
        s.u[lane][unit ^ (lane & 7)] = make_uint4(pack2(v[j], v[j + 1], T()), pack2(v[j + 2], v[j + 3], T()),
                                                  pack2(v[j + 4], v[j + 5], T()), pack2(v[j + 6], v[j + 7], T()));
}
template <typename T>
__device__ __forceinline__ void store_lines(const Lines &s, const MmaArgs &a, const Tile &q, int row0,
                                            int c0)
{
    constexpr int V = 16 / sizeof(T), kCols = 8 * V;
    const int lane = threadIdx.x & 31;
    const int n = min(kCols, q.cols - c0);
    T *p = static_cast<T *>(a.c) + q.e * a.c_e + row0 * a.c_m + q.n0 + c0;
    __syncwarp();
    if (a.wide && n % V == 0) {
        const int unit = lane & 7;
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
            const int row = i + (lane >> 3);
            if (row0 + row < a.m && unit * V < n)
                *reinterpret_cast<uint4 *>(p + row * a.c_m + unit * V) = s.u[row][unit ^ (row & 7)];
        }
    } else {
        auto value = [&](int row, int c) {
            return reinterpret_cast<const T *>(&s.u[row][(c / V) ^ (row & 7)])[c % V];
        };
        const int rows = min(32, a.m - row0);
        if constexpr (sizeof(T) == 2) {
            // rows that start on 2-byte boundaries: pairs from the next 4-byte boundary on, and
            // what is left at both ends; eight rows' values before their stores
            constexpr int kAhead = 8;
            for (int r0 = 0; r0 < rows; r0 += kAhead) {
                Vec<T, 2> v[kAhead];
                int first[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int row = r0 + i;
                    first[i] = int(reinterpret_cast<uintptr_t>(p + row * a.c_m) >> 1 & 1);
                    const int c = 2 * lane + first[i];
                    v[i].e[0] = value(row, c);
                    v[i].e[1] = value(row, (c + 1) & (kCols - 1));
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    T *r = p + (r0 + i) * a.c_m;
                    const int c = 2 * lane + first[i];
                    if (r0 + i >= rows) continue;
                    if (c + 1 < n)
                        *reinterpret_cast<Vec<T, 2> *>(r + c) = v[i];
                    else if (c < n)
                        r[c] = v[i].e[0];
                }
                // the first element of rows whose pairs start at the second: a lane per row
                if (lane < kAhead && r0 + lane < rows) {
                    T *r = p + (r0 + lane) * a.c_m;
                    if (reinterpret_cast<uintptr_t>(r) >> 1 & 1) r[0] = value(r0 + lane, 0);
                }
            }
        } else {
#pragma unroll 4
            for (int row = 0; row < rows; ++row)
                if (lane < n) p[row * a.c_m + lane] = value(row, lane);
        }
    }
    __syncwarp();
}

template <typename T, int MODE, int BN, int STAGES>
__global__ void __launch_bounds__(kThreads, 1)
expert_mma_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b,
                  const MmaArgs a)
{
    // B: boxes of up to 64 rows, or (MN-major) of 64 columns
    constexpr int kBoxRows = MODE == kWeights || BN / kPair > 64 ? 64 : BN / kPair;
    constexpr uint32_t kBBox = kBoxRows * kBKBytes;
    constexpr uint32_t kBBytes = kStageRows<MODE, BN> * kBKBytes;
    constexpr int kBK = kBKBytes / sizeof(T), kStep = 32 / sizeof(T);  // per stage, per product
    constexpr bool kTf32 = std::is_same<T, float>::value, kOut = MODE == kWeights || MODE == kWeightsK;
    constexpr bool kAMn = MODE == kRowsMN || MODE == kWeights;
    // Floats, whose sums are to lose no more than sums in floats do: hi hi is handed over every
    // block of 32 elements, four steps, and added up in registers, rounded; the sums of hi lo and
    // lo hi, 2^-11 of it, stay until the tile's end. 1.35e-7 off in the root mean square for 64
    // summed elements, 1.5e-7 for 512, 2.4e-7 for 4,096, where a 32-bit sum of one product after another
    // is 1.5, 4.1 and 11.5e-7 off. Every 16 steps: 2.0, 3.5 and 3.7e-7, and 540 us against 576 for
    // 16,384 rows over 8 experts x 2,048 x 2,048.
    constexpr int kRound = kTf32 ? 1 : kRound16;
    constexpr int kParts = kTf32 ? 2 : 1;
    constexpr uint32_t kStage = kParts * (kABytes + kBBytes);
    // two rounds' sums, one read while the other grows; floats: after them two tiles' sums of hi lo
    constexpr uint32_t kColumns = 2 * kParts * BN, kCross = 2 * BN;
    extern __shared__ unsigned char dyn[];
    __shared__ alignas(8) uint64_t full[STAGES], empty[STAGES], tail[STAGES], done[2], free_[2];
    __shared__ uint32_t tmem_at, gave_up;
    __shared__ uint32_t rounds;  // weights: finished by this CTA (counted by the copying thread, its loop is a tenth slower)
    __shared__ alignas(16) Lines lines[kOut ? 4 : 1];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = bw::cluster_rank();
    const uint32_t ring = (bw::smem_addr(dyn) + 1023u) & ~1023u;
    const Segments seg = segments_at(dyn + (ring - bw::smem_addr(dyn)) + STAGES * kStage, a.experts);
    auto bar = [](uint64_t *b) { return bw::smem_addr(b); };
    auto lead = [&](uint64_t *b) { return bw::map_to(bw::smem_addr(b), 0); };

    if (threadIdx.x == 0) {
        for (int i = 0; i < STAGES; ++i) {
            bw::bar_init(bar(&full[i]), kPair);
            bw::bar_init(bar(&empty[i]), 1);
            bw::bar_init(bar(&tail[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bw::bar_init(bar(&done[i]), 1);
            bw::bar_init(bar(&free_[i]), 4 * kPair);
        }
        gave_up = rounds = 0;
        bw::bar_init_fence();
    }
    if (warp == 5) bw::tmem_alloc(bw::smem_addr(&tmem_at), kColumns);
    if (warp == 4 && lane == 0) {
        bw::prefetch_map(&map_a);
        bw::prefetch_map(&map_b);
    }
    if (warp == 0)
        build_segments<MODE != kWeightsK>(seg, a.offsets, a.rows, a.experts, MODE == kWeightsK ? kPartRows : BN,
                       MODE == kWeightsK ? 1 : (a.m + kBM * kPair - 1) / (kBM * kPair));
    bw::fence_before();
    __syncthreads();
    bw::cluster_sync();
    bw::fence_after();
    const uint32_t tmem = tmem_at;
    const int tiles = tile_count<MODE, BN>(a, seg);
    const int step = int(gridDim.x) / kPair, first = int(blockIdx.x) / kPair;

    if (warp == 4) {
        if (bw::elect_one()) {  // copies
            int s = 0, filled = 0;  // the next stage; stages filled so far, up to all
            uint32_t phase = 1;     // of the stage's release: the first round waits for none
            bool ok = true;
            const uint32_t full0 = lead(&full[0]);
            for (int t = first; t < tiles && ok; t += step) {
                const Tile q = tile_at<MODE, BN>(a, seg, t);
                if (MODE == kWeightsK && q.cols == 0) continue;
                const int cols = (q.cols + 16 * kPair - 1) / (16 * kPair) * 16;  // of this CTA
                const int boxes = (cols + kBoxRows - 1) / kBoxRows;
                const int m = q.m0 + int(rank) * kBM, n = q.n0 + int(rank) * cols;
                const uint32_t bytes = kParts * (kABytes + boxes * kBBox);
                const int end = q.r0 + q.r;
                for (int r = q.r0; r < end; r += kBK) {
                    if (filled < STAGES)
                        ++filled;
                    else if (!(ok = bw::bar_wait(bar(&empty[s]), phase, &gave_up)))
                        break;
                    const uint32_t sa = ring + s * kStage, sb = sa + kParts * kABytes;
                    const bool zeros = MODE == kWeights && end - r <= kBK && ((end - r) & 15);
                    const uint32_t b = zeros ? bar(&tail[s]) : full0 + s * uint32_t(sizeof(uint64_t));
                    if (zeros) {
                        bw::bar_arrive_bytes(b, bytes);
                    } else if (rank == 0) {  // for both CTAs: the other's bytes count here too
                        bw::bar_arrive_bytes(bar(&full[s]), bytes * kPair);
                        bw::bar_arrive(bar(&full[s]));
                    }
                    if (kTf32) {  // both parts of both operands
#pragma unroll
                        for (int part = 0; part < kParts; ++part) {
                            const int x = r + part * q.r;
                            if (MODE == kWeightsK)
                                bw::copy_2d(sa + part * kABytes, &map_a, x, m, b);
                            else
                                bw::copy_3d(sa + part * kABytes, &map_a, x, m, q.e, b);
                            for (int i = 0; i < boxes; ++i)
                                bw::copy_2d(sb + part * kBBytes + i * kBBox, &map_b, x, n + kBoxRows * i, b);
                        }
                    } else if (MODE == kRowsK) {
                        bw::copy_3d(sa, &map_a, r, m, q.e, b);
                    } else if (MODE == kRowsMN) {
                        bw::copy_3d(sa, &map_a, m, r, q.e, b);
                        bw::copy_3d(sa + kBoxBytes, &map_a, m + 64, r, q.e, b);
                    } else {
                        bw::copy_2d(sa, &map_a, m, r, b);
                        bw::copy_2d(sa + kBoxBytes, &map_a, m + 64, r, b);
                    }
                    for (int i = 0; i < boxes && !kTf32; ++i)
                        if (MODE == kWeights)
                            bw::copy_2d(sb + i * kBBox, &map_b, n + kBoxRows * i, r, b);
                        else
                            bw::copy_2d(sb + i * kBBox, &map_b, r, n + kBoxRows * i, b);
                    if (++s == STAGES) {
                        s = 0;
                        phase ^= 1;
                    }
                }
            }
            // The products' arrivals land in this CTA's memory: it may not end before them. The
            // oldest stage in use comes next in turn.
            for (int i = 0; i < filled && ok; ++i) {
                const int at = filled == STAGES ? (s + i) % STAGES : i;
                const uint32_t ph = filled == STAGES ? (s + i < STAGES ? phase : phase ^ 1) : 0;
                ok = bw::bar_wait(bar(&empty[at]), ph, &gave_up);
            }
        }
    } else if (warp == 5) {
        if (rank == 0 && bw::elect_one()) {  // products
            int s = 0, tile = 0;
            uint32_t phase = 0, cross = tmem + kCross;
            bool ok = true;
            for (int t = first; t < tiles && ok; t += step) {
                const Tile q = tile_at<MODE, BN>(a, seg, t);
                if (MODE == kWeightsK && q.cols == 0) continue;
                const uint32_t n = (q.cols + 16 * kPair - 1) / (16 * kPair) * (16 * kPair);
                const uint32_t shape =
                    kTf32 ? bw::tf32_shape(kBM * kPair, n)
                          : bw::f16_shape(std::is_same<T, __nv_bfloat16>::value, kAMn, MODE == kWeights, kBM * kPair, n);
                const int blocks = (q.r + kBK - 1) / kBK;
                for (int k0 = 0; (k0 == 0 || k0 < blocks) && ok; k0 += kRound, ++tile) {
                    const int half = tile & 1;
                    ok = tile < 2 || bw::bar_wait(bar(&free_[half]), (tile / 2 - 1) & 1, &gave_up);
                    if (!ok) break;
                    bw::fence_after();
                    const uint32_t d = tmem + half * BN;
                    const int k1 = min(blocks, k0 + kRound);
                    for (int kb = k0; kb < k1; ++kb) {
                        ok = bw::bar_wait(bar(&full[s]), phase, &gave_up);
                        if (!ok) break;
                        const int left = q.r - kb * kBK;
                        if (MODE == kWeights && left <= kBK && (left & 15))
                            bw::fence_cluster();  // the other CTA's zeros
                        bw::fence_after();
                        const uint32_t sa = ring + s * kStage;
                        const uint64_t da = bw::operand(sa, kAMn ? kBoxBytes : 16);
                        const uint64_t db = bw::operand(sa + kParts * kABytes, MODE == kWeights ? kBoxBytes : 16);
                        auto step_of = [&](int i) {
                            const bool add = i > 0 || kb > k0;
                            if constexpr (kTf32) {
                                constexpr uint64_t kLowA = kABytes >> 4, kLowB = kBBytes >> 4;
                                bw::mma_tf32(d, da + i * 2, db + i * 2, shape, add);
                                bw::mma_tf32(cross, da + i * 2, db + kLowB + i * 2, shape, i > 0 || kb > 0);
                                bw::mma_tf32(cross, da + kLowA + i * 2, db + i * 2, shape, true);
                            } else {
                                bw::mma(d, da + i * (kAMn ? 128 : 2), db + i * (MODE == kWeights ? 128 : 2), shape, add);
                            }
                        };
                        if (left >= kBK) {  // straight on: a loop's branches would hold the products up
#pragma unroll
                            for (int i = 0; i < kBK / kStep; ++i) step_of(i);
                        } else {
                            for (int i = 0; i * kStep < left; ++i) step_of(i);
                        }
                        bw::commit(bar(&empty[s]));
                        if (++s == STAGES) {
                            s = 0;
                            phase ^= 1;
                        }
                    }
                    if (ok) bw::commit(bar(&done[half]));
                }
                cross ^= (tmem + kCross) ^ (tmem + kCross + BN);
            }
        }
    } else if (warp == 6) {
        if (MODE == kWeights) {  // zeros after an expert's last row
            int it = 0;
            uint32_t uses = 0;  // parity of each stage's tail barrier
            for (int t = first; t < tiles; t += step) {
                const Tile q = tile_at<MODE, BN>(a, seg, t);
                const int blocks = (q.r + kBK - 1) / kBK;
                it += blocks;
                if ((q.r & 15) == 0) continue;
                const int s = (it - 1) % STAGES;
                // all blocks since the last such one come before this one: seconds for long experts
                bool ok = bw::bar_wait(bar(&tail[s]), (uses >> s) & 1, &gave_up, &rounds);
                if (!__all_sync(0xffffffffu, ok)) break;
                uses ^= 1u << s;
                const int cols = (q.cols + 16 * kPair - 1) / (16 * kPair) * 16;
                const int boxes = 2 + (cols + 63) / 64;  // A's two come first
                const int r = (q.r - 1) % kBK + 1, lines = (r + 15) / 16 * 16 - r;
                unsigned char *at = dyn + (ring - bw::smem_addr(dyn)) + s * kStage + r * 128;
                for (int i = lane; i < boxes * lines * 8; i += 32) {
                    const int box = i / (lines * 8), j = i - box * (lines * 8);
                    *reinterpret_cast<uint4 *>(at + box * kBoxBytes + j * 16) = make_uint4(0, 0, 0, 0);
                }
                bw::fence_async();
                __syncwarp();
                if (lane == 0) bw::bar_arrive_cluster_release(lead(&full[s]));
            }
        }
    } else {  // finished tiles
        int tile = 0;
        uint32_t cross = kCross;
        bool ok = true;
        for (int t = first; t < tiles && ok; t += step) {
            const Tile q = tile_at<MODE, BN>(a, seg, t);
            if (MODE == kWeightsK && q.cols == 0) continue;
            const int feature = q.m0 + int(rank) * kBM + warp * 32 + lane;
            const int blocks = (q.r + kBK - 1) / kBK;
            auto out = [&](int c0, const float (&v)[32]) {
                if (kOut) {
                    constexpr int kCols = 128 / sizeof(T);  // of a staged line
                    stage_columns<T>(lines[warp], c0 % kCols * int(sizeof(T)) / 16, v);
                    if ((c0 + 32) % kCols == 0 || c0 + 32 >= q.cols)
                        store_lines<T>(lines[warp], a, q, feature - lane, c0 & ~(kCols - 1));
                } else {
                    store_rows<T>(a, q, feature, c0, v);
                }
            };
            constexpr int kChunks = BN / 32;
            float sum[kTf32 ? kChunks : 1][32];  // floats: the rounds so far
            if (kTf32) {
#pragma unroll
                for (int c = 0; c < (kTf32 ? kChunks : 1); ++c)
#pragma unroll
                    for (int j = 0; j < 32; ++j) sum[c][j] = 0.0f;
            }
            for (int k0 = 0; k0 == 0 || k0 < blocks; k0 += kRound, ++tile) {
                const int half = tile & 1;
                ok = bw::bar_wait(bar(&done[half]), (tile / 2) & 1, &gave_up);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                if (MODE == kWeights && threadIdx.x == 0) *const_cast<volatile uint32_t *>(&rounds) = uint32_t(tile) + 1;
                bw::fence_after();
                const uint32_t lanes = tmem + (uint32_t(warp * 32) << 16), at = lanes + half * BN;
                auto all_read = [&] {  // the half may be overwritten
                    bw::fence_before();
                    __syncwarp();
                    if (lane == 0) bw::bar_arrive_cluster(lead(&free_[half]));
                };
                if constexpr (kTf32) {
#pragma unroll
                    for (int c = 0; c < kChunks; c += 2) {
                        if (c * 32 < q.cols && blocks > 0) {
                            float v[64];
                            __syncwarp();
                            bw::tmem_load(at + c * 32, v);
#pragma unroll
                            for (int j = 0; j < 64; ++j) sum[c + j / 32][j % 32] += v[j];
                        }
                    }
                    if (k0 + kRound >= blocks) {
                        // hi hi alone knows an infinity's class: its factor's low part may be
                        // zero or have the other sign
#pragma unroll
                        for (int c = 0; c < kChunks; ++c) {
                            if (c * 32 < q.cols && blocks > 0) {
                                float v[32];
                                __syncwarp();
                                bw::tmem_load(lanes + cross + c * 32, v);
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (fabsf(sum[c][j]) < INFINITY) sum[c][j] += v[j];
                            }
                        }
                        cross ^= kCross ^ (kCross + BN);
                    }
                    all_read();
                } else {
                    float v[32];
                    if (blocks <= kRound) {
                        for (int c0 = 0; c0 < q.cols; c0 += 32) {
                            __syncwarp();
                            if (blocks > 0) {
                                bw::tmem_load(at + c0, v);
                            } else {
#pragma unroll
                                for (int j = 0; j < 32; ++j) v[j] = 0.0f;
                            }
                            if (c0 + 32 >= q.cols) all_read();
                            out(c0, v);
                        }
                    } else {
                        for (int c0 = 0; c0 < q.cols; c0 += 32) {
                            // a thread reads what it wrote itself
                            float *so_far = a.sums + (int64_t(blockIdx.x) * BN + c0) * kBM + warp * 32 + lane;
                            __syncwarp();
                            bw::tmem_load(at + c0, v);
                            if (c0 + 32 >= q.cols) all_read();
                            if (k0 > 0) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) v[j] += so_far[j * kBM];
                            }
                            if (k0 + kRound < blocks) {
#pragma unroll
                                for (int j = 0; j < 32; ++j) so_far[j * kBM] = v[j];
                            } else {
                                out(c0, v);
                            }
                        }
                    }
                }
            }
            if constexpr (kTf32) {
                if (ok) {
#pragma unroll
                    for (int c = 0; c < kChunks; ++c)
                        if (c * 32 < q.cols) out(c * 32, sum[c]);
                }
            }
        }
    }
    __syncwarp();
    if (*const_cast<volatile uint32_t *>(&gave_up)) {
        // copies and products in flight still write this CTA's memory: let them end
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        if (threadIdx.x == 0 && a.status) *a.status = DC_ERR_INTERNAL;
    }
    bw::fence_before();
    __syncthreads();
    bw::cluster_sync();
    if (warp == 5) bw::tmem_free(tmem, kColumns);
}

// ------------------------------------------------------------------------------ host
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                                 const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                                 const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled()
{
    static const EncodeTiled fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) !=
                cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return EncodeTiled(nullptr);
        return EncodeTiled(p);
    }();
    return fn;
}

// A map of elements [z][y][x], x contiguous, copied in boxes of 128 bytes x `box_y`.
bool make_map(CUtensorMap &map, int dtype, const void *base, int64_t x, int64_t y, int64_t z,
              int64_t stride_y, int64_t stride_z, int box_y)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    const cuuint64_t dims[3] = {cuuint64_t(x), cuuint64_t(y), cuuint64_t(z)};
    const int bytes = dtype_bytes(dtype);
    const cuuint64_t strides[2] = {cuuint64_t(stride_y) * bytes, cuuint64_t(stride_z) * bytes};
    const cuuint32_t box[3] = {cuuint32_t(kBKBytes / bytes), cuuint32_t(box_y), 1}, one[3] = {1, 1, 1};
    const CUtensorMapDataType type = dtype == DC_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                     : dtype == DC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                        : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    return encode(&map, type,
                  stride_z ? 3 : 2, const_cast<void *>(base), dims, strides, box, one,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int MODE, int BN, int STAGES>
cudaError_t launch_typed(const CUtensorMap &ma, const CUtensorMap &mb, const MmaArgs &a,
                         int64_t most_tiles, cudaStream_t stream)
{
    auto kernel = expert_mma_kernel<T, MODE, BN, STAGES>;
    constexpr size_t ring = size_t(STAGES) * (std::is_same<T, float>::value ? 2 : 1) * (kABytes + kStageRows<MODE, BN> * kBKBytes) + 1024;
    const size_t smem = ring + segments_bytes(a.experts);
    static DeviceCache cache;
    int ready = 0, sms = 0;
    cudaError_t e = cache.get(ready, [&](int &v) {
        v = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    int(ring + segments_bytes(DC_EXPERTS_MAX)));
    });
    if (e == cudaSuccess) e = sm_count(sms);
    if (e != cudaSuccess) return e;
    int64_t units = sms / kPair;
    if (most_tiles < units) units = most_tiles;
    if (a.sums && units > kMostPairs) units = kMostPairs;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(unsigned(units * kPair));
    lc.blockDim = dim3(kThreads);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = kPair;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    lc.attrs = at;
    lc.numAttrs = 1;
    return cudaLaunchKernelEx(&lc, kernel, ma, mb, a);
}

// Tiles of 256 rows (columns of dW) read the least. Tiles of 64 are four times as many, and a
// step of one takes some 320 cycles against 512, bound by what an SM can read; so they pay
// where all of them still fit in one round (1,234 rows over 7 experts x 515 x 1,001, dx: 8.7 us
// against 11.9), but not above (4,000 rows over 2 x 1,024 x 1,024 floats: 132 us against 76).
int tile_rows(int dtype, int64_t tiles) { return 4 * tiles <= 76 ? 64 : dtype == DC_FP32 ? 128 : 256; }

template <typename T, int MODE>
cudaError_t launch_size(int bn, const CUtensorMap &ma, const CUtensorMap &mb, const MmaArgs &a, int64_t tiles,
                        cudaStream_t stream)
{
    if constexpr (std::is_same<T, float>::value)  // 128 sums a thread of the four warps that add up the rounds
        return bn == 64 ? launch_typed<T, MODE, 64, 4>(ma, mb, a, tiles, stream)
                        : launch_typed<T, MODE, 128, 4>(ma, mb, a, tiles, stream);
    else
        return bn == 64 ? launch_typed<T, MODE, 64, 8>(ma, mb, a, tiles, stream)
                        : launch_typed<T, MODE, 256, 6>(ma, mb, a, tiles, stream);
}

// Rows (columns of dW) of a tile, and the most tiles that there can be.
struct Tiles {
    int bn;
    int64_t most;
};
Tiles tiles_for(int dtype, const ExpertArgs &g, bool weights)
{
    Tiles t;
    if (weights) {
        const int64_t nm = (g.m + 255) / 256;
        t.bn = tile_rows(dtype, g.experts * nm * ((g.n + 255) / 256));
        t.most = g.experts * nm * ((g.n + t.bn - 1) / t.bn);
    } else {  // the choice by an average expert
        const int64_t nm = (g.n + 255) / 256, each = (g.rows + g.experts - 1) / g.experts;
        t.bn = tile_rows(dtype, g.experts * nm * ((each + 255) / 256));
        t.most = (g.rows / t.bn + g.experts + 2) * nm;
    }
    return t;
}

}  // namespace

size_t expert_mma_sum_bytes(int dtype, const ExpertArgs &g, bool weights)
{
    if (dtype == DC_FP32 || (weights ? g.rows : g.r) <= kLongSum) return 0;
    const Tiles t = tiles_for(dtype, g, weights);
    return size_t(t.most < kMostPairs ? t.most : kMostPairs) * 2 * kBM * t.bn * sizeof(float);
}

// Operands on 16-byte boundaries, or tf32 parts, as expert_dispatch.cu makes them.
cudaError_t expert_mma_rows(int dtype, const ExpertArgs &g, float *sums, cudaStream_t stream)
{
    const bool k_major = g.b_r == 1;
    const int64_t stride = k_major ? g.b_n : g.b_r;
    const int parts = dtype == DC_FP32 ? 2 : 1;
    const int64_t inner = k_major ? parts * int64_t(g.r) : g.n, outer = k_major ? g.n : g.r;
    // with one expert the stride between experts is not used, but it has to be valid
    const int64_t expert = g.experts == 1 ? stride * outer : g.b_e;
    const Tiles t = tiles_for(dtype, g, false);
    const int bn = t.bn;
    CUtensorMap ma, mb;
    if (!make_map(ma, dtype, g.b, inner, outer, g.experts, stride, expert, k_major ? 128 : 64) ||
        !make_map(mb, dtype, g.a, parts * int64_t(g.r), g.rows, 1, g.a_m, 0, bn < 128 ? bn / 2 : 64))
        return cudaErrorInvalidValue;
    MmaArgs a = {g.c, 0, g.c_m, g.offsets, g.rows, g.experts, g.n, 0, g.r, g.status, false, 0, sums};
    a.wide = g.c_m % 2 == 0 && g.n % 2 == 0 && reinterpret_cast<uintptr_t>(g.c) % 4 == 0;
    const int64_t tiles = t.most;
    if (tiles > (int64_t(1) << 30)) return cudaErrorInvalidValue;  // more than memory holds
    if (dtype == DC_FP32) return launch_size<float, kRowsK>(bn, ma, mb, a, tiles, stream);
    if (dtype == DC_BF16)
        return k_major ? launch_size<__nv_bfloat16, kRowsK>(bn, ma, mb, a, tiles, stream)
                       : launch_size<__nv_bfloat16, kRowsMN>(bn, ma, mb, a, tiles, stream);
    return k_major ? launch_size<__half, kRowsK>(bn, ma, mb, a, tiles, stream)
                   : launch_size<__half, kRowsMN>(bn, ma, mb, a, tiles, stream);
}

// Floats: a and b are parts [feature][summed], of stride a_r and b_r, for experts of at least
// `least` rows.
cudaError_t expert_mma_weights(int dtype, const ExpertArgs &g, int least, float *sums, cudaStream_t stream)
{
    const Tiles t = tiles_for(dtype, g, true);
    const int bn = t.bn;
    CUtensorMap ma, mb;
    const bool parts = dtype == DC_FP32;
    if (parts ? !make_map(ma, dtype, g.a, g.a_r, g.m, 1, g.a_r, 0, 128) ||
                    !make_map(mb, dtype, g.b, g.b_r, g.n, 1, g.b_r, 0, bn < 128 ? bn / 2 : 64)
              : !make_map(ma, dtype, g.a, g.m, g.rows, 1, g.a_r, 0, 64) ||
                    !make_map(mb, dtype, g.b, g.n, g.rows, 1, g.b_r, 0, 64))
        return cudaErrorInvalidValue;
    MmaArgs a = {g.c, g.c_e, g.c_m, g.offsets, g.rows, g.experts, g.m, g.n, 0, g.status, false, least, sums};
    const int v = 16 / dtype_bytes(dtype);
    a.wide = g.c_m % v == 0 && g.c_e % v == 0 && aligned16(g.c);
    const int64_t tiles = t.most;
    if (tiles > (int64_t(1) << 30)) return cudaErrorInvalidValue;
    return parts              ? launch_size<float, kWeightsK>(bn, ma, mb, a, tiles, stream)
           : dtype == DC_BF16 ? launch_size<__nv_bfloat16, kWeights>(bn, ma, mb, a, tiles, stream)
                              : launch_size<__half, kWeights>(bn, ma, mb, a, tiles, stream);
}

}  // namespace dc
