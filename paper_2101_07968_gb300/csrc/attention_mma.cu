// Causal attention of 16-bit types on the tensor cores, forward.
//
// A CTA holds two tiles of 128 rows at a time: two heads of one key head, or, where the group
// is odd, neighbouring tiles of one head. Keys and values come in blocks of 128 through a ring.
// For each tile and block: scores S = q k^T [row][key] into tensor memory; four warps, a thread
// a row, take the row's maximum and write P = 2^(s - m) in 16 bits over the scores; y += P v,
// with P read from tensor memory and y held there. While one tile's warps are at their
// exponentials the tensor cores work on the other tile; what a tile waits for is its P v and next S, so
// the first 64 keys' P is handed over as soon as it is made.
//
//   warps 0-3, 4-7  a tile each: softmax
//   warps 8-11      the finished rows of both tiles, while the next tiles' scores are made
//   warp 12         copies (TMA)
//   warp 13         products, by one thread
//   warp 14         looks through the values on the diagonal
//   warp 15         looks up the items ahead of the others: the list is in memory, a thousand clocks away
// A launch has 128 registers a thread; the softmax's warps take more of them from the others.
//
// Measured (one GB300): one prompt of 16,384 tokens x 16 heads x 128 688 us, 1,598 TFLOP/s (library products of one
// matrix 1,859); x 64 572 us; 8 sequences of 2,048 x 32 heads on 8 x 128 265 us. Tensor cores busy 69 % of the time; a tile's
// block takes its softmax's 1,650 clocks and 1,390 until the next scores are there, of which the products are 1,024.
// Bound by that chain, and by shared memory: a product of scores reads two operands of 4 KB in its 64 clocks.
//
// Rounding: P is rounded to the operands' type for the tensor cores, at most half a step of each
// term, where y's own rounding is half a step of the sum; l adds the unrounded ones in floats.
// The reference m is not raised with every larger maximum but once it is 2^8 too low: P up to 256
// is as good in 16 bits with a floating point, and y in tensor memory is seldom rescaled. Halves have few
// exponents: P and l are held 2^7 times larger, up to 2^15, so that steps below their normal range are 2^-31 of the
// reference and what a term loses there is 2^-32 of it (without, 16,384 keys behind one that is ahead by 17 were 44 % off).
//
// A mask cuts only the block on the diagonal, the tile's last. Values there that are not finite
// would reach rows that must not see them through 0 * inf. So rows after the sequence's end are overwritten
// with zeros there, and the block's own are looked through: where one is not finite, that block's
// y += P v is done by its tile's threads (masked_product).
#include <cmath>

#include "attention_mma.cuh"

namespace dc {
namespace {

using namespace am;

constexpr int kThreads = 16 * 32;
constexpr int kSoftmaxRegs = 184, kOtherRegs = 72;
static_assert(2 * kSoftmaxRegs + 2 * kOtherRegs <= 4 * 128, "registers of the launch");
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.0f;  // how far, in powers of two, the reference may be below the maximum
template <typename T>
constexpr float kPPower = std::is_same<T, __half>::value ? 7.0f : 0.0f;  // P is held 2^kPPower times larger, and l

struct alignas(16) Item {
    int32_t head[2], row0[2], rows[2], blocks[2];
    int32_t kv, first;  // the key head; the sequence's first row
    bool last;          // no item: the end
};
constexpr int kItems = 4, kItemUsers = 15;  // looked up ahead; warps that read each

template <bool PAIR>
__device__ __forceinline__ Item item_at(const AttentionArgs &a, int64_t i)
{
    const int per = PAIR ? a.heads / 2 : a.heads;
    Item q;
    const int64_t at = i < (int64_t(1) << 31) ? int64_t(uint32_t(i) / uint32_t(per)) : i / per;
    const AttentionTile t = plan_tiles(a.plan)[at];
    const int h = int(i - at * per);
    const int before = (t.row0 - max(t.first, 0)) / kTile;
    if (PAIR) {
        q.head[0] = 2 * h;
        q.head[1] = 2 * h + 1;
        q.row0[0] = q.row0[1] = t.row0;
        q.rows[0] = q.rows[1] = t.rows;
        q.blocks[0] = q.blocks[1] = before + 1;
    } else {
        q.head[0] = q.head[1] = h;
        q.row0[0] = t.row0;
        q.row0[1] = t.row0 + kTile;
        q.rows[0] = min(kTile, t.rows);
        q.rows[1] = t.rows - q.rows[0];
        q.blocks[0] = before + 1;
        q.blocks[1] = q.rows[1] > 0 ? before + 2 : 0;
    }
    if (t.first < 0) q.blocks[0] = q.blocks[1] = 0;
    q.kv = q.head[0] / a.group;
    q.first = t.first;
    q.last = false;
    return q;
}
// Blocks of values on the diagonal, which are looked through: one for two heads, one for each of two tiles.
template <bool PAIR>
__device__ __forceinline__ uint32_t checks_of(const Item &q)
{
    return PAIR ? q.blocks[0] > 0 : (q.blocks[0] > 0) + (q.blocks[1] > 0);
}

// Tiles of queries in shared memory, taken in turn: the two at work, and what comes next (a tile's last scores
// are made well before its last P v, and rows come from memory).
template <int DP>
constexpr int kTilesOfQ = DP == 64 ? 4 : 3;
template <int DP>
constexpr int kRing = DP == 64 ? 8 : 4;  // blocks of keys or values
constexpr uint32_t kSharedBytes = 2944;  // barriers and rows' sums

template <typename T, int DP, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1)
attention_mma_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const AttentionArgs a)
{
    constexpr int kBoxes = DP / 64;
    constexpr uint32_t kBytes = kBoxes * kBox;  // of a tile in shared memory
    constexpr int kStages = kRing<DP>;
    constexpr int kQ = kTilesOfQ<DP>;
    constexpr int kChecks = 4;  // no more blocks of values are in the ring
    extern __shared__ __align__(1024) unsigned char dyn[];
    struct Shared {
        uint64_t q_full[kQ], q_free[kQ], full[kStages], empty[kStages], s_full[2], p_half[2], p_full[2], y_full[2],
            y_free[2], l_full[2], look[kChecks], checked[kChecks], item_full[kItems], item_free[kItems], last;
        uint64_t until;  // when waits end, set anew with every copy: an item takes as long as its keys are many
        uint32_t tmem_at, gave_up;
        uint32_t by_hand[kChecks];  // the check, counted from one, if its block's sums are done by hand
        float row_l[2][kTile], row_m[2][kTile];  // of finished tiles
        Item items[kItems];
    };
    static_assert(sizeof(Shared) <= kSharedBytes, "room behind the tiles");
    Shared &h = *reinterpret_cast<Shared *>(dyn + (kQ + kStages) * kBytes);
    uint32_t *const gave_up = &h.gave_up;
    volatile uint64_t *const until = &h.until;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bar = [](uint64_t *b) { return bw::smem_addr(b); };
    auto is_by_hand = [&](uint32_t check) {
        return *const_cast<volatile uint32_t *>(&h.by_hand[check % kChecks]) == check + 1;
    };
    const uint32_t base = bw::smem_addr(dyn), ring = base + kQ * kBytes;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kQ; ++i) {
            bw::bar_init(bar(&h.q_full[i]), 1);
            bw::bar_init(bar(&h.q_free[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            bw::bar_init(bar(&h.s_full[i]), 1);
            bw::bar_init(bar(&h.p_half[i]), 4);
            bw::bar_init(bar(&h.p_full[i]), 4);
            bw::bar_init(bar(&h.y_full[i]), 1);
            bw::bar_init(bar(&h.y_free[i]), 4);
            bw::bar_init(bar(&h.l_full[i]), 4);
        }
        for (int i = 0; i < kStages; ++i) {
            bw::bar_init(bar(&h.full[i]), 1);
            bw::bar_init(bar(&h.empty[i]), 1);
        }
        for (int i = 0; i < kChecks; ++i) {
            bw::bar_init(bar(&h.look[i]), 1);
            bw::bar_init(bar(&h.checked[i]), 1);
            h.by_hand[i] = 0;
        }
        for (int i = 0; i < kItems; ++i) {
            bw::bar_init(bar(&h.item_full[i]), 1);
            bw::bar_init(bar(&h.item_free[i]), kItemUsers);
        }
        bw::bar_init(bar(&h.last), 1);
        h.gave_up = 0;
        bw::bar_init_fence();
    }
    if (warp == 13) bw::tmem_alloc1(bw::smem_addr(&h.tmem_at), 512);
    if (warp == 12 && lane == 0) {
        bw::prefetch_map(&map_q);
        bw::prefetch_map(&map_k);
        bw::prefetch_map(&map_v);
    }
    pdl_wait();  // the list and the copies are there
    if (threadIdx.x == 0) bw::wait_on(until);
    bw::fence_before();
    __syncthreads();
    bw::fence_after();
    const uint32_t tmem = h.tmem_at;  // scores of both tiles, then y of both
    // the swizzled copies need tiles on 1,024-byte boundaries
    const int64_t items = (base & 1023u) ? 0 : int64_t(a.plan->tiles) * (PAIR ? a.heads / 2 : a.heads);
    if ((base & 1023u) && threadIdx.x == 0) h.gave_up = 1;
    // Item n of this CTA, by a thread or by a whole warp; false: there is none (or a wait was given up).
    auto item_of_thread = [&](uint32_t n, Item &q) {
        if (!bw::bar_wait_inline(bar(&h.item_full[n % kItems]), (n / kItems) & 1, gave_up, until)) return false;
        q = h.items[n % kItems];
        bw::bar_arrive(bar(&h.item_free[n % kItems]));
        return !q.last;
    };
    auto item_of_warp = [&](uint32_t n, Item &q) {
        const bool ok = bw::bar_wait_inline(bar(&h.item_full[n % kItems]), (n / kItems) & 1, gave_up, until);
        if (!__all_sync(0xffffffffu, ok)) return false;
        q = h.items[n % kItems];
        __syncwarp();
        if (lane == 0) bw::bar_arrive(bar(&h.item_free[n % kItems]));
        return !q.last;
    };

    if (warp >= 12) {
        bw::fewer_registers<kOtherRegs>();
        if (warp == 12) {
            if (bw::elect_one()) {  // copies
                int s = 0;
                uint32_t phase = 1, tiles = 0;  // of queries so far
                bool ok = true;
                auto block = [&](const CUtensorMap &map, int head, int row) {
                    ok = ok && bw::bar_wait_inline(bar(&h.empty[s]), phase, gave_up, until);
                    if (!ok) return;
                    bw::wait_on(until);
                    bw::bar_arrive_bytes(bar(&h.full[s]), kBytes);
                    for (int i = 0; i < kBoxes; ++i)
                        bw::copy_3d1(ring + s * kBytes + i * kBox, &map, 64 * i, head, row, bar(&h.full[s]));
                    if (++s == kStages) {
                        s = 0;
                        phase ^= 1;
                    }
                };
                uint32_t checks = 0;
                Item q;
                for (uint32_t item = 0; ok && item_of_thread(item, q); ++item) {
                    bw::wait_on(until);
                    for (int x = 0; x < 2; ++x) {
                        if (q.blocks[x] == 0) continue;
                        const uint32_t at = tiles % kQ;
                        ok = ok && (tiles < kQ ||
                                    bw::bar_wait_inline(bar(&h.q_free[at]), (tiles / kQ - 1) & 1, gave_up, until));
                        if (!ok) break;
                        ++tiles;
                        bw::bar_arrive_bytes(bar(&h.q_full[at]), kBytes);
                        for (int b = 0; b < kBoxes; ++b)
                            bw::copy_3d1(base + at * kBytes + b * kBox, &map_q, 64 * b, q.head[x], q.row0[x], bar(&h.q_full[at]));
                        if (x == 0) block(map_k, q.kv, q.first);
                    }
                    const int n = max(q.blocks[0], q.blocks[1]);
                    for (int j = 0; j < n && ok; ++j) {
                        if (j > 0) block(map_k, q.kv, q.first + j * kTile);
                        block(map_v, q.kv, q.first + j * kTile);
                        // values on the diagonal are to be looked through: their barrier's phase has begun, and does not
                        // end twice before they are
                        for (int x = 0; x < (PAIR ? 1 : 2) && ok; ++x)
                            if (j + 1 == q.blocks[x]) bw::bar_arrive(bar(&h.look[(checks + x) % kChecks]));
                    }
                    checks += checks_of<PAIR>(q);
                }
            }
        } else if (warp == 13) {
            if (bw::elect_one()) {  // products
                constexpr bool kBf = std::is_same<T, __nv_bfloat16>::value;
                const uint32_t shape_s = bw::f16_shape(kBf, false, false, kTile, kTile);
                const uint32_t shape_y = bw::f16_shape(kBf, false, true, kTile, DP);
                uint32_t c = 0;  // blocks of the ring before this item
                uint32_t tiles = 0, blocks[2] = {0, 0}, items_of[2] = {0, 0}, checks = 0;  // of either tile so far; of both
                uint32_t at[2] = {0, 0};  // where the tiles' queries are
                bool ok = true;
                auto have = [&](uint32_t n) {
                    ok = ok && bw::bar_wait_inline(bar(&h.full[n % kStages]), (n / kStages) & 1, gave_up, until);
                    return ok;
                };
                auto scores = [&](int x, uint32_t n) {
                    const uint64_t dq = bw::operand(base + at[x] * kBytes, 16), dk = bw::operand(ring + n % kStages * kBytes, 16);
                    bw::fence_after();
#pragma unroll
                    for (int i = 0; i < DP / 16; ++i) {
                        const uint64_t step = (i / 4) * (kBox >> 4) + (i % 4) * 2;
                        bw::mma1(tmem + x * kTile, dq + step, dk + step, shape_s, i > 0);
                    }
                };
                Item q;
                for (uint32_t item = 0; ok && item_of_thread(item, q); ++item) {
                    const int n = max(q.blocks[0], q.blocks[1]);
                    for (int x = 0; x < 2 && ok; ++x) {
                        if (q.blocks[x] == 0) continue;
                        at[x] = tiles % kQ;
                        ok = bw::bar_wait_inline(bar(&h.q_full[at[x]]), (tiles / kQ) & 1, gave_up, until);
                        ++tiles;
                        if (!have(c)) break;
                        scores(x, c);
                        bw::commit1(bar(&h.s_full[x]));
                        if (q.blocks[x] == 1) bw::commit1(bar(&h.q_free[at[x]]));
                    }
                    if (n > 0) bw::commit1(bar(&h.empty[c % kStages]));
                    for (int j = 0; j < n && ok; ++j) {
                        const uint32_t k = c + 2 * j + 2, v = c + 2 * j + 1;
                        if (!have(v)) break;
                        for (int x = 0; x < 2 && ok; ++x) {
                            if (j >= q.blocks[x]) continue;
                            const uint64_t dv = bw::operand(ring + v % kStages * kBytes, kBox);
                            auto half = [&](int i0) {
#pragma unroll
                                for (int i = i0; i < i0 + kTile / 32; ++i)
                                    bw::mma1_tmem(tmem + 2 * kTile + x * DP, tmem + x * kTile + i * 8, dv + i * 128, shape_y,
                                                  j > 0 || i > 0);
                            };
                            // the rows before these have left
                            ok = j > 0 || items_of[x]++ == 0 ||
                                 bw::bar_wait_inline(bar(&h.y_free[x]), items_of[x] & 1, gave_up, until);
                            ok = ok && bw::bar_wait_inline(bar(&h.p_half[x]), blocks[x] & 1, gave_up, until);
                            if (!ok) break;
                            bw::fence_after();
                            // (known before the first half is handed over)
                            const bool own = j + 1 < q.blocks[x] || !is_by_hand(checks + (PAIR ? 0 : x));
                            if (own) half(0);
                            ok = bw::bar_wait_inline(bar(&h.p_full[x]), blocks[x]++ & 1, gave_up, until);
                            if (!ok) break;
                            bw::fence_after();
                            if (own) half(kTile / 32);
                            if (j + 1 < q.blocks[x]) {
                                if (!have(k)) break;
                                scores(x, k);
                                bw::commit1(bar(&h.s_full[x]));
                                if (j + 2 == q.blocks[x]) bw::commit1(bar(&h.q_free[at[x]]));
                            } else {
                                bw::commit1(bar(&h.y_full[x]));
                            }
                        }
                        bw::commit1(bar(&h.empty[v % kStages]));
                        if (j + 1 < n) bw::commit1(bar(&h.empty[k % kStages]));
                    }
                    c += 2 * n;
                    checks += checks_of<PAIR>(q);
                }
                // arrivals land in this CTA's memory: it may not end before the last
                bw::commit1(bar(&h.last));
                bw::bar_wait_inline(bar(&h.last), 0, gave_up, until);
            }
        } else if (warp == 14) {  // values on the diagonal
            uint32_t c = 0, checks = 0;
            bool ok = true;
            Item q;
            for (uint32_t item = 0; ok && item_of_warp(item, q); ++item) {
                const uint32_t n = checks_of<PAIR>(q);
                for (uint32_t x = 0; x < n; ++x, ++checks) {
                    const uint32_t v = c + 2 * q.blocks[x] - 1;
                    ok = bw::bar_wait_idle(bar(&h.look[checks % kChecks]), (checks / kChecks) & 1, gave_up, until) &&
                         bw::bar_wait_inline(bar(&h.full[v % kStages]), (v / kStages) & 1, gave_up, until);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    unsigned char *tile = dyn + (kQ + v % kStages) * kBytes;
                    for (int r = lane; r < kTile; r += 32)
                        if (look_through<T, DP>(tile, r, q.rows[x]))
                            *const_cast<volatile uint32_t *>(&h.by_hand[checks % kChecks]) = checks + 1;
                    __syncwarp();
                    if (lane == 0) bw::bar_arrive(bar(&h.checked[checks % kChecks]));
                }
                c += 2 * max(q.blocks[0], q.blocks[1]);
            }
        } else {
            if (bw::elect_one()) {  // items
                bool ok = true;
                bool more = true;
                for (int64_t round = 0; ok && more; ++round) {
                    const int64_t i = dealt(round, items);
                    const uint32_t at = uint32_t(round % kItems);
                    Item q = {};
                    q.last = true;
                    if (i >= 0) q = item_at<PAIR>(a, i);
                    more = !q.last;
                    ok = round < kItems || bw::bar_wait_idle(bar(&h.item_free[at]), uint32_t(round / kItems - 1) & 1, gave_up,
                                                             until);
                    if (!ok) break;
                    h.items[at] = q;
                    bw::bar_arrive(bar(&h.item_full[at]));
                    // the queries come to the L2
                    for (int x = 0; x < 2; ++x)
                        for (int b = 0; b < kBoxes && q.blocks[x] > 0; ++b) bw::fetch_3d(&map_q, 64 * b, q.head[x], q.row0[x]);
                }
            }
        }
    } else if (warp >= 8) {  // finished rows
        bw::fewer_registers<kOtherRegs>();
        const int w = warp & 3, r = w * 32 + lane;
        const uint32_t at_y = tmem + (uint32_t(w * 32) << 16) + 2 * kTile;
        const bool wide = a.D % 8 == 0 && (reinterpret_cast<uintptr_t>(a.y) & 15) == 0;
        const float scale = a.scale * kLog2e;
        uint32_t done[2] = {0, 0};
        bool ok = true;
        Item q;
        for (uint32_t item = 0; ok && item_of_warp(item, q); ++item) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                T *y = static_cast<T *>(a.y) + (int64_t(q.row0[x]) + r) * a.heads * a.D + int64_t(q.head[x]) * a.D;
                float *lse = a.lse + q.head[x] * a.tokens + q.row0[x] + r;
                if (q.blocks[x] == 0) {
                    if (r < q.rows[x]) {  // of no sequence
                        put_zeros(y, a.D, wide);
                        *lse = 0.0f;
                    }
                    continue;
                }
                const uint32_t phase = done[x]++ & 1;
                ok = ok && bw::bar_wait_inline(bar(&h.l_full[x]), phase, gave_up, until) &&
                     bw::bar_wait_inline(bar(&h.y_full[x]), phase, gave_up, until);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                bw::fence_after();
                const float l = h.row_l[x][r], m = h.row_m[x][r], by = 1.0f / l;
#pragma unroll 1
                for (int d = 0; d < DP; d += 32) {
                    float v[32];
                    __syncwarp();
                    bw::tmem_load(at_y + x * DP + d, v);
                    if (d + 32 == DP) {
                        bw::fence_before();
                        __syncwarp();
                        if (lane == 0) bw::bar_arrive(bar(&h.y_free[x]));
                    }
                    if (r < q.rows[x]) put_row(y + d, v, by, a.D - d, wide);
                }
                if (r < q.rows[x]) *lse = (m * scale + (log2f(l) - kPPower<T>)) * kLn2;
            }
        }
    } else {  // softmax
        bw::more_registers<kSoftmaxRegs>();
        const int x = warp >> 2, w = warp & 3, r = w * 32 + lane;
        const uint32_t lanes = tmem + (uint32_t(w * 32) << 16);
        const uint32_t at_s = lanes + x * kTile, at_y = lanes + 2 * kTile + x * DP;
        const float scale = a.scale * kLog2e;  // positive, so that unscaled scores can be compared
        uint32_t blocks = 0, done = 0, c = 0, checks = 0;  // blocks and rounds of this tile; blocks of the ring; checks
        bool ok = true;
        Item q;
        for (uint32_t item = 0; ok && item_of_warp(item, q); ++item) {
            const int n = q.blocks[x];
            float m = -INFINITY, l = 0.0f;
            auto hand_over = [&](uint64_t(&to)[2]) {  // P so far, to the products
                bw::tmem_stored();
                bw::fence_before();
                __syncwarp();
                if (lane == 0) bw::bar_arrive(bar(&to[x]));
            };
            for (int j = 0; j < n; ++j) {
                ok = __all_sync(0xffffffffu, bw::bar_wait_inline(bar(&h.s_full[x]), blocks++ & 1, gave_up, until));
                if (!ok) break;
                bw::fence_after();
                float s[kTile];
                {
                    float(&lo)[64] = *reinterpret_cast<float(*)[64]>(s), (&hi)[64] = *reinterpret_cast<float(*)[64]>(s + 64);
                    bw::tmem_load(at_s, lo);
                    bw::tmem_load(at_s + 64, hi);
                }
                const bool diagonal = j == n - 1;
                if (diagonal) {  // a warp's rows see all of the 32 keys before theirs, and none of those after
#pragma unroll
                    for (int e0 = 0; e0 < kTile; e0 += 32) {
                        if (e0 < w * 32) continue;
                        const int last = e0 == w * 32 ? lane : -1;
#pragma unroll
                        for (int e = 0; e < 32; ++e) s[e0 + e] = e <= last ? s[e0 + e] : -INFINITY;
                    }
                }
                float top[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = fmaxf(s[2 * e], s[2 * e + 1]);
#pragma unroll
                for (int e = 8; e < kTile; e += 2) top[e / 2 & 3] = max3(top[e / 2 & 3], s[e], s[e + 1]);
                const float most = fmaxf(max3(top[0], top[1], top[2]), top[3]);
                const float raised = fmaxf(m, most);
                // (a row by its own scores alone: its bits do not depend on its neighbours)
                const bool low = !((raised - m) * scale <= kSlack);
                if (__any_sync(0xffffffffu, low)) {
                    // y is not in use: the products before these scores are done
                    float old = 1.0f;
                    if (low) {
                        old = m == -INFINITY ? 0.0f : exp2_fast((m - raised) * scale);
                        m = raised;
                        l *= old;
                    }
                    if (j > 0) {
#pragma unroll 1
                        for (int d = 0; d < DP; d += 32) {
                            float v[32];
                            bw::tmem_load(at_y + d, v);
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] *= old;
                            bw::tmem_store(at_y + d, v);
                        }
                    }
                }
                // nothing but -inf so far: any finite reference will do
                const float2 minus = twice(kPPower<T> + (m == -INFINITY ? 0.0f : -m * scale)), by = twice(scale);
                float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
                for (int e0 = 0; e0 < kTile; e0 += 32) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float2 t = __ffma2_rn(make_float2(s[e0 + e], s[e0 + e + 1]), by, minus);
                        t.x = exp2_fast(t.x);
                        t.y = exp2_fast(t.y);
                        sum[e / 2 & 1] = __fadd2_rn(sum[e / 2 & 1], t);
                        p[e / 2] = pack2(t.x, t.y, T());
                    }
                    bw::tmem_store(at_s + e0 / 2, p);
                    // the first half's products may start
                    if (e0 == 32 && !diagonal) hand_over(h.p_half);
                }
                sum[0] = __fadd2_rn(sum[0], sum[1]);
                l += sum[0].x + sum[0].y;
                if (diagonal) {
                    bw::tmem_stored();
                    const uint32_t check = checks + (PAIR ? 0 : x), v = c + 2 * j + 1;
                    ok = bw::bar_wait_inline(bar(&h.checked[check % kChecks]), (check / kChecks) & 1, gave_up, until);
                    // y, l and m of the rows before have been read
                    ok = ok && (done == 0 || bw::bar_wait_inline(bar(&h.y_free[x]), (done - 1) & 1, gave_up, until));
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    h.row_l[x][r] = l;
                    h.row_m[x][r] = m;
                    if (is_by_hand(check))
                        masked_product<T, DP>(at_y, [&](int g) { return at_s + g * 16; }, 4,
                                              dyn + (kQ + v % kStages) * kBytes, 0, 0, r + 1, j > 0);
                    hand_over(h.p_half);
                    if (lane == 0) bw::bar_arrive(bar(&h.l_full[x]));
                }
                hand_over(h.p_full);
            }
            c += 2 * max(q.blocks[0], q.blocks[1]);
            checks += checks_of<PAIR>(q);
            done += n > 0;
        }
    }
    __syncwarp();
    if (*const_cast<volatile uint32_t *>(gave_up)) {
        // copies and products in flight still write this CTA's memory: let them end
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
        if (threadIdx.x == 0 && a.status) *a.status = DC_ERR_INTERNAL;
    }
    bw::fence_before();
    __syncthreads();
    if (warp == 13) bw::tmem_free1(tmem, 512);
}

// ------------------------------------------------------------------------------ host
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                 const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

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

template <typename T, int DP, bool PAIR>
cudaError_t launch(int dtype, const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    CUtensorMap q, k, v;
    if (!am::heads_map(q, dtype, a.q, a.D, a.heads, a.tokens, a.q_head, a.q_token) ||
        !am::heads_map(k, dtype, a.k, a.D, a.kv_heads, a.tokens, a.k_head, a.k_token) ||
        !am::heads_map(v, dtype, a.v, a.D, a.kv_heads, a.tokens, a.v_head, a.v_token))
        return cudaErrorInvalidValue;
    auto kernel = attention_mma_kernel<T, DP, PAIR>;
    constexpr size_t smem = (kTilesOfQ<DP> + kRing<DP>) * size_t(DP / 64) * kBox + kSharedBytes;
    static_assert(smem <= 232448, "shared memory of a CTA");
    static DeviceCache cache;
    int ready = 0, sms = 0;
    cudaError_t e = cache.get(ready, [&](int &n) {
        n = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
    });
    if (e == cudaSuccess) e = sm_count(sms);
    if (e != cudaSuccess) return e;
    const int64_t items = most * (PAIR ? a.heads / 2 : a.heads);
    return launch_early(kernel, items < sms ? items : sms, kThreads, smem, stream, q, k, v, a);
}

}  // namespace

namespace am {

bool heads_map(CUtensorMap &map, int dtype, const void *base, int32_t D, int32_t heads, int64_t tokens, int64_t head,
               int64_t token)
{
    const EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    // a dimension of one element has no stride of its own, but it has to be valid
    const int64_t row = (D + 7) / 8 * 8;
    if (heads == 1) head = row;
    if (tokens == 1) token = heads * head;
    const cuuint64_t dims[3] = {cuuint64_t(D), cuuint64_t(heads), cuuint64_t(tokens)};
    const cuuint64_t strides[2] = {cuuint64_t(head) * 2, cuuint64_t(token) * 2};
    const cuuint32_t box[3] = {64, 1, kTile}, one[3] = {1, 1, 1};
    return encode(&map, dtype == DC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
                  const_cast<void *>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace am

// Two heads of a group at a time; tiles of two blocks where the group is odd.
int attention_mma_rows(const AttentionArgs &a) { return a.group % 2 == 0 ? kMmaRows : 2 * kMmaRows; }

cudaError_t launch_attention_mma(int dtype, const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    const bool pair = a.group % 2 == 0;
    auto go = [&](auto t) {
        using T = decltype(t);
        if (a.D <= 64)
            return pair ? launch<T, 64, true>(dtype, a, most, stream) : launch<T, 64, false>(dtype, a, most, stream);
        return pair ? launch<T, 128, true>(dtype, a, most, stream) : launch<T, 128, false>(dtype, a, most, stream);
    };
    return dtype == DC_BF16 ? go(__nv_bfloat16()) : go(__half());
}

}  // namespace dc
