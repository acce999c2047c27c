// The gradient of causal attention of 16-bit types on the tensor cores.
//
//   P = 2^(scale' S - lse'), dS = P (dy v^T - delta), delta = dy . y
//   columns: a tile of 128 keys and a key head, over its group's heads and the rows from it on:
//            S^T = k q^T, dP^T = v dy^T, dv += P^T dy, dk += dS^T q
//   rows:    a tile of 128 rows and a head, over the keys up to it: S = q k^T, dP = dy v^T, dq += dS k,
//            b += P k
// Seven products a block instead of the five that one pass would need: dq of one pass would be summed
// by many CTAs, in memory and in an order that depends on timing; so each sum has one owner.
// The eighth, b, takes back what y's rounding does to delta: as a row of P sums to one, a row of dS sums to zero,
// and what it sums to instead, E, is what delta lacks. So the rows' pass comes first, gives dq - E b, and leaves
// delta + E for the columns' (in rows of 16 keys bfloat16's dq is 4.0e-3 off without, 2.3 with; 1.6 is its own
// rounding). Where tiles and key heads are few, a group's heads are dealt to several CTAs, whose sums are joined
// afterwards.
//
// Both are one kernel: two stationary tiles, two rings of moving ones (X: q or k, Y: dy or v), scores
// and dP in tensor memory [128][128], the sums [128][D] beside them, 512 columns in all.
//   warps 0-7  a lane a row, four warps either half of the columns: P, then dS, in 16 bits over what
//              they were made of (A operands may lie in tensor memory)
//   warp 8     copies (TMA)       warp 9  products, by one thread
//   warp 10    columns: lse and delta of each block's rows
//   warp 11    looks through the blocks that a mask cuts
// The products of one kind run while the warps make the other: S of the next block and dv beside dS,
// dP of the next block and dk beside P.
//
// Measured (one GB300): 32,768 tokens in 14 sequences x 32 heads on 8 x 128, rows 1,119 us, columns 1,380 us; one
// prompt of 16,384 x 16 x 128 2.51 ms, 1,752 TFLOP/s of the eight products. Tensor cores busy 75-81 % of the time; heads
// of 64 are bound by the warps: a step of 128 x 128 takes them 1,900 clocks (rows) and 2,500 (columns; halves 2,700), the
// products 1,024.
//
// Rounding: P and dS are rounded to the operands' type for the tensor cores, half a step of each
// term. Halves have few exponents: P, at most 1, is held 2^14 times larger, and dS in a power of
// two of the lane's own, row or key, that nothing which it may see can overflow (attention_plan.cu); both are
// undone in floats at the end. What a mask hides is zero by selection, and operands' rows behind it are
// looked through as in the forward pass.
#include <cmath>

#include "attention_mma.cuh"

namespace dc {
namespace {

using namespace am;

constexpr int kThreads = 12 * 32;
constexpr int kChecks = 4;  // no more blocks that a mask cuts are in a ring
constexpr float kLog2e = 1.4426950408889634f;

template <int DP, bool COLUMNS>
struct Shape {
    static constexpr uint32_t kBytes = DP / 64 * kBox;
    static constexpr int kX = DP == 64 ? 4 : 3, kY = DP == 64 ? 4 : 2, kL = 2;
    static constexpr uint32_t kTiles = (2 + kX + kY) * kBytes;
    static constexpr uint32_t kStats = (COLUMNS ? kL * 2 : 2) * kTile * sizeof(float);
    static constexpr uint32_t kBars = 512;
    static constexpr uint32_t kSmem = kTiles + kStats + kBars;
};

// A block of columns: its first row (key), how many there are of it, the head, and whether the mask cuts it.
struct Step {
    int32_t head, c0, count;
    bool diagonal, cut;
};
// Where an item's work is: the head of the group, and its block.
struct Walk {
    int32_t head = 0, block = 0;
    __device__ __forceinline__ void next(int per_head)
    {
        if (++block == per_head) {
            block = 0;
            ++head;
        }
    }
};
template <bool COLUMNS>
struct Item {
    AttentionTile t;
    int32_t outer, kv, part, head0, per_head, steps;
    __device__ __forceinline__ Step step(const Walk &w) const
    {
        Step s;
        s.head = head0 + w.head;
        s.c0 = (COLUMNS ? t.row0 : t.first) + w.block * kTile;
        s.count = min(kTile, (COLUMNS ? t.end : t.row0 + t.rows) - s.c0);
        s.diagonal = w.block == (COLUMNS ? 0 : per_head - 1);
        s.cut = s.diagonal || (COLUMNS && s.count < kTile);
        return s;
    }
};
template <bool COLUMNS>
__device__ __forceinline__ Item<COLUMNS> item_at(const AttentionArgs &a, int64_t i)
{
    const int outer = COLUMNS ? a.kv_heads * a.split : a.heads;
    Item<COLUMNS> q;
    const int64_t at = i < (int64_t(1) << 31) ? int64_t(uint32_t(i) / uint32_t(outer)) : i / outer;
    q.t = plan_tiles(a.plan)[at];
    const int j = int(i - at * outer);
    q.part = COLUMNS ? j / a.kv_heads : 0;
    q.outer = j - q.part * a.kv_heads;
    q.kv = COLUMNS ? q.outer : q.outer / a.group;
    q.head0 = COLUMNS ? q.kv * a.group + q.part * a.group / a.split : q.outer;
    if (q.t.first < 0) {
        q.per_head = q.steps = 0;
        return q;
    }
    const int n = (q.t.end - q.t.first + kTile - 1) / kTile, before = (q.t.row0 - q.t.first) / kTile;
    if (COLUMNS) {  // tile i from the end has the work of tile i from the start
        q.t.row0 = q.t.first + (n - 1 - before) * kTile;
        q.t.rows = min(kTile, q.t.end - q.t.row0);
        q.per_head = before + 1;
        q.steps = q.per_head * ((q.part + 1) * a.group / a.split - q.part * a.group / a.split);
    } else {
        q.per_head = q.steps = before + 1;
    }
    return q;
}

template <typename T, int DP, bool COLUMNS>
__global__ void __launch_bounds__(kThreads, 1)
attention_grad_mma_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                          const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_dy,
                          const AttentionArgs a)
{
    using G = Shape<DP, COLUMNS>;
    constexpr int kBoxes = DP / 64;
    constexpr uint32_t kBytes = G::kBytes;
    constexpr bool kHalf = std::is_same<T, __half>::value;
    constexpr int kPPower = kHalf ? 14 : 0;  // P is held 2^kPPower times larger
    extern __shared__ __align__(1024) unsigned char dyn[];
    struct Bars {
        uint64_t still_full, still_free, x_full[G::kX], x_free[G::kX], y_full[G::kY], y_free[G::kY], l_full[G::kL],
            l_free[G::kL], s_full, p_full, dp_full, ds_full, sums_full, met, last,
            look[kChecks], x_checked[kChecks], y_checked[kChecks];
        uint32_t tmem_at, gave_up;
        uint32_t progress;  // blocks done: an item takes as long as its rows are many, and so do some waits
        // the check, counted from one, if the sums with its block of X (Y) are done by hand
        uint32_t x_by_hand[kChecks], y_by_hand[kChecks];
    };
    static_assert(sizeof(Bars) <= G::kBars, "barriers' room");
    Bars &b = *reinterpret_cast<Bars *>(dyn + G::kTiles + G::kStats);
    float *const stats = reinterpret_cast<float *>(dyn + G::kTiles);  // columns: [kL][lse, delta][128]; rows: [2][128], E

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto bar = [](uint64_t *p) { return bw::smem_addr(p); };
    const uint32_t base = bw::smem_addr(dyn), ring_x = base + 2 * kBytes, ring_y = ring_x + G::kX * kBytes;
    uint32_t *const gave_up = &b.gave_up;
    volatile uint32_t *const progress = &b.progress;

    if (threadIdx.x == 0) {
        bw::bar_init(bar(&b.still_full), 1);
        bw::bar_init(bar(&b.still_free), 1);
        for (int i = 0; i < G::kX; ++i) {
            bw::bar_init(bar(&b.x_full[i]), 1);
            bw::bar_init(bar(&b.x_free[i]), 1);
        }
        for (int i = 0; i < G::kY; ++i) {
            bw::bar_init(bar(&b.y_full[i]), 1);
            bw::bar_init(bar(&b.y_free[i]), 1);
        }
        for (int i = 0; i < G::kL; ++i) {
            bw::bar_init(bar(&b.l_full[i]), 1);
            bw::bar_init(bar(&b.l_free[i]), 8);
        }
        bw::bar_init(bar(&b.s_full), 1);
        bw::bar_init(bar(&b.p_full), 8);
        bw::bar_init(bar(&b.dp_full), 1);
        bw::bar_init(bar(&b.ds_full), 8);
        bw::bar_init(bar(&b.sums_full), 1);
        bw::bar_init(bar(&b.met), 8);
        bw::bar_init(bar(&b.last), 1);
        for (int i = 0; i < kChecks; ++i) {
            bw::bar_init(bar(&b.look[i]), 1);
            bw::bar_init(bar(&b.x_checked[i]), 1);
            bw::bar_init(bar(&b.y_checked[i]), 1);
            b.x_by_hand[i] = b.y_by_hand[i] = 0;
        }
        b.gave_up = b.progress = 0;
        bw::bar_init_fence();
    }
    if (warp == 9) bw::tmem_alloc1(bw::smem_addr(&b.tmem_at), 512);
    if (warp == 8 && lane == 0) {
        bw::prefetch_map(&map_q);
        bw::prefetch_map(&map_k);
        bw::prefetch_map(&map_v);
        bw::prefetch_map(&map_dy);
    }
    pdl_wait();  // the list, the copies and delta are there (for columns, from the rows' pass)
    bw::fence_before();
    __syncthreads();
    bw::fence_after();
    const uint32_t tmem = b.tmem_at;
    constexpr uint32_t kDp = kTile, kSum1 = 2 * kTile, kSum0 = kSum1 + DP;  // columns: dv or b, and dk or dq
    // A operand of step i of eight: pairs of 16 columns; the halves are 64 columns apart
    auto packed_at = [](int i) { return uint32_t(i / 4 * 64 + i % 4 * 8); };
    auto by_hand = [&](const uint32_t(&of)[kChecks], uint32_t check) {
        return *const_cast<const volatile uint32_t *>(&of[check % kChecks]) == check + 1;
    };
    // the swizzled copies need tiles on 1,024-byte boundaries
    const int64_t items = (base & 1023u) ? 0 : int64_t(a.plan->tiles) * (COLUMNS ? a.kv_heads * a.split : a.heads);
    if ((base & 1023u) && threadIdx.x == 0) b.gave_up = 1;

    if (warp == 8) {
        if (bw::elect_one()) {  // copies
            int done = 0;
            uint32_t nx = 0, ny = 0;
            bool ok = true;
            auto tile = [&](uint32_t to, const CUtensorMap &map, int head, int row, uint32_t full) {
                for (int i = 0; i < kBoxes; ++i) bw::copy_3d1(to + i * kBox, &map, 64 * i, head, row, full);
            };
            uint32_t checks = 0;
            int64_t i = dealt(0, items);
            Item<COLUMNS> next = {};
            if (i >= 0) next = item_at<COLUMNS>(a, i);
            for (int64_t round = 1; ok && i >= 0; ++round) {
                const Item<COLUMNS> q = next;
                // the next item is looked up, and its stationary tiles come to the L2, while this one is at work
                i = dealt(round, items);
                if (i >= 0) {
                    next = item_at<COLUMNS>(a, i);
                    const int head = COLUMNS ? next.kv : next.outer;
                    for (int d = 0; d < kBoxes && next.steps > 0; ++d) {
                        bw::fetch_3d(COLUMNS ? &map_k : &map_q, 64 * d, head, next.t.row0);
                        bw::fetch_3d(COLUMNS ? &map_v : &map_dy, 64 * d, head, next.t.row0);
                    }
                }
                if (q.steps == 0) continue;
                ok = done == 0 || bw::bar_wait(bar(&b.still_free), (done - 1) & 1, gave_up, progress);
                if (!ok) break;
                ++done;
                bw::bar_arrive_bytes(bar(&b.still_full), 2 * kBytes);
                tile(base, COLUMNS ? map_k : map_q, COLUMNS ? q.kv : q.outer, q.t.row0, bar(&b.still_full));
                tile(base + kBytes, COLUMNS ? map_v : map_dy, COLUMNS ? q.kv : q.outer, q.t.row0, bar(&b.still_full));
                Walk w;
                for (int j = 0; j < q.steps; ++j, w.next(q.per_head)) {
                    const Step s = q.step(w);
                    const int head = COLUMNS ? s.head : q.kv;
                    const uint32_t x = nx % G::kX, y = ny % G::kY;
                    ok = nx < G::kX || bw::bar_wait(bar(&b.x_free[x]), (nx / G::kX - 1) & 1, gave_up, progress);
                    if (!ok) break;
                    bw::bar_arrive_bytes(bar(&b.x_full[x]), kBytes);
                    tile(ring_x + x * kBytes, COLUMNS ? map_q : map_k, head, s.c0, bar(&b.x_full[x]));
                    ++nx;
                    ok = ny < G::kY || bw::bar_wait(bar(&b.y_free[y]), (ny / G::kY - 1) & 1, gave_up, progress);
                    if (!ok) break;
                    bw::bar_arrive_bytes(bar(&b.y_full[y]), kBytes);
                    tile(ring_y + y * kBytes, COLUMNS ? map_dy : map_v, head, s.c0, bar(&b.y_full[y]));
                    ++ny;
                    // to be looked through: the barriers' phases have begun, and do not end twice before that
                    if (s.cut) bw::bar_arrive(bar(&b.look[checks++ % kChecks]));
                }
            }
        }
    } else if (warp == 9) {
        if (bw::elect_one()) {  // products
            constexpr bool kBf = !kHalf;
            const uint32_t shape_s = bw::f16_shape(kBf, false, false, kTile, kTile);
            const uint32_t shape_d = bw::f16_shape(kBf, false, true, kTile, DP);
            int done = 0;
            uint32_t n = 0;  // blocks so far
            bool ok = true;
            auto x_there = [&](uint32_t m) {
                return ok = ok && bw::bar_wait(bar(&b.x_full[m % G::kX]), (m / G::kX) & 1, gave_up, progress);
            };
            auto y_there = [&](uint32_t m) {
                return ok = ok && bw::bar_wait(bar(&b.y_full[m % G::kY]), (m / G::kY) & 1, gave_up, progress);
            };
            auto scores = [&](uint32_t d, uint32_t still, uint32_t moving) {
                const uint64_t da = bw::operand(still, 16), db = bw::operand(moving, 16);
                bw::fence_after();
#pragma unroll
                for (int i = 0; i < DP / 16; ++i) {
                    const uint64_t at = (i / 4) * (kBox >> 4) + (i % 4) * 2;
                    bw::mma1(tmem + d, da + at, db + at, shape_s, i > 0);
                }
            };
            auto sums = [&](uint32_t d, uint32_t packed, uint32_t moving, bool add) {
                const uint64_t db = bw::operand(moving, kBox);
#pragma unroll
                for (int i = 0; i < kTile / 16; ++i)
                    bw::mma1_tmem(tmem + d, tmem + packed + packed_at(i), db + i * 128, shape_d, add || i > 0);
            };
            uint32_t checks = 0;
            int64_t i = dealt(0, items);
            Item<COLUMNS> next = {};
            if (i >= 0) next = item_at<COLUMNS>(a, i);
            for (int64_t round = 1; ok && i >= 0; ++round) {
                const Item<COLUMNS> q = next;
                i = dealt(round, items);
                if (q.steps == 0) {
                    if (i >= 0) next = item_at<COLUMNS>(a, i);
                    continue;
                }
                ok = bw::bar_wait(bar(&b.still_full), done & 1, gave_up, progress);
                ++done;
                auto first = [&](uint32_t m) {  // S of block m
                    if (!x_there(m)) return;
                    scores(0, base, ring_x + m % G::kX * kBytes);
                    bw::commit1(bar(&b.s_full));
                };
                auto second = [&](uint32_t m, bool end) {  // dP
                    if (!y_there(m)) return;
                    scores(kDp, base + kBytes, ring_y + m % G::kY * kBytes);
                    bw::commit1(bar(&b.dp_full));
                    if (!COLUMNS) bw::commit1(bar(&b.y_free[m % G::kY]));
                    if (end) bw::commit1(bar(&b.still_free));
                };
                first(n);
                second(n, q.steps == 1);
                if (i >= 0) next = item_at<COLUMNS>(a, i);  // looked up while this one is at work
                Walk w;
                for (int j = 0; j < q.steps && ok; ++j, ++n, w.next(q.per_head)) {
                    const Step s = q.step(w);
                    ok = bw::bar_wait(bar(&b.p_full), n & 1, gave_up, progress);
                    if (!ok) break;
                    bw::fence_after();
                    if (!s.diagonal || !by_hand(COLUMNS ? b.y_by_hand : b.x_by_hand, checks))
                        sums(kSum1, 0, COLUMNS ? ring_y + n % G::kY * kBytes : ring_x + n % G::kX * kBytes, j > 0);
                    if (COLUMNS) bw::commit1(bar(&b.y_free[n % G::kY]));
                    if (j + 1 < q.steps) first(n + 1);
                    ok = ok && bw::bar_wait(bar(&b.ds_full), n & 1, gave_up, progress);
                    if (!ok) break;
                    bw::fence_after();
                    if (!s.diagonal || !by_hand(b.x_by_hand, checks)) sums(kSum0, kDp, ring_x + n % G::kX * kBytes, j > 0);
                    checks += s.cut;
                    *progress = n + 1;
                    bw::commit1(bar(&b.x_free[n % G::kX]));
                    if (j + 1 < q.steps) second(n + 1, j + 2 == q.steps);
                }
                if (ok) bw::commit1(bar(&b.sums_full));
            }
            // arrivals land in this CTA's memory: it may not end before the last
            bw::commit1(bar(&b.last));
            bw::bar_wait(bar(&b.last), 0, gave_up, progress);
        }
    } else if (warp == 10) {
        if (COLUMNS) {  // lse and delta, as the warps use them
            uint32_t n = 0;
            bool ok = true;
            for (int64_t round = 0, i; ok && (i = dealt(round, items)) >= 0; ++round) {
                const Item<COLUMNS> q = item_at<COLUMNS>(a, i);
                Walk w;
                for (int j = 0; j < q.steps; ++j, ++n, w.next(q.per_head)) {
                    const Step s = q.step(w);
                    const int64_t at = s.head * a.tokens + s.c0;
                    float l[4], d[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int c = lane + 32 * k;
                        l[k] = c < s.count ? a.lse[at + c] : 0.0f;
                        d[k] = c < s.count ? a.delta[at + c] : 0.0f;
                    }
                    ok = n < G::kL || bw::bar_wait(bar(&b.l_free[n % G::kL]), (n / G::kL - 1) & 1, gave_up, progress);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    float *to = stats + n % G::kL * 2 * kTile;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        to[lane + 32 * k] = -l[k] * kLog2e + float(kPPower);
                        to[kTile + lane + 32 * k] = -d[k];
                    }
                    __syncwarp();
                    if (lane == 0) bw::bar_arrive(bar(&b.l_full[n % G::kL]));
                }
            }
        }
    } else if (warp == 11) {  // blocks that a mask cuts
        uint32_t n = 0, checks = 0;
        bool ok = true;
        for (int64_t round = 0, i; ok && (i = dealt(round, items)) >= 0; ++round) {
            const Item<COLUMNS> q = item_at<COLUMNS>(a, i);
            Walk w;
            for (int j = 0; j < q.steps; ++j, ++n, w.next(q.per_head)) {
                const Step s = q.step(w);
                if (!s.cut) continue;
                const uint32_t at = checks % kChecks;
                ok = bw::bar_wait(bar(&b.look[at]), (checks / kChecks) & 1, gave_up, progress);
                // rows behind the mask: of Y where it is summed too, and of X
                for (int of_x = COLUMNS ? 0 : 1; of_x < 2; ++of_x) {
                    const uint32_t stage = of_x ? n % G::kX : n % G::kY, phase = of_x ? n / G::kX : n / G::kY;
                    ok = __all_sync(0xffffffffu, ok && bw::bar_wait(bar(of_x ? &b.x_full[stage] : &b.y_full[stage]), phase & 1,
                                                                     gave_up, progress));
                    if (!ok) break;
                    unsigned char *const tile = dyn + (2 + (of_x ? 0 : G::kX) + stage) * kBytes;
                    bool bad = false;
                    for (int r = lane; r < kTile; r += 32) bad |= look_through<T, DP>(tile, r, s.count);
                    if (bad && s.diagonal)
                        *const_cast<volatile uint32_t *>(of_x ? &b.x_by_hand[at] : &b.y_by_hand[at]) = checks + 1;
                    __syncwarp();
                    if (lane == 0) bw::bar_arrive(bar(of_x ? &b.x_checked[at] : &b.y_checked[at]));
                }
                if (!ok) break;
                ++checks;
            }
        }
    } else {  // P, dS and the finished sums
        const int side = warp >> 2, r = (warp & 3) * 32 + lane;
        const uint32_t lanes = tmem + (uint32_t((warp & 3) * 32) << 16);
        const uint32_t at_s = lanes + side * 64, at_dp = at_s + kDp;
        const float scale = a.scale * kLog2e, by1 = ldexpf(1.0f, -kPPower);
        const bool wide = a.D % 8 == 0 && ((reinterpret_cast<uintptr_t>(COLUMNS ? a.dk : a.dq) |
                                            reinterpret_cast<uintptr_t>(COLUMNS ? a.dv : a.dq)) & 15) == 0;
        const float2 by = twice(scale);
        uint32_t n = 0, finished = 0, checks = 0;
        bool ok = true;
        uint32_t meetings = 0;
        auto meet = [&] {  // all eight warps
            bw::fence_before();
            __syncwarp();
            if (lane == 0) bw::bar_arrive(bar(&b.met));
            ok = __all_sync(0xffffffffu, bw::bar_wait(bar(&b.met), meetings++ & 1, gave_up, progress) && ok);
            bw::fence_after();
        };
        for (int64_t round = 0, i; ok && (i = dealt(round, items)) >= 0; ++round) {
            const Item<COLUMNS> q = item_at<COLUMNS>(a, i);
            const int64_t row = (int64_t(q.t.row0) + r) * (COLUMNS ? a.kv_heads : a.heads) * a.D + int64_t(q.outer) * a.D;
            T *const out = static_cast<T *>(!COLUMNS ? a.dq : side ? a.dk : a.dv) + row;
            float *const part = !COLUMNS || a.split == 1 ? nullptr
                                : a.partial + ((side ? 0 : a.split) + q.part) * a.tokens * a.kv_heads * a.D + row;
            if (q.steps == 0) {  // rows of no sequence
                if (r < q.t.rows && (COLUMNS || side == 0)) {
                    if (part)
                        for (int d = 0; d < a.D; ++d) part[d] = 0.0f;
                    else
                        put_zeros(out, a.D, wide);
                }
                continue;
            }
            float2 lse = {}, delta = {}, excess = {};  // excess: rows, what dS sums to
            const int64_t own = q.outer * a.tokens + q.t.row0 + r;  // the lane's row or key
            const bool there = r < q.t.rows;
            const int power = kHalf && there ? (COLUMNS ? a.key_power : a.row_power)[own] : 0;
            const float2 fs = twice(ldexpf(1.0f, power - kPPower));
            if (!COLUMNS) {
                lse = twice((there ? -a.lse[own] * kLog2e : 0.0f) + float(kPPower));
                delta = twice(there ? -a.delta[own] * fs.x : 0.0f);
            }
            Walk w;
            for (int j = 0; j < q.steps; ++j, ++n, w.next(q.per_head)) {
                const Step s = q.step(w);
                const float *const l = stats + n % G::kL * 2 * kTile + side * 64;
                ok = bw::bar_wait(bar(&b.s_full), n & 1, gave_up, progress);
                if (COLUMNS) ok = ok && bw::bar_wait(bar(&b.l_full[n % G::kL]), (n / G::kL) & 1, gave_up, progress);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                bw::fence_after();
                // columns of this side that count: rows from the key on, or keys up to the row
                const bool cut = s.cut;
                const int from = (COLUMNS && s.diagonal ? r : 0) - side * 64;
                const int end = (!COLUMNS && s.diagonal ? r + 1 : s.count) - side * 64;
                float p[64];
                bw::tmem_load(at_s, p);
                auto make_p = [&](auto masked) {
#pragma unroll
                    for (int e0 = 0; e0 < 64; e0 += 32) {
                        uint32_t out16[16];
#pragma unroll
                        for (int e = e0; e < e0 + 32; e += 4) {
                            const float4 minus = COLUMNS ? *reinterpret_cast<const float4 *>(l + e)
                                                         : make_float4(lse.x, lse.x, lse.x, lse.x);
                            const float2 t = __ffma2_rn(make_float2(p[e], p[e + 1]), by, make_float2(minus.x, minus.y));
                            const float2 u = __ffma2_rn(make_float2(p[e + 2], p[e + 3]), by, make_float2(minus.z, minus.w));
                            p[e] = exp2_fast(t.x);
                            p[e + 1] = exp2_fast(t.y);
                            p[e + 2] = exp2_fast(u.x);
                            p[e + 3] = exp2_fast(u.y);
                            if constexpr (decltype(masked)::value)
#pragma unroll
                                for (int k = e; k < e + 4; ++k) p[k] = k >= from && k < end ? p[k] : 0.0f;
                            out16[(e - e0) / 2] = pack2(p[e], p[e + 1], T());
                            out16[(e - e0) / 2 + 1] = pack2(p[e + 2], p[e + 3], T());
                        }
                        bw::tmem_store(at_s + e0 / 2, out16);
                    }
                };
                // most blocks are whole: the mask's selections would double the work of a block
                if (cut) make_p(std::true_type());
                else make_p(std::false_type());
                bw::tmem_stored();
                const uint32_t at = checks % kChecks, check_phase = (checks / kChecks) & 1;
                // what P is multiplied with (Y, or X) has been looked through
                bool hand = false;
                if (cut) {
                    ok = __all_sync(0xffffffffu, bw::bar_wait(bar(COLUMNS ? &b.y_checked[at] : &b.x_checked[at]), check_phase,
                                                              gave_up, progress));
                    if (!ok) break;
                    hand = s.diagonal && by_hand(COLUMNS ? b.y_by_hand : b.x_by_hand, checks);
                    if (hand) {
                        meet();
                        if (!ok) break;
                        if (side == 0)
                            masked_product<T, DP>(lanes + kSum1, [&](int g) { return lanes + packed_at(2 * g); }, 4,
                                                  dyn + (COLUMNS ? 2 + G::kX + n % G::kY : 2 + n % G::kX) * kBytes, 0,
                                                  COLUMNS ? r : 0, COLUMNS ? s.count : r + 1, j > 0);
                    }
                }
                bw::fence_before();
                __syncwarp();
                if (lane == 0) bw::bar_arrive(bar(&b.p_full));
                ok = __all_sync(0xffffffffu, ok && bw::bar_wait(bar(&b.dp_full), n & 1, gave_up, progress));
                if (!ok) break;
                bw::fence_after();
                auto make_ds = [&](auto masked) {
#pragma unroll
                    for (int e0 = 0; e0 < 64; e0 += 32) {
                        float d[32];
                        bw::tmem_load(at_dp + e0, d);
                        uint32_t out16[16];
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 minus = COLUMNS ? *reinterpret_cast<const float4 *>(l + kTile + e0 + e)
                                                         : make_float4(delta.x, delta.x, delta.x, delta.x);
                            float2 t = make_float2(d[e], d[e + 1]), u = make_float2(d[e + 2], d[e + 3]);
                            if constexpr (kHalf && !COLUMNS) {  // delta is in the row's scale
                                t = __ffma2_rn(t, fs, make_float2(minus.x, minus.y));
                                u = __ffma2_rn(u, fs, make_float2(minus.z, minus.w));
                            } else {
                                t = __fadd2_rn(t, make_float2(minus.x, minus.y));
                                u = __fadd2_rn(u, make_float2(minus.z, minus.w));
                            }
                            if constexpr (kHalf && COLUMNS) {  // a lane is a key: one product more, 609 -> 652 us of
                                t = __fmul2_rn(t, fs);         // columns (16,384 tokens in 2 sequences x 16 x 64)
                                u = __fmul2_rn(u, fs);
                            }
                            t = __fmul2_rn(t, make_float2(p[e0 + e], p[e0 + e + 1]));
                            u = __fmul2_rn(u, make_float2(p[e0 + e + 2], p[e0 + e + 3]));
                            if constexpr (decltype(masked)::value) {
                                const int k = e0 + e;
                                t.x = k >= from && k < end ? t.x : 0.0f;
                                t.y = k + 1 >= from && k + 1 < end ? t.y : 0.0f;
                                u.x = k + 2 >= from && k + 2 < end ? u.x : 0.0f;
                                u.y = k + 3 >= from && k + 3 < end ? u.y : 0.0f;
                            }
                            if (!COLUMNS) excess = __fadd2_rn(excess, __fadd2_rn(t, u));
                            out16[e / 2] = pack2(t.x, t.y, T());
                            out16[e / 2 + 1] = pack2(u.x, u.y, T());
                        }
                        bw::tmem_store(at_dp + e0 / 2, out16);
                    }
                };
                if (cut) make_ds(std::true_type());
                else make_ds(std::false_type());
                bw::tmem_stored();
                if (cut) {
                    if (COLUMNS) {  // X too
                        ok = __all_sync(0xffffffffu, bw::bar_wait(bar(&b.x_checked[at]), check_phase, gave_up, progress));
                        if (!ok) break;
                        hand = s.diagonal && by_hand(b.x_by_hand, checks);
                    }
                    if (hand) {
                        meet();
                        if (!ok) break;
                        if (side == (COLUMNS ? 1 : 0))
                            masked_product<T, DP>(lanes + kSum0, [&](int g) { return lanes + kDp + packed_at(2 * g); }, 4,
                                                  dyn + (2 + n % G::kX) * kBytes, 0, COLUMNS ? r : 0, COLUMNS ? s.count : r + 1,
                                                  j > 0);
                    }
                    ++checks;
                }
                bw::fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (COLUMNS) bw::bar_arrive(bar(&b.l_free[n % G::kL]));
                    bw::bar_arrive(bar(&b.ds_full));
                }
            }
            ok = ok && bw::bar_wait(bar(&b.sums_full), finished & 1, gave_up, progress);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ++finished;
            bw::fence_after();
            float lacks = 0.0f;
            if (!COLUMNS) {
                // (read long before they are written again: an item's sums wait for every warp)
                stats[side * kTile + r] = excess.x + excess.y;
                meet();
                if (!ok) break;
                lacks = stats[r] + stats[kTile + r];
                if (side == 0 && r < q.t.rows) a.delta[own] += lacks * ldexpf(1.0f, -power);
                lacks *= by1;  // b is P's
            }
            constexpr int kCols = COLUMNS ? DP : DP / 2;  // of a thread
            const int d0 = COLUMNS ? 0 : side * kCols;
            const uint32_t from = lanes + (COLUMNS && side == 0 ? kSum1 : kSum0) + d0;
            const float by_sum = COLUMNS && side == 0 ? by1 : a.scale * ldexpf(1.0f, -power);
#pragma unroll 1
            for (int d = 0; d < kCols; d += 32) {
                float v[32], b_row[32];
                __syncwarp();
                bw::tmem_load(from + d, v);
                if (!COLUMNS) {
                    bw::tmem_load(lanes + kSum1 + d0 + d, b_row);
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] -= lacks * b_row[e];
                }
                if (r >= q.t.rows) continue;
                if (part)
                    put_floats(part + d, v, by_sum, a.D - d);
                else
                    put_row(out + d0 + d, v, by_sum, a.D - d0 - d, wide);
            }
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
    if (warp == 9) bw::tmem_free1(tmem, 512);
}

// ------------------------------------------------------------------------------ host
struct Maps {
    CUtensorMap q, k, v, dy;
};

template <typename T, int DP, bool COLUMNS>
cudaError_t launch(const Maps &m, const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    auto kernel = attention_grad_mma_kernel<T, DP, COLUMNS>;
    constexpr int smem = int(Shape<DP, COLUMNS>::kSmem);
    static_assert(smem <= 232448, "shared memory of a CTA");
    static DeviceCache cache;
    int ready = 0, sms = 0;
    cudaError_t e = cache.get(ready, [&](int &n) {
        n = 1;
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    });
    if (e == cudaSuccess) e = sm_count(sms);
    if (e != cudaSuccess) return e;
    const int64_t items = most * (COLUMNS ? a.kv_heads * a.split : a.heads);
    return launch_early(kernel, items < sms ? items : sms, kThreads, smem, stream, m.q, m.k, m.v, m.dy, a);
}

// The rows' pass first: it completes delta.
template <typename T, int DP>
cudaError_t both(const Maps &m, const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    const cudaError_t e = launch<T, DP, false>(m, a, most, stream);
    return e == cudaSuccess ? launch<T, DP, true>(m, a, most, stream) : e;
}

}  // namespace

cudaError_t launch_attention_grad_mma(int dtype, const AttentionArgs &a, int64_t most, cudaStream_t stream)
{
    Maps m;
    if (!heads_map(m.q, dtype, a.q, a.D, a.heads, a.tokens, a.q_head, a.q_token) ||
        !heads_map(m.k, dtype, a.k, a.D, a.kv_heads, a.tokens, a.k_head, a.k_token) ||
        !heads_map(m.v, dtype, a.v, a.D, a.kv_heads, a.tokens, a.v_head, a.v_token) ||
        !heads_map(m.dy, dtype, a.dy, a.D, a.heads, a.tokens, a.dy_head, a.dy_token))
        return cudaErrorInvalidValue;
    if (dtype == DC_BF16)
        return a.D <= 64 ? both<__nv_bfloat16, 64>(m, a, most, stream) : both<__nv_bfloat16, 128>(m, a, most, stream);
    return a.D <= 64 ? both<__half, 64>(m, a, most, stream) : both<__half, 128>(m, a, most, stream);
}

}  // namespace dc
