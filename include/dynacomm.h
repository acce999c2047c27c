/*
 * dynacomm.h -- C ABI of the GB300 (sm_103a) DynaComm scheduling library.
 *
 * DynaComm (Cai et al., arXiv 2101.07968) splits the parameter pull before the
 * forward pass and the gradient push after the backward pass of one training
 * iteration into contiguous multi-layer transmissions, so that transfers
 * overlap layer computation, and picks the split that minimises the makespan
 * with two dynamic programs (Sec. IV-B, Eq. 8 / Algorithm 3 and Eq. 9 /
 * Algorithm 4). This library solves very many independent instances of that
 * problem (Sec. III-B, the 0-1 program over p and g) at once on one GPU.
 *
 * Conventions that hold for every call below:
 *  - Times are int64 microseconds (the paper uses real-valued times; integer
 *    microseconds make GPU and CPU results comparable bit for bit).
 *  - Per-layer arrays are row-major [batch][L]; element [i][l-1] belongs to layer
 *    l of instance i, layers numbered 1..L in forward order (Sec. III-A).
 *  - Unless stated otherwise, array pointers are DEVICE pointers owned by the
 *    caller, 8-byte aligned for int64 and 4-byte aligned for 32-bit arrays. The
 *    library keeps no pointer after a call returns and allocates no memory: the
 *    scratch the solver needs comes from the caller's workspace.
 *  - Calls are asynchronous on `stream` (0 = the legacy default stream). Errors
 *    the host can see (null pointers, bad sizes, short workspace, bad config)
 *    return synchronously and launch nothing. batch == 0 returns DC_OK and does
 *    nothing. DC_ERR_CUDA reports a launch error from the CUDA runtime.
 *  - Data-dependent faults are per instance and never stop the batch: an
 *    instance with a negative cost or latency gets status DC_ERR_NEGATIVE, one
 *    whose bound L*dt + sum(xfer) + sum(comp) is >= 2^52 gets DC_ERR_RANGE; its
 *    makespan is written as -(status), its nseg as 0 and its bits as 0.
 *  - Decision bits: W = ceil((L-1)/32) uint32 words per instance (W = 0 when
 *    L = 1). Bit (l-1)%32 of word (l-1)/32 is p_l for the forward direction (a
 *    new pull starts at layer l+1) and g_l for the backward direction (the last
 *    l layers are pushed apart from layer L-l), Sec. III-B.
 */
#ifndef DYNACOMM_H
#define DYNACOMM_H

#include <stddef.h>
#include <stdint.h>

#include <cuda_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum dc_status {
    DC_OK = 0,
    DC_ERR_NULL = 1,       /* a required pointer is NULL */
    DC_ERR_BAD_SHAPE = 2,  /* batch < 0, L < 1, L > DC_L_MAX, or dir not 0/1 */
    DC_ERR_NEGATIVE = 3,   /* per instance: a negative cost or latency */
    DC_ERR_RANGE = 4,      /* per instance: L*dt + sum(xfer) + sum(comp) >= 2^52 */
    DC_ERR_WORKSPACE = 5,  /* workspace NULL or smaller than the query returned */
    DC_ERR_CUDA = 6,       /* the CUDA runtime reported an error for a launch */
    DC_ERR_BAD_CONFIG = 7, /* a profile-generator config field is out of range */
    DC_ERR_INTERNAL = 8,   /* per instance: solver self-check failed (a bug) */
    DC_ERR_BAD_LAYER = 9   /* a layer operator's size, stride, type or option is out of range */
} dc_status;

#define DC_L_MAX 4096

/* ------------------------------------------------------------------------
 * dc_profile_gen -- seeded synthetic profiles (stand-in for the real-time
 * profiler of Sec. IV-A, which reads pt, fc, bc, gt and dt off a framework
 * profiler; no profiler or real training exists here).
 *
 * For instance i (global index g = cfg->inst0 + i) and layer l (0-based):
 *   draw(field, l) = SplitMix64 output number ctr+1 for state cfg->seed, with
 *                    ctr = g<<20 | field<<12 | l (field: 0 rate, 1 bandwidth,
 *                    2 latency, 3 params, 4 FLOPs)
 *   uniform-int [a,b]  = a + floor(r * (b-a+1) / 2^64)
 *   log-uniform [a,b]  = knots T(j) = llround(a * exp((j/512) * ln(b/a))),
 *                        T(0) = a, T(512) = b, evaluated in IEEE double;
 *                        j = r>>55, f = (r>>23) & 0xffffffff,
 *                        value = T(j) + floor((T(j+1)-T(j)) * f / 2^32)
 *   rate (FLOP/us), bw (kbit/s), dt (us, uniform-int) per instance;
 *   params, FLOPs per layer: fixed tables or per-instance draws;
 *   fc = ceil(FLOPs/rate), bc = ceil(bwd_flops_mult*FLOPs/rate),
 *   pt = gt = ceil(bits_per_param*1000*params/bw).
 * Outputs fc, pt, bc, gt: [batch][L] int64; dt: [batch] int64 (device).
 * fixed_params / fixed_flops are HOST pointers of L entries, read during the
 * call only. Limits (else DC_ERR_BAD_CONFIG): 1 <= L <= DC_L_MAX (<= 1024 with
 * fixed tables); inst0 >= 0, inst0 + batch <= 2^44; 1 <= rate_lo <= rate_hi <
 * 2^31 and the same for bw; 0 <= dt_lo <= dt_hi <= 2^40; params and FLOPs
 * (drawn ranges or fixed entries) in [0, 2^40], lo >= 1 for log-uniform draws;
 * 1 <= bwd_flops_mult <= 16; 1 <= bits_per_param <= 64.
 * ---------------------------------------------------------------------- */
#define DC_LAYERS_FIXED 0
#define DC_LAYERS_UNIFORM 1
#define DC_LAYERS_LOGUNIFORM 2
#define DC_DIST_UNIFORM 0
#define DC_DIST_LOGUNIFORM 1

typedef struct dc_profile_cfg {
    int32_t L;
    int32_t layer_mode; /* DC_LAYERS_* */
    int64_t batch;
    int64_t inst0;
    uint64_t seed;
    const int64_t *fixed_params; /* host, L entries, DC_LAYERS_FIXED only */
    const int64_t *fixed_flops;  /* host, L entries, DC_LAYERS_FIXED only */
    int64_t params_lo, params_hi, flops_lo, flops_hi;
    int32_t rate_dist, bw_dist; /* DC_DIST_* */
    int64_t rate_lo, rate_hi;   /* FLOP per microsecond */
    int64_t bw_lo, bw_hi;       /* kbit per second */
    int64_t dt_lo, dt_hi;       /* per-transmission overhead, microseconds */
    int32_t bwd_flops_mult;
    int32_t bits_per_param;
} dc_profile_cfg;

dc_status dc_profile_gen(const dc_profile_cfg *cfg, int64_t *fc, int64_t *pt, int64_t *bc,
                         int64_t *gt, int64_t *dt, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_schedule_workspace_bytes -- device scratch a schedule call needs for
 * (batch, L): a work list for instances that the first pass leaves to a
 * second (values that its kept columns cannot hold in 32 bits, or an optimum
 * with more segments than it keeps columns for); from L = 17 on the kept columns
 * of its resident threads, warps or CTAs, and for L > 192 their flags and the
 * per-launch counters; for L > 64, per-CTA tables of the second pass. Pure host
 * function, no CUDA call.
 * ---------------------------------------------------------------------- */
size_t dc_schedule_workspace_bytes(int64_t batch, int32_t L);

/* ------------------------------------------------------------------------
 * dc_schedule_kernel_launches -- how many kernels one dc_schedule_forward_batch
 * or dc_schedule_backward_batch call with (batch, L) launches: a first pass and
 * a second pass over its work list, or a single pass for small batches of L <= 64
 * (some ten thousand instances); for L > 256 the first pass is split into
 * launches of four resident waves each, chained
 * so that each may start while the one before drains. For counting only (the
 * calls need no caller action per launch). Returns 0 for batch <= 0 or L out of
 * range. Pure host function, no CUDA call.
 * ---------------------------------------------------------------------- */
int32_t dc_schedule_kernel_launches(int64_t batch, int32_t L);

/* ------------------------------------------------------------------------
 * dc_schedule_forward_batch -- Algorithm 3 / Eq. 8 for every instance:
 *   F[m][n] = min_{k} max(F[k][n-1], n*dt + sum_{l<=m} pt_l) + sum_{k<l<=m} fc_l
 * with F[0][0] = 0, then T = min_n F[L][n] (lowest n on ties), then the
 * traceback of Algorithm 3, in which every Path[m][n] is the LOWEST k that
 * attains F[m][n]. Inputs fc, pt: [batch][L]; dt: [batch]. Outputs: makespan
 * [batch] (= T), bits [batch][W] (p_1..p_{L-1}), nseg [batch] (number of
 * pulls, nullable), status [batch] (nullable). The results equal those of
 * Algorithm 3 run in exact integer arithmetic, bit for bit.
 * workspace: device, >= dc_schedule_workspace_bytes(batch, L) bytes, used
 * during the call's kernels only (reuse it after the stream passes them).
 * ---------------------------------------------------------------------- */
dc_status dc_schedule_forward_batch(int64_t batch, int32_t L, const int64_t *fc,
                                    const int64_t *pt, const int64_t *dt, int64_t *makespan,
                                    uint32_t *bits, int32_t *nseg, int32_t *status,
                                    void *workspace, size_t workspace_bytes,
                                    cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_schedule_backward_batch -- Algorithm 4 / Eq. 9 for every instance, with m
 * counting the LAST m layers:
 *   B[m][n] = min_k max(B[k][n-1], sum_{L-m<l<=L} bc_l) + dt + sum_{L-m<l<=L-k} gt_l
 * Inputs bc, gt: [batch][L] in forward layer order; outputs as for the
 * forward call with g_1..g_{L-1} in bits. Same workspace rule.
 * ---------------------------------------------------------------------- */
dc_status dc_schedule_backward_batch(int64_t batch, int32_t L, const int64_t *bc,
                                     const int64_t *gt, const int64_t *dt, int64_t *makespan,
                                     uint32_t *bits, int32_t *nseg, int32_t *status,
                                     void *workspace, size_t workspace_bytes,
                                     cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_schedule_generated_batch -- dc_profile_gen followed by both
 * dc_schedule_forward_batch and dc_schedule_backward_batch for 1 <= L <= 16,
 * fused: every instance's profile is drawn inside the solving kernel (the same
 * pure function of seed, instance, field and layer that dc_profile_gen writes
 * out) and never stored, so the profiles make no round trip through device
 * memory. The results are those of the unfused calls on dc_profile_gen's output,
 * bit for bit. Outputs, forward first then backward: makespan [2][batch],
 * bits [2][batch][W], nseg [2][batch] and status [2][batch] (both nullable).
 * workspace: device, >= dc_schedule_generated_workspace_bytes(batch, L) bytes
 * (the two work lists and a copy of the generator's tables). Errors: those of
 * dc_profile_gen (config), DC_ERR_BAD_SHAPE for L > 16, DC_ERR_NULL,
 * DC_ERR_WORKSPACE, DC_ERR_CUDA. There is no counterpart in the paper, whose
 * profiler produces the profiles (Sec. IV-A).
 * ---------------------------------------------------------------------- */
size_t dc_schedule_generated_workspace_bytes(int64_t batch, int32_t L);
dc_status dc_schedule_generated_batch(const dc_profile_cfg *cfg, int64_t *makespan, uint32_t *bits,
                                      int32_t *nseg, int32_t *status, void *workspace,
                                      size_t workspace_bytes, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_step_batch -- a whole step for 1 <= L <= 16 in one pass over the batch:
 * dc_schedule_generated_batch that also writes the profiles it draws (fc, pt, bc,
 * gt [batch][L], dt [batch], as dc_profile_gen) and f_m of each decision (replay
 * [2][batch], as dc_eval_timeline_batch). The results are those of the separate
 * calls, bit for bit. Workspace and errors as for dc_schedule_generated_batch; the
 * profile arrays and replay must not be NULL.
 * ---------------------------------------------------------------------- */
dc_status dc_step_batch(const dc_profile_cfg *cfg, int64_t *fc, int64_t *pt, int64_t *bc,
                        int64_t *gt, int64_t *dt, int64_t *makespan, uint32_t *bits, int32_t *nseg,
                        int32_t *status, int64_t *replay, void *workspace, size_t workspace_bytes,
                        cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_step_kernel_launches -- how many kernels one dc_step_batch or
 * dc_schedule_generated_batch call launches: one for a small batch, otherwise a
 * copy of the generator's tables, the pass over the batch and a list pass per
 * direction. For counting only. Returns 0 for batch <= 0 or L outside [1, 16]. Pure
 * host function, no CUDA call.
 * ---------------------------------------------------------------------- */
int32_t dc_step_kernel_launches(int64_t batch, int32_t L, int32_t layer_mode);

/* ------------------------------------------------------------------------
 * dc_greedy_forward_batch, dc_greedy_backward_batch -- the paper's competing
 * schedulers (Sec. II-C), for comparison with the DP: greedy parameter
 * scheduling of iBatch (Algorithm 1, forward; inputs as
 * dc_schedule_forward_batch) and greedy gradient scheduling of iPart
 * (Algorithm 2, backward; inputs as dc_schedule_backward_batch). Readings of the
 * listings' open points: ties keep the first candidate of the listing's
 * enumeration; an empty Options set takes the position with the largest slack;
 * Algorithm 1's first pair is the qualifying pair with the largest first-segment
 * compute, then the smallest first transfer, then the smallest slack (with no
 * qualifying pair, the largest slack); Algorithm 2 keeps the candidate with the
 * least f_m. Outputs per instance: bits [batch][W] (the decision, same layout
 * as dc_schedule_*) and makespan [batch] (f_m of that decision, as
 * dc_eval_timeline_batch gives it), or -(status) and zero bits for an instance
 * with a negative or out-of-range input (status 3 or 4). No workspace. Errors:
 * DC_ERR_NULL, DC_ERR_BAD_SHAPE (batch < 0 or > 2^32-1, L outside [1, 4096]),
 * DC_ERR_CUDA. Asynchronous on `stream`.
 * ---------------------------------------------------------------------- */
dc_status dc_greedy_forward_batch(int64_t batch, int32_t L, const int64_t *fc, const int64_t *pt,
                                  const int64_t *dt, int64_t *makespan, uint32_t *bits,
                                  cudaStream_t stream);
dc_status dc_greedy_backward_batch(int64_t batch, int32_t L, const int64_t *bc, const int64_t *gt,
                                   const int64_t *dt, int64_t *makespan, uint32_t *bits,
                                   cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_eval_timeline_batch -- the cost measurement f_m of Sec. III-B for one
 * direction: replays ANY decision (bits [batch][W]) under the partial orders of
 * Eq. 1-7 and writes its makespan. dir 0: comp = fc, xfer = pt, the pulls run
 * back to back on the link and layer l computes once its pull has arrived and
 * layer l-1 is done. dir 1: comp = bc, xfer = gt, the backward compute runs
 * from layer L down without waiting and a push starts once its layers are
 * computed and the previous push is done. Every transmission costs dt + the
 * sum of its layers' transfer costs. A failed instance gets -(status) as its
 * makespan (no status array here).
 * ---------------------------------------------------------------------- */
dc_status dc_eval_timeline_batch(int64_t batch, int32_t L, int32_t dir, const int64_t *comp,
                                 const int64_t *xfer, const int64_t *dt, const uint32_t *bits,
                                 int64_t *makespan, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_schedule_replay_batch -- dc_schedule_forward_batch (dir 0) or
 * dc_schedule_backward_batch (dir 1) and, for each instance, the cost measurement
 * f_m of the decision it writes, evaluated while the instance's prefix sums are on
 * chip: replay [batch] holds what dc_eval_timeline_batch gives for the same rows
 * and bits (-(status) for a failed instance). comp, xfer: fc, pt or bc, gt; the
 * other arguments, the workspace and the errors as for the schedule calls (replay
 * NULL: DC_ERR_NULL; dir not 0/1: DC_ERR_BAD_SHAPE). A dc_time_next_pass request
 * is used up here too.
 * ---------------------------------------------------------------------- */
dc_status dc_schedule_replay_batch(int32_t dir, int64_t batch, int32_t L, const int64_t *comp,
                                   const int64_t *xfer, const int64_t *dt, int64_t *makespan,
                                   uint32_t *bits, int32_t *nseg, int32_t *status,
                                   int64_t *replay, void *workspace, size_t workspace_bytes,
                                   cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_schedule_batch_static -- the paper has no counterpart: this is a
 * deployment variant of the two schedule calls above for callers that cannot
 * allocate device memory where they schedule (a scheduler embedded in a
 * training runtime whose allocator owns all device memory and refuses other
 * allocations once training runs, or one that schedules inside the idle window
 * between a gradient push and the next pull, where a cudaMalloc that can
 * synchronise the device is not acceptable). It takes no workspace.
 *
 * dir 0 is the forward call's problem (comp = fc, xfer = pt), dir 1 the
 * backward call's (comp = bc, xfer = gt); inputs, outputs and per-instance
 * status are exactly those of dc_schedule_forward_batch /
 * dc_schedule_backward_batch, including a NULL status (a failed instance's
 * makespan then carries -status).
 * Limits: 1 <= L <= 16 (else DC_ERR_BAD_SHAPE); batch <= 1,048,576
 * (DC_STATIC_MAX_BATCH; a larger batch returns DC_ERR_WORKSPACE, launching
 * nothing).
 * Scratch: a 4 MiB + 256 B array in the library's device memory, held by every
 * GPU that loads the library until the process exits, shared by all calls on a
 * device: calls that overlap on one GPU race on it, so serialise them (one
 * stream, or an event between them). Each call clears what must start at zero.
 * Every call looks up the array's device address on the current device
 * (cudaGetSymbolAddress, which allocates nothing); on a device's first call
 * that lookup also loads the library's device code there if needed, so make
 * the first call on each device before any stream capture. No cudaMalloc,
 * cudaFree or other allocating call is made.
 * ---------------------------------------------------------------------- */
#define DC_STATIC_MAX_BATCH 1048576
dc_status dc_schedule_batch_static(int32_t dir, int64_t batch, int32_t L, const int64_t *comp,
                                   const int64_t *xfer, const int64_t *dt, int64_t *makespan,
                                   uint32_t *bits, int32_t *nseg, int32_t *status,
                                   cudaStream_t stream);

/* ------------------------------------------------------------------------
 * Layer operators -- the training block of a mixture of experts, forward and
 * backward. The costs fc and bc of Sec. IV-A are a profiler's times of a model's
 * layers; these are layers of large language models that run on this GPU, so that such
 * a model's costs can be measured here and scheduled. No counterpart in the paper.
 *
 * Conventions: device pointers, asynchronous on `stream`, no allocation, errors as
 * above. Elements are bfloat16, IEEE half or float (DC_BF16, DC_FP16, DC_FP32) and
 * aligned to their size; rows are contiguous, and a stride (ld...) is the distance of
 * two rows in elements. Sums, statistics and gradients of parameters are held in 32-bit
 * floats, and each output is rounded once. Outputs must not overlap inputs unless a
 * call says so. No sum's order depends on timing: equal calls give equal bits.
 * ---------------------------------------------------------------------- */
#define DC_BF16 0
#define DC_FP16 1
#define DC_FP32 2
#define DC_EXPERTS_MAX 1024
#define DC_LAYER_DIM_MAX 1048576 /* N, K and the columns of dropout and gated units */
#define DC_NORM_DIM_MAX 16384    /* D of the block norms: a row stays in registers */

/* ------------------------------------------------------------------------
 * dc_expert_matmul, dc_expert_matmul_grad_input, dc_expert_matmul_grad_weight --
 * matrix products grouped by expert. Row r of x [rows][K] belongs to expert e when
 * offsets[e] <= r < offsets[e+1] (offsets: experts + 1 device int64, in order):
 *   y[r]  = W_e x[r]                  (y [rows][N], W_e [N][K])
 *   dx[r] = W_e^T dy[r]
 *   dW_e  = sum over e's rows of dy[r] x[r]^T
 * Rows of no expert (before offsets[0] or from offsets[experts] on) get zeros in y and
 * dx and count in no dW; an expert of no rows gets dW_e = 0. An offset outside [0, rows],
 * or below an earlier one, counts as the nearest valid value. w and dw have the strides
 * w_expert, w_n, w_k (elements); one of w_n and w_k is 1.
 * 16-bit operands run on the tensor cores; those whose rows start off 16-byte boundaries
 * are first copied into the workspace, row by row, so that they start on them. Floats go
 * there in two parts of 11 significant bits, whose products are summed as floats (small
 * products of floats run on the CUDA cores): 1.35e-7 off in the root mean square for 64 summed
 * elements and 2.4e-7 for 4,096, where a 32-bit sum of one product after another is 1.5e-7 and 11e-7 off.
 * Digits below 2^-136 are not seen there, so that a float below 2^-137 counts as zero. Infinities and NaN come out as the definition has them. 16-bit products summed over more than 8,192
 * elements are added up from parts of that many, in floats in the workspace. Up to DC_FEW_ROWS rows in all (floats: 16 times
 * as many) take a pass that streams the weights over every SM. workspace: dc_expert_workspace_bytes(shape, product, a,
 * b) bytes, 256-byte aligned, used during the call's kernels only, where product is 0 for
 * y, 1 for dx, 2 for dW and a, b are the call's two operands in its order (their addresses
 * decide whether copies are needed); NULL where that is 0. status (device, nullable): set
 * to DC_ERR_INTERNAL if a kernel gave up a wait (its outputs are then incomplete), else left
 * as it is.
 * Errors: DC_ERR_NULL; DC_ERR_BAD_LAYER (dtype; rows outside [0, 2^31 - 1]; experts
 * outside [1, DC_EXPERTS_MAX]; N or K outside [1, DC_LAYER_DIM_MAX]; a stride shorter than its
 * row, or above 2^37); DC_ERR_WORKSPACE; DC_ERR_CUDA.
 * ---------------------------------------------------------------------- */
#define DC_FEW_ROWS 4
typedef struct dc_expert_shape {
    int32_t dtype; /* of x, y, w and their gradients */
    int32_t experts;
    int64_t rows;
    int32_t N, K;
    int64_t ldx, ldy;           /* rows of x or dx, rows of y or dy */
    int64_t w_expert, w_n, w_k; /* w[e][n][k] or dw[e][n][k] */
} dc_expert_shape;

size_t dc_expert_workspace_bytes(const dc_expert_shape *shape, int32_t product, const void *a,
                                 const void *b);
dc_status dc_expert_matmul(const dc_expert_shape *shape, const void *x, const void *w,
                           const int64_t *offsets, void *y, int32_t *status, void *workspace,
                           size_t workspace_bytes, cudaStream_t stream);
dc_status dc_expert_matmul_grad_input(const dc_expert_shape *shape, const void *dy, const void *w,
                                      const int64_t *offsets, void *dx, int32_t *status,
                                      void *workspace, size_t workspace_bytes,
                                      cudaStream_t stream);
dc_status dc_expert_matmul_grad_weight(const dc_expert_shape *shape, const void *dy, const void *x,
                                       const int64_t *offsets, void *dw, int32_t *status,
                                       void *workspace, size_t workspace_bytes,
                                       cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_gated_unit, dc_gated_unit_grad -- a[r][c] = act(h[r][c]) * h[r][F + c] for
 * h [rows][2F], and from da [rows][F] the gradient dh [rows][2F] (act is evaluated again,
 * nothing is kept). act: DC_ACT_SILU x / (1 + e^-x) or DC_ACT_GELU x Phi(x).
 * Errors: DC_ERR_NULL, DC_ERR_BAD_LAYER, DC_ERR_CUDA.
 * ---------------------------------------------------------------------- */
#define DC_ACT_SILU 0
#define DC_ACT_GELU 1
dc_status dc_gated_unit(int32_t dtype, int32_t act, int64_t rows, int32_t F, const void *h,
                        int64_t ldh, void *a, int64_t lda, cudaStream_t stream);
dc_status dc_gated_unit_grad(int32_t dtype, int32_t act, int64_t rows, int32_t F, const void *da,
                             int64_t ldda, const void *h, int64_t ldh, void *dh, int64_t lddh,
                             cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_dropout -- y = keep ? x / (1 - q) : 0, plus residual if not NULL, with a mask that
 * is never stored: it is a function of (seed, offset, row, column), so that the same call
 * on a gradient (without residual) is the backward pass. Column c of row r is kept when
 * 16-bit field c % 4 (the lowest first) of SplitMix64 output number
 *   offset + r * ceil(cols / 4) + c / 4 + 1      (state seed, as dc_profile_gen's draws)
 * is at least t = floor(65536 p + 0.5), and q = t / 65536 is the probability in effect, so the
 * mean is exact. p = 1 drops everything; dropped elements give 0 (or the residual)
 * whatever they held. A call uses rows * ceil(cols / 4) draws: add that to offset for the
 * next one. y may be x or residual themselves. Errors: DC_ERR_NULL,
 * DC_ERR_BAD_LAYER (p outside [0, 1] or NaN, offset < 0, a size or stride), DC_ERR_CUDA.
 * ---------------------------------------------------------------------- */
dc_status dc_dropout(int32_t dtype, int64_t rows, int32_t cols, const void *x, int64_t ldx,
                     const void *residual, int64_t ldr, void *y, int64_t ldy, double p,
                     uint64_t seed, int64_t offset, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_block_norm, dc_block_norm_grad -- the end of one block and the start of the next in
 * one pass over the rows:
 *   y = residual_scale * x + gate * drop(w_post * n(f))
 *   h = w_pre * n(y)                                 (of y before it is rounded)
 * n(v) = v / sqrt(mean(v^2) + eps) (DC_NORM_RMS) or the same of v - mean(v)
 * (DC_NORM_LAYER); f is the block's output, drop the dropout of dc_dropout over
 * [rows][D]. gate [ceil(rows / rows_per_gate)][D]: row r takes gate row
 * r / rows_per_gate (1: one a token; >= rows: one for all). Every array is contiguous.
 * Forms: with f NULL the call is the first norm alone (h = w_pre * n(x); y, gate and
 * w_post not used); with h NULL it ends at y. gate, w_post and w_pre may be NULL (ones).
 * The gradient takes dy and dh (the gradients of y and h; dy NULL: zero; dh NULL: no h), the
 * saved y (x itself where f is NULL) and f, and writes
 *   t = dy + n'(y)^T (dh * w_pre),  dx = residual_scale * t (t where f is NULL),  df,
 *   dgate (of gate's type), dw_post and dw_pre (float, [D]); statistics are computed again.
 * dgate, dw_post, dw_pre may be NULL (not wanted). workspace:
 * dc_block_norm_grad_workspace_bytes(cfg) bytes, used during the call's kernels only.
 * Errors: DC_ERR_NULL, DC_ERR_BAD_LAYER (dtype, kind, rows < 0 or > 2^31 - 1, D outside
 * [1, DC_NORM_DIM_MAX], rows_per_gate < 1, eps < 0, p, offset), DC_ERR_WORKSPACE, DC_ERR_CUDA.
 * ---------------------------------------------------------------------- */
#define DC_NORM_RMS 0
#define DC_NORM_LAYER 1
typedef struct dc_block_norm_cfg {
    int32_t dtype, kind;
    int64_t rows;
    int32_t D;
    int64_t rows_per_gate;
    double residual_scale, eps, p;
    uint64_t seed;
    int64_t offset;
} dc_block_norm_cfg;

dc_status dc_block_norm(const dc_block_norm_cfg *cfg, const void *x, const void *f,
                        const void *gate, const void *w_post, const void *w_pre, void *y, void *h,
                        cudaStream_t stream);
size_t dc_block_norm_grad_workspace_bytes(const dc_block_norm_cfg *cfg);
dc_status dc_block_norm_grad(const dc_block_norm_cfg *cfg, const void *dy, const void *dh,
                             const void *y, const void *f, const void *gate, const void *w_post,
                             const void *w_pre, void *dx, void *df, void *dgate, float *dw_post,
                             float *dw_pre, void *workspace, size_t workspace_bytes,
                             cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_head_norm_rotary, dc_head_norm_rotary_grad -- the norms of queries and keys for each
 * head and the rotation by position, in one pass over both. q [tokens][heads][D] and k
 * [tokens][kv_heads][D] have contiguous heads and the strides q_token, q_head, k_token,
 * k_head (elements); q_out and k_out are contiguous. For a head's elements x, with w its
 * weight w_q or w_k [D] (NULL: ones):
 *   z = w x / sqrt(mean(x^2) + eps)           (norm 0: z = w x)
 * and pair i of the first `rotary` elements, (i, i + rotary / 2), or (2i, 2i + 1) where
 * interleaved is not 0, turns by the angle a = positions[token] base^(-2i / rotary):
 *   out1 = z1 cos a - z2 sin a,  out2 = z2 cos a + z1 sin a
 * The other elements are z. Positions (device, int64) may have any value; the angle's whole
 * turns are dropped in integers, from frequencies of 128 bits, so that far positions lose nothing.
 * The gradient takes dq_out and dk_out (contiguous) and q and k again, and writes dq, dk
 * (contiguous) and dw_q, dw_k (float [D]; NULL: not wanted). workspace:
 * dc_head_norm_rotary_grad_workspace_bytes(cfg) bytes, used during the call's kernels only.
 * Outputs may be their own inputs (q_out = q of contiguous q; dq = dq_out).
 * Errors: DC_ERR_NULL, DC_ERR_BAD_LAYER (dtype; tokens outside [0, 2^31 - 1]; heads or kv_heads
 * outside [1, DC_HEADS_MAX]; D outside [1, DC_HEAD_NORM_DIM_MAX]; rotary odd, negative or above D;
 * base outside [DC_ROTARY_BASE_MIN, DC_ROTARY_BASE_MAX]; eps < 0 or not finite; heads that overlap),
 * DC_ERR_WORKSPACE, DC_ERR_CUDA.
 * ---------------------------------------------------------------------- */
#define DC_HEADS_MAX 1024
#define DC_HEAD_NORM_DIM_MAX 256
#define DC_ROTARY_BASE_MIN 1e-3
#define DC_ROTARY_BASE_MAX 1e30
typedef struct dc_head_norm_cfg {
    int32_t dtype, heads, kv_heads, D, rotary, interleaved, norm;
    int64_t tokens;
    int64_t q_token, q_head, k_token, k_head;
    double base, eps;
} dc_head_norm_cfg;

dc_status dc_head_norm_rotary(const dc_head_norm_cfg *cfg, const void *q, const void *k,
                              const int64_t *positions, const void *w_q, const void *w_k,
                              void *q_out, void *k_out, cudaStream_t stream);
size_t dc_head_norm_rotary_grad_workspace_bytes(const dc_head_norm_cfg *cfg);
dc_status dc_head_norm_rotary_grad(const dc_head_norm_cfg *cfg, const void *dq_out,
                                   const void *dk_out, const void *q, const void *k,
                                   const int64_t *positions, const void *w_q, const void *w_k,
                                   void *dq, void *dk, float *dw_q, float *dw_k, void *workspace,
                                   size_t workspace_bytes, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_attention, dc_attention_grad -- causal attention of packed sequences. Row t of q
 * [tokens][heads][D] belongs to sequence s when offsets[s] <= t < offsets[s+1] (offsets:
 * sequences + 1 device int64, in order); head h reads key head h / (heads / kv_heads) of k
 * and v [tokens][kv_heads][D]. Over the keys j of the same sequence with j <= i:
 *   S_ij = scale q_i . k_j,  lse_i = log(sum_j e^S_ij),  y_i = sum_j e^(S_ij - lse_i) v_j
 * with y [tokens][heads][D] and lse (float) [heads][tokens] contiguous. The gradient takes dy
 * (of y; contiguous), the call's inputs, y and lse, and writes dq, dk, dv (contiguous):
 *   P = e^(S - lse),  dS_ij = P_ij (dy_i . v_j - dy_i . y_i),
 *   dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij dy_i
 * with the sums of dk and dv over every head that reads the key head. 16-bit types run on the tensor
 * cores: P and dS are rounded to the type for their products (each at most half a step of a term; halves
 * in powers of two: dS one of each row's for dq and of each key's for dk, from what that row or key sees, so that small
 * gradients keep their digits beside large ones; a term of P loses no more than 2^-32 of its row's largest forward,
 * 2^-39 backward), everything else is in floats,
 * and what y's own rounding does to dy_i . y_i is taken back, since a row of dS sums to zero. Sums on the
 * tensor cores are cut off toward zero where floats would round: by some 2^-24 of their terms' magnitudes for
 * every 16 terms (6e-5 for 16,384 terms of one sign). Floats run on the CUDA cores. What stands in rows of
 * other sequences, or of keys after a row, has no effect on it, infinities and NaN included.
 * Rows of no sequence (before offsets[0] or from offsets[sequences] on) get zeros in y, lse,
 * dq, dk and dv. An offset outside [0, tokens], or below an earlier one, counts as the nearest
 * valid value. q, k and v have contiguous heads and the strides given (elements).
 * workspace: dc_attention_workspace_bytes(shape, grad, q, k, v, dy) bytes, 256-byte aligned, used
 * during the call's kernels only (grad 0 or 1; the addresses decide whether copies are
 * needed; dy of no account for grad 0). status (device, nullable): as for the expert products.
 * Errors: DC_ERR_NULL; DC_ERR_BAD_LAYER (dtype; tokens outside [0, DC_ATTENTION_TOKENS_MAX]; sequences outside
 * [0, DC_SEQUENCES_MAX]; heads or kv_heads outside [1, DC_HEADS_MAX]; heads not a multiple of
 * kv_heads; (tokens / 64 + 1) heads / kv_heads above 2^31 - 1; D outside [1, DC_ATTENTION_DIM_MAX]; a scale that is
 * not finite (twice it, as a float); heads that overlap, or strides above 2^37); DC_ERR_WORKSPACE; DC_ERR_CUDA.
 * ---------------------------------------------------------------------- */
#define DC_ATTENTION_DIM_MAX 128
#define DC_SEQUENCES_MAX 1048576
#define DC_ATTENTION_TOKENS_MAX 2147482624 /* 2^31 - 1024 */
typedef struct dc_attention_shape {
    int32_t dtype, heads, kv_heads, D, sequences;
    int64_t tokens;
    int64_t q_token, q_head, k_token, k_head, v_token, v_head;
    double scale;
} dc_attention_shape;

size_t dc_attention_workspace_bytes(const dc_attention_shape *shape, int32_t grad, const void *q,
                                    const void *k, const void *v, const void *dy);
dc_status dc_attention(const dc_attention_shape *shape, const void *q, const void *k,
                       const void *v, const int64_t *offsets, void *y, float *lse,
                       int32_t *status, void *workspace, size_t workspace_bytes,
                       cudaStream_t stream);
dc_status dc_attention_grad(const dc_attention_shape *shape, const void *dy, const void *q,
                            const void *k, const void *v, const void *y, const float *lse,
                            const int64_t *offsets, void *dq, void *dk, void *dv, int32_t *status,
                            void *workspace, size_t workspace_bytes, cudaStream_t stream);

/* Static description of a status code. Never NULL. */
const char *dc_status_string(dc_status s);

/* ------------------------------------------------------------------------
 * dc_time_next_pass -- measurement support, not part of the method. The next
 * dc_schedule_forward_batch, dc_schedule_backward_batch or
 * dc_schedule_batch_static call made by the calling thread records `start` on
 * its stream right before it launches its first pass over the batch (the
 * dense, looped, warp- or CTA-per-instance kernel, all of its launches) and `stop`
 * right after them, before its work-list pass; cudaEventElapsedTime(start,
 * stop) is then that pass's time on the GPU. start, stop: events created by
 * the caller on the current device, both non-NULL (DC_ERR_NULL if only one
 * is); both NULL withdraw a pending request. The request belongs to the
 * calling thread and is used up by its next schedule call, whether that call
 * succeeds or not; no other call consumes it. This is the one state the
 * library keeps between calls.
 * ---------------------------------------------------------------------- */
dc_status dc_time_next_pass(cudaEvent_t start, cudaEvent_t stop);

/* ------------------------------------------------------------------------
 * dc_roof_int_probe -- measurement support, not part of the method: a
 * register-only loop of the DP's per-transition integer operations on
 * `blocks` x `threads` threads, `iters` iterations of 8 transitions each.
 * Variant 0: the 32-bit passes' shifted form (one 32-bit add-then-max per
 * candidate, one 3-input min per two candidates); variant 1: the 64-bit
 * passes' max, subtract, min. Time it with events on `stream`; it performs
 * blocks*threads*iters*8 transitions. sink: device, blocks*threads uint32.
 * ---------------------------------------------------------------------- */
dc_status dc_roof_int_probe(int32_t variant, int32_t blocks, int32_t threads, int64_t iters,
                            uint32_t *sink, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_wait_probe -- test support: one small block in which four threads wait, as the layer
 * operators' kernels do, for copies that nothing has started. The waits run out within some
 * two seconds, and the kernel ends and sets status (device) to DC_ERR_INTERNAL as theirs do.
 * ---------------------------------------------------------------------- */
dc_status dc_wait_probe(int32_t *status, cudaStream_t stream);

/* ------------------------------------------------------------------------
 * dc_head_parts_probe -- test support, on the host alone: how the head norms deal a token's heads
 * to groups of lanes where tokens are few. Part i of `parts` has the heads from i * per_part on, per_part
 * of them or, the last part, what is left; `wanted` units of work fill the GPU, and a part
 * other than the last has `least` heads or more where there are as many.
 * ---------------------------------------------------------------------- */
void dc_head_parts_probe(int64_t tokens, int32_t heads, int64_t wanted, int32_t least, int32_t *parts,
                         int32_t *per_part);

#ifdef __cplusplus
}
#endif
#endif /* DYNACOMM_H */
