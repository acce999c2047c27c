// C ABI of the layer operators (declared in include/dynacomm.h): host-side argument
// checks, then kernel launches on the caller's stream. No allocation, no synchronisation.
#include "blackwell.cuh"
#include "layers.cuh"

namespace dc {

cudaError_t sm_count(int &n)
{
    static DeviceCache cache;
    return cache.get(n, [](int &v) {
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        return e != cudaSuccess ? e
                                : cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev);
    });
}

namespace {

constexpr int64_t kRowsMax = (int64_t(1) << 31) - 1;
constexpr int64_t kStrideMax = int64_t(1) << 37;  // tile copies take strides below 2^40 bytes

bool rows_ok(int64_t rows) { return rows >= 0 && rows <= kRowsMax; }
bool dim_ok(int64_t n) { return n >= 1 && n <= DC_LAYER_DIM_MAX; }
bool stride_ok(int64_t ld, int64_t row) { return ld >= row && ld <= kStrideMax; }

dc_status result(cudaError_t e) { return e == cudaSuccess ? DC_OK : DC_ERR_CUDA; }

dc_status check_experts(const dc_expert_shape *s)
{
    if (!s) return DC_ERR_NULL;
    if (!dtype_ok(s->dtype) || !rows_ok(s->rows) || s->experts < 1 ||
        s->experts > DC_EXPERTS_MAX || !dim_ok(s->N) || !dim_ok(s->K))
        return DC_ERR_BAD_LAYER;
    if (!stride_ok(s->ldx, s->K) || !stride_ok(s->ldy, s->N)) return DC_ERR_BAD_LAYER;
    const bool nk = s->w_k == 1 && stride_ok(s->w_n, s->K);
    const bool kn = s->w_n == 1 && stride_ok(s->w_k, s->N);
    if (!nk && !kn) return DC_ERR_BAD_LAYER;
    const int64_t matrix = (s->N - 1) * s->w_n + (s->K - 1) * s->w_k + 1;
    if (s->experts > 1 && !stride_ok(s->w_expert, matrix)) return DC_ERR_BAD_LAYER;
    return DC_OK;
}

// y, dx or dW (product 0, 1, 2) of operands a and b as one strided product
ExpertArgs expert_args(const dc_expert_shape *s, int product, const void *a, const void *b,
                       const int64_t *offsets, void *c, int32_t *status)
{
    ExpertArgs g = {};
    g.c = c;
    g.offsets = offsets;
    g.rows = s->rows;
    g.experts = s->experts;
    g.status = status;
    if (product < 2) {
        g.a = a;
        g.b = b;
        g.a_r = 1;
        g.b_e = s->w_expert;
        g.a_m = product ? s->ldy : s->ldx;
        g.c_m = product ? s->ldx : s->ldy;
        g.b_n = product ? s->w_k : s->w_n;
        g.b_r = product ? s->w_n : s->w_k;
        g.n = product ? s->K : s->N;
        g.r = product ? s->N : s->K;
    } else {  // dw[e][n][k], or its transpose: the kernels take C with contiguous columns
        const bool nk = s->w_k == 1;
        g.a = nk ? a : b;
        g.b = nk ? b : a;
        g.a_m = g.b_n = 1;
        g.a_r = nk ? s->ldy : s->ldx;
        g.b_r = nk ? s->ldx : s->ldy;
        g.c_e = s->w_expert;
        g.c_m = nk ? s->w_n : s->w_k;
        g.m = nk ? s->N : s->K;
        g.n = nk ? s->K : s->N;
    }
    return g;
}

dc_status expert_product(const dc_expert_shape *s, int product, const void *a, const void *b,
                         const int64_t *offsets, void *c, int32_t *status, void *workspace,
                         size_t workspace_bytes, cudaStream_t stream)
{
    const dc_status st = check_experts(s);
    if (st != DC_OK) return st;
    if (s->rows == 0 && product < 2) return DC_OK;
    if (!offsets || !c || (s->rows > 0 && (!a || !b))) return DC_ERR_NULL;
    const ExpertArgs g = expert_args(s, product, a, b, offsets, c, status);
    const size_t need = s->rows ? expert_workspace(s->dtype, g, product == 2) : 0;
    if (need && (!workspace || workspace_bytes < need)) return DC_ERR_WORKSPACE;
    return result(product < 2 ? launch_expert_rows(s->dtype, g, workspace, stream)
                              : launch_expert_weights(s->dtype, g, workspace, stream));
}

dc_status check_drop(double p, int64_t offset)
{
    return p >= 0.0 && p <= 1.0 && offset >= 0 ? DC_OK : DC_ERR_BAD_LAYER;
}

dc_status check_norm(const dc_block_norm_cfg *c)
{
    if (!c) return DC_ERR_NULL;
    if (!dtype_ok(c->dtype) || (c->kind != DC_NORM_RMS && c->kind != DC_NORM_LAYER) ||
        !rows_ok(c->rows) || c->D < 1 || c->D > DC_NORM_DIM_MAX || c->rows_per_gate < 1 ||
        !(c->eps >= 0.0))
        return DC_ERR_BAD_LAYER;
    return check_drop(c->p, c->offset);
}

NormArgs norm_args(const dc_block_norm_cfg *c)
{
    NormArgs a = {};
    a.rows = c->rows;
    a.rows_per_gate = c->rows_per_gate < c->rows ? c->rows_per_gate : c->rows;
    a.D = c->D;
    a.layer = c->kind == DC_NORM_LAYER;
    a.alpha = float(c->residual_scale);
    a.eps = float(c->eps);
    a.drop = drop_rule(c->p, c->seed, c->offset);
    return a;
}

// Both warps' waits end: the first to run out makes the other give up.
__global__ void wait_probe_kernel(int32_t *status)
{
    __shared__ alignas(8) uint64_t bars[2];
    __shared__ uint32_t gave_up;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) bw::bar_init(bw::smem_addr(&bars[i]), 1);
        gave_up = 0;
        bw::bar_init_fence();
    }
    __syncthreads();
    bool arrived = false;
    if (threadIdx.x % 32 == 0) arrived = bw::bar_wait(bw::smem_addr(&bars[threadIdx.x / 32]), 0, &gave_up);
    const bool any = __syncthreads_or(arrived);
    if (threadIdx.x == 0 && gave_up && !any) *status = DC_ERR_INTERNAL;
}

}  // namespace
}  // namespace dc

extern "C" {

size_t dc_expert_workspace_bytes(const dc_expert_shape *s, int32_t product, const void *a,
                                 const void *b)
{
    if (dc::check_experts(s) != DC_OK || product < 0 || product > 2 || s->rows == 0) return 0;
    return dc::expert_workspace(s->dtype, dc::expert_args(s, product, a, b, nullptr, nullptr, nullptr),
                                product == 2);
}

dc_status dc_expert_matmul(const dc_expert_shape *s, const void *x, const void *w,
                           const int64_t *offsets, void *y, int32_t *status, void *workspace,
                           size_t workspace_bytes, cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_expert_matmul");
    return dc::expert_product(s, 0, x, w, offsets, y, status, workspace, workspace_bytes, stream);
}

dc_status dc_expert_matmul_grad_input(const dc_expert_shape *s, const void *dy, const void *w,
                                      const int64_t *offsets, void *dx, int32_t *status,
                                      void *workspace, size_t workspace_bytes, cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_expert_matmul_grad_input");
    return dc::expert_product(s, 1, dy, w, offsets, dx, status, workspace, workspace_bytes, stream);
}

dc_status dc_expert_matmul_grad_weight(const dc_expert_shape *s, const void *dy, const void *x,
                                       const int64_t *offsets, void *dw, int32_t *status,
                                       void *workspace, size_t workspace_bytes,
                                       cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_expert_matmul_grad_weight");
    return dc::expert_product(s, 2, dy, x, offsets, dw, status, workspace, workspace_bytes, stream);
}

dc_status dc_gated_unit(int32_t dtype, int32_t act, int64_t rows, int32_t F, const void *h,
                        int64_t ldh, void *a, int64_t lda, cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_gated_unit");
    if (!dc::dtype_ok(dtype) || (act != DC_ACT_SILU && act != DC_ACT_GELU) || !dc::rows_ok(rows) ||
        !dc::dim_ok(F) || !dc::stride_ok(ldh, 2 * int64_t(F)) || !dc::stride_ok(lda, F))
        return DC_ERR_BAD_LAYER;
    if (rows == 0) return DC_OK;
    if (!h || !a) return DC_ERR_NULL;
    return dc::result(dc::launch_gated(dtype, act, rows, F, h, ldh, a, lda, stream));
}

dc_status dc_gated_unit_grad(int32_t dtype, int32_t act, int64_t rows, int32_t F, const void *da,
                             int64_t ldda, const void *h, int64_t ldh, void *dh, int64_t lddh,
                             cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_gated_unit_grad");
    if (!dc::dtype_ok(dtype) || (act != DC_ACT_SILU && act != DC_ACT_GELU) || !dc::rows_ok(rows) ||
        !dc::dim_ok(F) || !dc::stride_ok(ldh, 2 * int64_t(F)) || !dc::stride_ok(ldda, F) ||
        !dc::stride_ok(lddh, 2 * int64_t(F)))
        return DC_ERR_BAD_LAYER;
    if (rows == 0) return DC_OK;
    if (!da || !h || !dh) return DC_ERR_NULL;
    return dc::result(
        dc::launch_gated_grad(dtype, act, rows, F, da, ldda, h, ldh, dh, lddh, stream));
}

dc_status dc_dropout(int32_t dtype, int64_t rows, int32_t cols, const void *x, int64_t ldx,
                     const void *residual, int64_t ldr, void *y, int64_t ldy, double p,
                     uint64_t seed, int64_t offset, cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_dropout");
    if (!dc::dtype_ok(dtype) || !dc::rows_ok(rows) || !dc::dim_ok(cols) ||
        !dc::stride_ok(ldx, cols) || !dc::stride_ok(ldy, cols) ||
        (residual && !dc::stride_ok(ldr, cols)))
        return DC_ERR_BAD_LAYER;
    const dc_status st = dc::check_drop(p, offset);
    if (st != DC_OK) return st;
    if (rows == 0) return DC_OK;
    if (!x || !y) return DC_ERR_NULL;
    return dc::result(dc::launch_dropout(dtype, rows, cols, x, ldx, residual, ldr, y, ldy,
                                         dc::drop_rule(p, seed, offset), stream));
}

dc_status dc_block_norm(const dc_block_norm_cfg *cfg, const void *x, const void *f,
                        const void *gate, const void *w_post, const void *w_pre, void *y, void *h,
                        cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_block_norm");
    const dc_status st = dc::check_norm(cfg);
    if (st != DC_OK) return st;
    if (cfg->rows == 0) return DC_OK;
    if (!x || (f && !y) || (!f && !h)) return DC_ERR_NULL;
    dc::NormArgs a = dc::norm_args(cfg);
    a.x = x;
    a.f = f;
    a.gate = f ? gate : nullptr;
    a.w_post = f ? w_post : nullptr;
    a.w_pre = w_pre;
    a.y = f ? y : nullptr;
    a.h = h;
    return dc::result(dc::launch_norm(cfg->dtype, a, stream));
}

size_t dc_block_norm_grad_workspace_bytes(const dc_block_norm_cfg *cfg)
{
    if (dc::check_norm(cfg) != DC_OK || cfg->rows == 0) return 0;
    return dc::norm_grad_workspace(cfg->dtype, cfg->rows, cfg->D);
}

dc_status dc_block_norm_grad(const dc_block_norm_cfg *cfg, const void *dy, const void *dh,
                             const void *y, const void *f, const void *gate, const void *w_post,
                             const void *w_pre, void *dx, void *df, void *dgate, float *dw_post,
                             float *dw_pre, void *workspace, size_t workspace_bytes,
                             cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_block_norm_grad");
    const dc_status st = dc::check_norm(cfg);
    if (st != DC_OK) return st;
    if (cfg->rows == 0) {  // sums over no rows; there are no gate rows
        cudaError_t e = cudaSuccess;
        if (dw_post) e = cudaMemsetAsync(dw_post, 0, sizeof(float) * cfg->D, stream);
        if (dw_pre && e == cudaSuccess)
            e = cudaMemsetAsync(dw_pre, 0, sizeof(float) * cfg->D, stream);
        return dc::result(e);
    }
    if (!y || !dx || (!dy && !dh) || (!f && !dh) || (f && !df)) return DC_ERR_NULL;
    if (!workspace ||
        workspace_bytes < dc::norm_grad_workspace(cfg->dtype, cfg->rows, cfg->D))
        return DC_ERR_WORKSPACE;
    dc::NormArgs a = dc::norm_args(cfg);
    a.x = y;
    a.f = f;
    a.gate = f ? gate : nullptr;
    a.w_post = f ? w_post : nullptr;
    a.w_pre = w_pre;
    a.dy = dy;
    a.dh = dh;
    a.dx = dx;
    a.df = f ? df : nullptr;
    a.dgate = f ? dgate : nullptr;
    a.dw_post = f ? dw_post : nullptr;
    a.dw_pre = dh ? dw_pre : nullptr;
    if (!f) a.alpha = 1.0f;
    return dc::result(
        dc::launch_norm_grad(cfg->dtype, a, static_cast<float *>(workspace), stream));
}

dc_status dc_wait_probe(int32_t *status, cudaStream_t stream)
{
    const dc::NvtxRange nvtx("dc_wait_probe");
    if (!status) return DC_ERR_NULL;
    dc::wait_probe_kernel<<<1, 64, 0, stream>>>(status);
    return dc::result(cudaGetLastError());
}

}  // extern "C"
