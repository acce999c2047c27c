// The block norms' kernels for bfloat16 rows, and the choice of the type (one type per translation unit, so that
// they compile side by side).
#include "layer_norms.cuh"

namespace dc {

size_t norm_grad_workspace(int dtype, int64_t rows, int D)
{
    const int64_t a = norms::grad_runs(dtype, rows, D, true), b = norms::grad_runs(dtype, rows, D, false);
    return size_t(a > b ? a : b) * norms::kSlots * size_t(D) * sizeof(float);
}

cudaError_t norm_forward_fp16(const NormArgs &a, cudaStream_t stream);
cudaError_t norm_forward_fp32(const NormArgs &a, cudaStream_t stream);
cudaError_t norm_gradient_fp16(const NormArgs &a, float *partial, cudaStream_t stream);
cudaError_t norm_gradient_fp32(const NormArgs &a, float *partial, cudaStream_t stream);

cudaError_t launch_norm(int dtype, const NormArgs &a, cudaStream_t stream)
{
    return dtype == DC_BF16   ? norms::forward<__nv_bfloat16>(dtype, a, stream)
           : dtype == DC_FP16 ? norm_forward_fp16(a, stream)
                              : norm_forward_fp32(a, stream);
}

cudaError_t launch_norm_grad(int dtype, const NormArgs &a, float *partial, cudaStream_t stream)
{
    return dtype == DC_BF16   ? norms::gradient<__nv_bfloat16>(dtype, a, partial, stream)
           : dtype == DC_FP16 ? norm_gradient_fp16(a, partial, stream)
                              : norm_gradient_fp32(a, partial, stream);
}

}  // namespace dc
