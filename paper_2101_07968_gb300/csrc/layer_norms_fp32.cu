// The block norms' kernels for float rows (one type per translation unit, so that
// they compile side by side).
#include "layer_norms.cuh"

namespace dc {

cudaError_t norm_forward_fp32(const NormArgs &a, cudaStream_t stream)
{
    return norms::forward<float>(DC_FP32, a, stream);
}

cudaError_t norm_gradient_fp32(const NormArgs &a, float *partial, cudaStream_t stream)
{
    return norms::gradient<float>(DC_FP32, a, partial, stream);
}

}  // namespace dc
