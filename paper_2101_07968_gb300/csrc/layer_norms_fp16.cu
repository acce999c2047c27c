// The block norms' kernels for half rows (one type per translation unit, so that
// they compile side by side).
#include "layer_norms.cuh"

namespace dc {

cudaError_t norm_forward_fp16(const NormArgs &a, cudaStream_t stream)
{
    return norms::forward<__half>(DC_FP16, a, stream);
}

cudaError_t norm_gradient_fp16(const NormArgs &a, float *partial, cudaStream_t stream)
{
    return norms::gradient<__half>(DC_FP16, a, partial, stream);
}

}  // namespace dc
