// Gradients of the norms for a float residual stream (fem_norm_bwd.cuh).
#include "fem_norm_bwd.cuh"

namespace fem {

cudaError_t norm_bwd_f32(const NormArgs &a, int y_type, int num_sms, int *blocks, cudaStream_t stream) {
  return y_type == kTypeF32 ? types<float, float>(a, num_sms, blocks, stream)
                            : types<float, __nv_bfloat16>(a, num_sms, blocks, stream);
}

}  // namespace fem
