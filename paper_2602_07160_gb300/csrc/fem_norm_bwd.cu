// Gradients of the norms for a bf16 residual stream, and the sums of the weights' gradients (fem_norm_bwd.cuh).
#include "fem_norm_bwd.cuh"

namespace fem {

namespace {

// Adds the partial sums of `blocks` rows, 32 columns a block, its 32 warps taking every 32nd row; the first kernel's
// dependent, it waits where that one's sums are read.
__global__ void __launch_bounds__(1024) norm_bwd_sum_kernel(const float *part, int blocks, int sums, int D, float *w_post,
                                                            float *b_post, float *w_pre, float *b_pre) {
  __shared__ float s_sum[32][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, k = blockIdx.y, e = blockIdx.x * 32 + lane;
  float *out = k == 0 ? w_post : k == 1 ? w_pre : k == 2 ? b_post : b_pre;
  grid_dep_wait();
  if (!out) return;
  float v = 0.f;
  if (e < D) {
#pragma unroll 4
    for (int i = w; i < blocks; i += 32) v += part[(static_cast<long long>(i) * sums + k) * D + e];
  }
  s_sum[w][lane] = v;
  __syncthreads();
  v = s_sum[lane][w];  // column w, the part of warp `lane`
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0 && blockIdx.x * 32 + w < D) out[blockIdx.x * 32 + w] = v;
}

}  // namespace

cudaError_t launch_norm_sums(const NormArgs &a, int blocks, int sums, cudaStream_t stream) {
  return launch_kernel(norm_bwd_sum_kernel, dim3((a.D + 31) / 32, sums), dim3(1024), 0, stream, true, a.part, blocks, sums, a.D, a.dw[0],
                       a.dw[1], a.dw[2], a.dw[3]);
}

cudaError_t norm_bwd_blocks(const NormArgs &a, int x_type, int y_type, int num_sms, int *blocks) {
  return x_type == kTypeF32 ? norm_bwd_f32(a, y_type, num_sms, blocks, nullptr)
                            : types<__nv_bfloat16, __nv_bfloat16>(a, num_sms, blocks, nullptr);
}

cudaError_t launch_norm_bwd(const NormArgs &a, int x_type, int y_type, int blocks, cudaStream_t stream) {
  return x_type == kTypeF32 ? norm_bwd_f32(a, y_type, 0, &blocks, stream) : types<__nv_bfloat16, __nv_bfloat16>(a, 0, &blocks, stream);
}

}  // namespace fem
