// Shared by the operators around the read (rotary positions, the gated recurrence, norms with gate and residual):
// their arguments as the kernels take them, and elements as they lie in memory.
#pragma once

#include <atomic>

#include "fem_common.cuh"

namespace fem {

constexpr int kTypeBf16 = 0, kTypeF32 = 2;  // fem_type

// Element (b, t, h, j) of [B, T, H, d] at p + b sb + t st + h sh + j.
struct HeadsView {
  void *p;
  long long sb, st, sh;
};

struct RopeArgs {
  HeadsView in[2], out[2];  // queries, keys
  int heads[2];             // heads[1] = 0: no keys
  int B, T, d, rotary;
  const unsigned long long *turns;
  const int *pos;
  float amplitude;
  int inverse;
};
cudaError_t launch_rope(const RopeArgs &a, int type, bool interleaved, int num_sms, cudaStream_t stream);

constexpr long long kRecurMostStride = 1ll << 20;  // elements between rows: a thread's 16 steps of them are products of 32 bits
struct RecurArgs {
  const void *s, *u, *h, *dh;  // h is read by the backward pass only
  long long s_st, u_st, h_st, dh_st;
  void *out, *du;  // h, or ds and du
  long long out_st, du_st;
  const int *offsets, *state_rows;
  int S, T, N, C, num_states;
  const float *first;  // h0, or dh_last: the state that a scan starts from
  float *last;         // h_last, or dh0
  const float *h0;     // backward: what precedes h at a sequence's first step
  unsigned *err;
};
// `ws` holds recur_workspace_bytes() bytes, 0 where lines are not cut.
size_t recur_workspace_bytes(const RecurArgs &a, int type, bool bwd, int num_sms);
cudaError_t launch_recur(const RecurArgs &a, int type, bool mean, bool bwd, int num_sms, void *ws, cudaStream_t stream);

struct NormArgs {
  int B, T, H, d, N, D;
  int post, pre, act;  // fem_norm_kind; act -1: no gate
  float scale, eps;
  const float *w_post, *b_post, *w_pre, *b_pre;
  const void *x;       // forward: x; backward: r
  HeadsView y, gate;   // y.p NULL: no block before
  void *r, *z;         // forward's outputs
  const void *dr, *dz;
  void *dx;
  HeadsView dy, dgate;
  float *dw[4];        // dw_post, db_post, dw_pre, db_pre, or NULL
  float *part;         // [blocks, 4, D] at most, or NULL: no sums
};
cudaError_t launch_norm_fwd(const NormArgs &a, int x_type, int y_type, int num_sms, cudaStream_t stream);
// `blocks` of norm_bwd_blocks, each of which leaves a row of partial sums of the weights' gradients.
cudaError_t norm_bwd_blocks(const NormArgs &a, int x_type, int y_type, int num_sms, int *blocks);
cudaError_t launch_norm_bwd(const NormArgs &a, int x_type, int y_type, int blocks, cudaStream_t stream);

// Blocks of `kernel` that an SM holds, with `smem` bytes of dynamic shared memory, which it is allowed to have; asked of
// the driver once for each device and `Tag`, a type of the kernel's own.
template <typename Tag, typename Kernel>
cudaError_t resident_blocks(Kernel *kernel, int threads, int smem, int *blocks) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 64 && (*blocks = known[dev].load(std::memory_order_relaxed)) > 0) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, kernel, threads, smem);
  if (e == cudaSuccess && *blocks < 1) e = cudaErrorInvalidConfiguration;
  if (e == cudaSuccess && dev < 64) known[dev].store(*blocks, std::memory_order_relaxed);
  return e;
}

__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16_pack(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}

// Eight elements of a row as they lie in memory.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 a;
};
template <>
struct Eight<float> {
  float4 a, b;
};

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

}  // namespace fem
