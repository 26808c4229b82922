// The read of new tokens over a paged cache, exact to fp32 rounding, on CUDA cores.
//
// One block per (new token, query head).  The block walks the row's keys in
// tiles of 128: a thread per key forms s_i = q . k_i / sqrt(d); then a thread
// per channel folds the tile's values in order.  With m the running row
// maximum and P_i = exp(s_i - m) it keeps per channel
//   LSE_j = log sum_i exp(s_i + beta_j v_ij)      as a running maximum a_j and sum A_j,
//   W_j   = sum_i P_i expm1(beta_j (v_ij - c_j)) / beta_j   (v_ij - c_j at beta 0),
// c_j the running maximum of the visible values.  When c grows to c',
// W <- exp(beta (c - c')) W + expm1(beta (c - c'))/beta L.  The read is
//   o = c + log1p(beta W / L) / beta   when beta W / L > -1/2 (no cancellation),
//   o = (LSE_j - lse) / beta           otherwise,
//   o = c + W / L                      at beta = 0 (the prior mean),
// so no spread of beta v and no prior, however peaked, loses the result.
// Every row costs (keys x d) exponentials twice and shares nothing with its
// neighbours: the path of fp32 caches and of the head dimensions the tensor
// cores do not take, and of single rows the other kernels hand over.
#include "fem_launch.h"
#include "fem_paged.cuh"
#include "fem_paged_exact.cuh"

namespace fem {

namespace {

template <int FORMAT>
__global__ void __launch_bounds__(kExactThreads) paged_exact_kernel(const PagedReadArgs a) {
  __shared__ ExactShared sh;
  const int row = blockIdx.x, hq = blockIdx.y;
  // the sequence that owns the row: the last s with q_off[s] <= row (empty sequences in between own none)
  int lo = 0, hi = a.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (__ldg(a.q_off + mid) <= row) lo = mid; else hi = mid;
  }
  const SeqInfo si = paged_seq(a, lo);
  const int t = row - si.q0;
  if (t < 0 || t >= si.n) return;  // a row no sequence owns
  paged_exact_row<FORMAT>(a, lo, si, t, hq, sh);
}

}  // namespace

cudaError_t launch_paged_exact(const PagedReadArgs &a, cudaStream_t stream) {
  const dim3 grid(a.N, a.Hq);
  if (a.c.format == kCacheBf16) paged_exact_kernel<kCacheBf16><<<grid, kExactThreads, 0, stream>>>(a);
  else if (a.c.format == kCacheE4m3) paged_exact_kernel<kCacheE4m3><<<grid, kExactThreads, 0, stream>>>(a);
  else paged_exact_kernel<kCacheF32><<<grid, kExactThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace fem
