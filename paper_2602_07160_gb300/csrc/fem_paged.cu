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
#include "fem_paged_split.cuh"

namespace fem {

namespace {

template <int FORMAT>
__global__ void __launch_bounds__(kExactThreads) paged_exact_kernel(const PagedReadArgs a) {
  __shared__ ExactShared sh;
  const int row = blockIdx.x, hq = blockIdx.y;
  const int s = paged_owner(a, row);
  const SeqInfo si = paged_seq(a, s);
  const int t = row - si.q0;
  if (t < 0 || t >= si.n) return;  // a row no sequence owns
  paged_exact_row<FORMAT>(a, s, si, t, hq, sh);
}

// The rows that the reading kernel left: items cut by the ends of CTAs'
// stretches are joined from their pieces, in the line's order, a warp per row
// (its lanes side by side over the channels); rows whose result the ranges
// could have spoilt are then recomputed by the whole block.  A warp looks after
// RW rows.
template <int FORMAT, int D>
__global__ void __launch_bounds__(kExactThreads)
    paged_finish_kernel(const PagedReadArgs a, const PagedSplit sp, int row_tile, int grid, int RW) {
  constexpr int E = D / 32;  // channels per lane
  __shared__ ExactShared sh;
  __shared__ long long s_list[kExactThreads];
  __shared__ int s_count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long rows = static_cast<long long>(a.N) * a.Hq;
  const long long first = (static_cast<long long>(blockIdx.x) * (kExactThreads / 32) + warp) * RW;
  if (tid == 0) s_count = 0;
  __syncthreads();
  grid_dep_wait();
  const uint32_t mine = lane < RW && first + lane < rows ? sp.todo[first + lane] : 0u;
  const size_t size = piece_floats(row_tile, D);
  for (unsigned mask = __ballot_sync(0xffffffffu, mine != 0u); mask; mask &= mask - 1) {
    const int at = __ffs(mask) - 1;
    const uint32_t word = __shfl_sync(0xffffffffu, mine, at);
    const long long orow = first + at;
    bool exact = word == kRowExact;
    if (!exact) {
      const int rr = (word >> 2) & 255, g0 = (word >> 10) & 1023, n = static_cast<int>(word >> 20);
      // a word that a reading kernel which gave up left unwritten
      if ((word & 3u) != kRowSplit || rr >= row_tile || n < 1 || g0 + n > grid) continue;
      const int hq = static_cast<int>(orow % a.Hq), h = hq / a.group;
      const float *base = sp.pieces + static_cast<size_t>(g0) * 2 * size;  // piece 0 in slot 1, the others in slot 0
      auto piece = [&](int i) { return base + (static_cast<size_t>(i) * 2 + (i == 0 ? 1 : 0)) * size; };
      // the first pieces' accumulators are on their way while the weights are formed
      constexpr int kAhead = 4;
      float v[kAhead][E];
      auto load = [&](int i, float (&x)[E]) {
        const float *p = piece(i) + static_cast<size_t>(rr) * D + lane * E;
        if (E == 4) {
          const float4 y = *reinterpret_cast<const float4 *>(p);
          x[0] = y.x;
          x[1] = y.y;
          x[E - 2] = y.z;
          x[E - 1] = y.w;
        } else {
          const float2 y = *reinterpret_cast<const float2 *>(p);
          x[0] = y.x;
          x[1] = y.y;
        }
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (i < n) load(i, v[i]);
      float beta[E], kind[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        beta[e] = a.beta ? __ldg(a.beta + static_cast<long long>(h) * D + lane * E + e) : 0.f;
        kind[e] = piece(0)[row_tile * D + 2 * row_tile + lane * E + e];
      }
      float M = -INFINITY;
      for (int i = lane; i < n; i += 32) M = fmaxf(M, piece(i)[row_tile * D + 2 * rr]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      float acc[E], L = 0.f, wide = 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
      for (int i0 = 0; i0 < n; i0 += 32) {
        float w = 0.f;
        if (i0 + lane < n) {
          const float *p = piece(i0 + lane);
          const float m = p[row_tile * D + 2 * rr], l = p[row_tile * D + 2 * rr + 1];
          w = m == -INFINITY ? (l != l ? 1.f : 0.f) : ex2_approx(m - M);  // NaN scores have no maximum
          L += w * l;
          wide += p[row_tile * D + 2 * row_tile + D];
        }
        const int cnt = min(32, n - i0);
        if (i0 == 0) {
#pragma unroll
          for (int i = 0; i < kAhead; ++i) {
            const float wi = __shfl_sync(0xffffffffu, w, i);
            if (i < n) {
#pragma unroll
              for (int e = 0; e < E; ++e) acc[e] = fmaf(wi, v[i][e], acc[e]);
            }
          }
        }
#pragma unroll 8
        for (int i = i0 == 0 ? kAhead : 0; i < cnt; ++i) {
          const float wi = __shfl_sync(0xffffffffu, w, i);
          float x[E];
          load(i0 + i, x);
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e] = fmaf(wi, x[e], acc[e]);
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        L += __shfl_xor_sync(0xffffffffu, L, o);
        wide += __shfl_xor_sync(0xffffffffu, wide, o);
      }
      const bool empty = M == -INFINITY && L == 0.f;
      bool good = true;
      float o[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        bool ok;
        o[e] = paged_out(out_coef(beta[e], kind[e], a.beta && wide != 0.f), acc[e] / L, &ok);
        if (empty) o[e] = 0.f;
        good = good && (ok || empty);
      }
      __nv_bfloat162 *dst = reinterpret_cast<__nv_bfloat162 *>(static_cast<__nv_bfloat16 *>(a.out) + orow * D + lane * E);
#pragma unroll
      for (int e = 0; e < E; e += 2) dst[e / 2] = __floats2bfloat162_rn(o[e], o[e + 1]);
      if (lane == 0 && a.lse != nullptr) a.lse[orow] = empty ? -INFINITY : (M + log2f(L)) * kLn2;
      exact = !__all_sync(0xffffffffu, good);
    }
    if (exact && lane == 0) s_list[atomicAdd(&s_count, 1)] = orow;
  }
  __syncthreads();
  for (int i = 0; i < s_count; ++i) {
    const long long orow = s_list[i];
    const int row = static_cast<int>(orow / a.Hq), hq = static_cast<int>(orow - static_cast<long long>(row) * a.Hq);
    const int s = paged_owner(a, row);
    const SeqInfo si = paged_seq(a, s);
    const int t = row - si.q0;
    if (t >= 0 && t < si.n) paged_exact_row<FORMAT>(a, s, si, t, hq, sh);
  }
}

}  // namespace

cudaError_t launch_paged_finish(const PagedReadArgs &a, const PagedSplit &sp, const SplitShape &shape, int grid,
                                int num_sms, cudaStream_t stream) {
  if (grid > kMaxSplitCtas || shape.row_tile > 256) return cudaErrorInvalidValue;
  const long long rows = static_cast<long long>(a.N) * a.Hq;
  // a row per warp while that is at most about one wave of blocks; then 8, most of which need nothing
  const int warps = kExactThreads / 32, RW = rows <= 16ll * warps * num_sms ? 1 : 8;
  const dim3 blocks(static_cast<unsigned>((rows + RW * warps - 1) / (RW * warps)));
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, blocks, dim3(kExactThreads), 0, stream, true, a, sp, shape.row_tile, grid, RW);
  };
  if (a.c.format == kCacheBf16)
    return a.c.d == 64 ? go(paged_finish_kernel<kCacheBf16, 64>) : go(paged_finish_kernel<kCacheBf16, 128>);
  return a.c.d == 64 ? go(paged_finish_kernel<kCacheE4m3, 64>) : go(paged_finish_kernel<kCacheE4m3, 128>);
}

cudaError_t launch_paged_exact(const PagedReadArgs &a, cudaStream_t stream) {
  const dim3 grid(a.N, a.Hq);
  if (a.c.format == kCacheBf16) paged_exact_kernel<kCacheBf16><<<grid, kExactThreads, 0, stream>>>(a);
  else if (a.c.format == kCacheE4m3) paged_exact_kernel<kCacheE4m3><<<grid, kExactThreads, 0, stream>>>(a);
  else paged_exact_kernel<kCacheF32><<<grid, kExactThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace fem
