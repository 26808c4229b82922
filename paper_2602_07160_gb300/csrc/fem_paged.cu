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

// The rows that the reading kernel left: items cut by the ends of CTAs'
// stretches are joined from their pieces, in the line's order, and rows whose
// result the ranges could have spoilt are recomputed.  Blocks take RB rows.
constexpr int kMaxSplitCtas = 1024;

template <int FORMAT>
__global__ void __launch_bounds__(kExactThreads)
    paged_finish_kernel(const PagedReadArgs a, const PagedSplit sp, const SplitShape shape, int grid, int RB) {
  __shared__ ExactShared sh;
  __shared__ SplitScan<kExactThreads> scan;
  __shared__ float s_w[kMaxSplitCtas];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = a.c.d;
  const long long rows = static_cast<long long>(a.N) * a.Hq, first = static_cast<long long>(blockIdx.x) * RB;
  grid_dep_wait();
  unsigned mask = 0;
  if (RB == 1) {
    mask = sp.todo[first] == kRowDone ? 0u : 1u;
  } else {
    mask = __ballot_sync(0xffffffffu, lane < RB && first + lane < rows && sp.todo[first + lane] != kRowDone);
  }
  long long W = -1;
  int s_of = -1;  // the sequence that prefix belongs to
  long long prefix = 0;
  for (; mask; mask &= mask - 1) {
    const long long orow = first + __ffs(mask) - 1;
    const int row = static_cast<int>(orow / a.Hq), hq = static_cast<int>(orow - static_cast<long long>(row) * a.Hq);
    int lo = 0, hi = a.S;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (__ldg(a.q_off + mid) <= row) lo = mid; else hi = mid;
    }
    const SeqInfo si = paged_seq(a, lo);
    const int t = row - si.q0;
    if (t < 0 || t >= si.n) continue;  // nobody's row: its mark was never written
    bool exact = sp.todo[orow] == kRowExact;
    if (!exact) {
      if (W < 0) W = split_total(a, shape, scan);
      // the row's place: packed rows, or row tiles of whole tokens
      const int G = split_ctas(W, grid, shape), h = hq / a.group, gr = hq % a.group;
      const int tile = shape.tok ? t / shape.tok : (t * a.group + gr) / shape.row_tile;
      const int rr = shape.tok ? (t - tile * shape.tok) * a.group + gr : (t * a.group + gr) % shape.row_tile;
      const int kt = row_key_tiles(si, tile, a.causal, shape);
      if (s_of != lo) {
        // tiles before sequence lo
        long long w = 0;
        for (int s = tid; s < lo; s += kExactThreads) w += seq_tiles(a, paged_seq(a, s), shape);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
        __syncthreads();
        if (lane == 0) scan.warp[warp] = w;
        __syncthreads();
        prefix = 0;
#pragma unroll
        for (int i = 0; i < kExactThreads / 32; ++i) prefix += scan.warp[i];
        s_of = lo;
      }
      const long long x = prefix + h * head_key_tiles(si, seq_row_tiles(si, a.group, shape), a.group, a.causal, shape) +
                          head_key_tiles(si, tile, a.group, a.causal, shape);
      const int g0 = split_owner(W, G, x), g1 = split_owner(W, G, x + kt - 1), n = g1 - g0 + 1;
      const size_t size = piece_floats(shape.row_tile, d);
      const float *p0 = sp.pieces + (static_cast<size_t>(g0) * 2 + 1) * size;  // then every other slot 0
      auto piece = [&](int i) { return i == 0 ? p0 : sp.pieces + static_cast<size_t>(g0 + i) * 2 * size; };
      const float *stat = nullptr;
      float M = -INFINITY;
      for (int i = tid; i < n; i += kExactThreads) {
        stat = piece(i) + static_cast<size_t>(shape.row_tile) * d + 2 * rr;
        M = fmaxf(M, stat[0]);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      __syncthreads();
      if (lane == 0) sh.red[0][warp] = M;
      __syncthreads();
      M = fmaxf(fmaxf(sh.red[0][0], sh.red[0][1]), fmaxf(sh.red[0][2], sh.red[0][3]));
      float L = 0.f, wide = 0.f;
      for (int i = tid; i < n; i += kExactThreads) {
        stat = piece(i) + static_cast<size_t>(shape.row_tile) * d + 2 * rr;
        const float m = stat[0], l = stat[1];
        const float w = m == -INFINITY ? (l != l ? 1.f : 0.f) : ex2_approx(m - M);  // NaN scores have no maximum
        s_w[i] = w;
        L += w * l;
        wide += piece(i)[static_cast<size_t>(shape.row_tile) * d + 2 * shape.row_tile + d];
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) {
        L += __shfl_xor_sync(0xffffffffu, L, o);
        wide += __shfl_xor_sync(0xffffffffu, wide, o);
      }
      __syncthreads();
      if (lane == 0) {
        sh.red[0][warp] = L;
        sh.red[1][warp] = wide;
      }
      __syncthreads();
      L = (sh.red[0][0] + sh.red[0][1]) + (sh.red[0][2] + sh.red[0][3]);
      wide = (sh.red[1][0] + sh.red[1][1]) + (sh.red[1][2] + sh.red[1][3]);
      bool ok = true;
      if (tid < d) {
        float acc = 0.f;
        int i = 0;
        for (; i + 16 <= n; i += 16) {
          float v[16];
#pragma unroll
          for (int u = 0; u < 16; ++u) v[u] = piece(i + u)[static_cast<size_t>(rr) * d + tid];
#pragma unroll
          for (int u = 0; u < 16; ++u) acc = fmaf(s_w[i + u], v[u], acc);
        }
        for (; i < n; ++i) acc = fmaf(s_w[i], piece(i)[static_cast<size_t>(rr) * d + tid], acc);
        const float shift = p0[static_cast<size_t>(shape.row_tile) * d + 2 * shape.row_tile + tid];
        float o = 0.f;
        if (!(M == -INFINITY && L == 0.f))
          o = paged_out(a.beta ? a.beta[static_cast<long long>(h) * d + tid] : 0.f, shift, acc / L, wide != 0.f, &ok);
        static_cast<__nv_bfloat16 *>(a.out)[orow * d + tid] = __float2bfloat16_rn(o);
      }
      if (tid == 0 && a.lse != nullptr) a.lse[orow] = M == -INFINITY && L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
      exact = !__syncthreads_and(ok);
    }
    if (exact) paged_exact_row<FORMAT>(a, lo, si, t, hq, sh);
  }
}

}  // namespace

cudaError_t launch_paged_finish(const PagedReadArgs &a, const PagedSplit &sp, const SplitShape &shape, int grid,
                                int num_sms, cudaStream_t stream) {
  if (grid > kMaxSplitCtas) return cudaErrorInvalidValue;
  const long long rows = static_cast<long long>(a.N) * a.Hq;
  // a block per row while that is a few waves; then 32 rows, most of which need nothing
  const int RB = rows <= 32ll * num_sms ? 1 : 32;
  const dim3 blocks(static_cast<unsigned>((rows + RB - 1) / RB));
  if (a.c.format == kCacheBf16)
    return launch_kernel(paged_finish_kernel<kCacheBf16>, blocks, dim3(kExactThreads), 0, stream, true, a, sp, shape, grid,
                         RB);
  return launch_kernel(paged_finish_kernel<kCacheE4m3>, blocks, dim3(kExactThreads), 0, stream, true, a, sp, shape, grid,
                       RB);
}

cudaError_t launch_paged_exact(const PagedReadArgs &a, cudaStream_t stream) {
  const dim3 grid(a.N, a.Hq);
  if (a.c.format == kCacheBf16) paged_exact_kernel<kCacheBf16><<<grid, kExactThreads, 0, stream>>>(a);
  else if (a.c.format == kCacheE4m3) paged_exact_kernel<kCacheE4m3><<<grid, kExactThreads, 0, stream>>>(a);
  else paged_exact_kernel<kCacheF32><<<grid, kExactThreads, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace fem
