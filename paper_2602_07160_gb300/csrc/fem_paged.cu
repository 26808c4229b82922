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

// What the reading kernel left.  Block (g, part): the item that CTA g began and
// did not end is joined from its pieces, in the line's order, a warp per row
// (its lanes side by side over the channels), RW rows per warp; then rows whose
// result the ranges could have spoilt, these and those CTA g finished, are
// recomputed by the whole block.
template <int FORMAT, int D>
__global__ void __launch_bounds__(kExactThreads)
    paged_finish_kernel(const PagedReadArgs a, const PagedSplit sp, const SplitShape shape, int grid, int RW) {
  constexpr int E = D / 32, kWarps = kExactThreads / 32;  // channels per lane
  __shared__ ExactShared sh;
  __shared__ int s_list[256];
  __shared__ int s_count;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g0 = blockIdx.x, part = blockIdx.y;
  const int row_tile = shape.row_tile;
  if (tid == 0) s_count = 0;
  __syncthreads();
  grid_dep_wait();
  const SplitRecord rec = sp.records[g0];
  const size_t size = piece_floats(row_tile, D);
  const int n = rec.n;
  if (n > 0) {
    const SeqInfo si = paged_seq(a, rec.s);
    const float *base = sp.pieces + static_cast<size_t>(g0) * 2 * size;  // piece 0 in slot 1, the others in slot 0
    auto piece = [&](int i) { return (static_cast<size_t>(i) * 2 + (i == 0 ? 1 : 0)) * size; };
    for (int k = 0; k < RW; ++k) {
      const int rr = (part * kWarps + warp) * RW + k, h = rec.h;
      if (rr >= rec.rows) break;
      const int t = (rec.row0 + rr) / a.group, hq = h * a.group + (rec.row0 + rr) % a.group;
      const long long orow = (static_cast<long long>(si.q0) + t) * a.Hq + hq;
      const float *row = base + static_cast<size_t>(rr) * D + lane * E, *stat = base + row_tile * D + 2 * rr;
      // lane: piece; then every lane its channels of one piece after the other
      float M = -INFINITY, L = 0.f, wide = 0.f, acc[E];
#pragma unroll 1
      for (int i = lane; i < n; i += 32) M = fmaxf(M, stat[piece(i)]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
#pragma unroll 1
      for (int i0 = 0; i0 < n; i0 += 32) {
        float w = 0.f;
        if (i0 + lane < n) {
          const float m = stat[piece(i0 + lane)], l = stat[piece(i0 + lane) + 1];
          w = m == -INFINITY ? (l != l ? 1.f : 0.f) : ex2_approx(m - M);  // NaN scores have no maximum
          L += w * l;
          wide += base[piece(i0 + lane) + row_tile * D + 2 * row_tile + D];
        }
        const int cnt = min(32, n - i0);
#pragma unroll 8
        for (int i = 0; i < cnt; ++i) {
          const float wi = __shfl_sync(0xffffffffu, w, i);
          if (E == 4) {
            const float4 x = *reinterpret_cast<const float4 *>(row + piece(i0 + i));
            acc[0] = fmaf(wi, x.x, acc[0]);
            acc[1] = fmaf(wi, x.y, acc[1]);
            acc[E - 2] = fmaf(wi, x.z, acc[E - 2]);
            acc[E - 1] = fmaf(wi, x.w, acc[E - 1]);
          } else {
            const float2 x = *reinterpret_cast<const float2 *>(row + piece(i0 + i));
            acc[0] = fmaf(wi, x.x, acc[0]);
            acc[1] = fmaf(wi, x.y, acc[1]);
          }
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
        const int j = lane * E + e;
        const float beta = a.beta ? __ldg(a.beta + static_cast<long long>(h) * D + j) : 0.f;
        o[e] = paged_out(out_coef(beta, base[piece(0) + row_tile * D + 2 * row_tile + j], a.beta && wide != 0.f), acc[e] / L, &ok);
        if (empty) o[e] = 0.f;
        good = good && (ok || empty);
      }
      __nv_bfloat162 *dst = reinterpret_cast<__nv_bfloat162 *>(static_cast<__nv_bfloat16 *>(a.out) + orow * D + lane * E);
#pragma unroll
      for (int e = 0; e < E; e += 2) dst[e / 2] = __floats2bfloat162_rn(o[e], o[e + 1]);
      if (lane == 0 && a.lse != nullptr) a.lse[orow] = empty ? -INFINITY : (M + log2f(L)) * kLn2;
      if (!__all_sync(0xffffffffu, good) && lane == 0) s_list[atomicAdd(&s_count, 1)] = rr;
    }
    __syncthreads();
    for (int i = 0; i < s_count; ++i) {
      const int r = rec.row0 + s_list[i];
      paged_exact_row<FORMAT>(a, rec.s, si, r / a.group, rec.h * a.group + r % a.group, sh);
    }
  }
  if (rec.any_exact) {
    // CTA g's whole items again, for their marked rows
    __shared__ SplitScan<kExactThreads> scan;
    SplitWalk walk;
    SplitSeg sg;
    if (!split_begin(a, shape, g0, grid, scan, walk)) return;
    while (walk.next(a, shape, sg)) {
      if (sg.kt0 != 0 || sg.kt1 != sg.kt_all) continue;
      const int row0 = shape.tok ? sg.r * shape.tok * a.group : sg.r * row_tile;
      const int rows = min(shape.tok ? shape.tok * a.group : row_tile, sg.si.n * a.group - row0);
      // the rows this block looks after, a thread each (at most 256 / gridDim.y of them)
      const int mine = part + tid * gridDim.y;
      __syncthreads();
      if (tid == 0) s_count = 0;
      __syncthreads();
      if (mine < rows) {
        const int t = (row0 + mine) / a.group, hq = sg.h * a.group + (row0 + mine) % a.group;
        if (sp.exact[(static_cast<long long>(sg.si.q0) + t) * a.Hq + hq]) s_list[atomicAdd(&s_count, 1)] = row0 + mine;
      }
      __syncthreads();
      for (int i = 0; i < s_count; ++i)
        paged_exact_row<FORMAT>(a, sg.s, sg.si, s_list[i] / a.group, sg.h * a.group + s_list[i] % a.group, sh);
    }
  }
}

}  // namespace

cudaError_t launch_paged_finish(const PagedReadArgs &a, const PagedSplit &sp, const SplitShape &shape, int grid,
                                cudaStream_t stream) {
  if (shape.row_tile > 256) return cudaErrorInvalidValue;
  // a row per warp for the row tiles of few rows, two for those of 256
  const int warps = kExactThreads / 32, RW = shape.row_tile > 16 ? 2 : 1;
  const dim3 blocks(grid, shape.row_tile / (RW * warps));
  auto go = [&](auto kernel) {
    return launch_kernel(kernel, blocks, dim3(kExactThreads), 0, stream, true, a, sp, shape, grid, RW);
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
