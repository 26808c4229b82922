// The read of new tokens over a paged cache, exact to fp32 rounding, on CUDA cores.
//
// One block per (new token, query head), or, where these are few, several that
// share its channels out.  The block walks the row's keys in tiles of 128: a
// thread per key forms s_i = q . k_i / sqrt(d); then the threads of each channel
// (one, or as many as there are for it) fold the tile's values.  With m the
// running row maximum and P_i = exp(s_i - m) they keep per channel
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
// cores do not take, and of single channels the other kernels hand over.  256
// tokens of 8 heads of 128 over 2048 fp32 keys (causal) take 2.3 ms, one token over
// 4096 keys 0.2 ms (1.3 with a block to a row).
#include "fem_launch.h"
#include "fem_paged.cuh"
#include "fem_paged_exact.cuh"
#include "fem_paged_split.cuh"

namespace fem {

namespace {

template <int FORMAT>
__global__ void __launch_bounds__(kExactThreads) paged_exact_kernel(const PagedReadArgs a, int channels) {
  __shared__ ExactShared sh;
  const int row = blockIdx.x, hq = blockIdx.y;
  const int s = paged_owner(a, row);
  const SeqInfo si = paged_seq(a, s);
  const int t = row - si.q0;
  if (t < 0 || t >= si.n) return;  // a row no sequence owns
  const int j_lo = blockIdx.z * channels;
  paged_exact_row<FORMAT>(a, s, si, t, hq, sh, j_lo, j_lo + channels, false);
}

// What the reading kernel left.  Block (g, part): rows 8 part .. of the item that
// CTA g began and did not end are joined from its pieces.  The four warps share
// the pieces out; a lane has row (lane & 7) and every fourth group of 4
// channels, so that each load is four full lines of a piece, whatever its
// length; the warps' sums meet in shared memory in the pieces' order.  Where
// there are few rows and many pieces the channels are shared out over blocks as
// well, CH to each (blockIdx.z).  Then
// channels whose result the ranges could have spoilt (marked in the output), of
// these rows and of those CTA g finished, are recomputed by the whole block.
// Alone it takes 21 us after a prompt of 8192 (304 pieces of 256 rows, 40 MB from L2)
// and 13 us after one token over 131071 keys; as a programmatic dependent its launch
// hides behind the reading kernel's tail.
template <int FORMAT, int D, int CH>
__global__ void __launch_bounds__(kExactThreads, 7)
    paged_finish_kernel(const PagedReadArgs a, const PagedSplit sp, const SplitShape shape, int grid) {
  constexpr int kWarps = kExactThreads / 32, C = CH / 16;  // C: groups of 4 channels per lane
  __shared__ union {
    ExactShared exact;
    float part[kWarps][8][CH + 4];
  } u;
  __shared__ float s_m[kWarps][8], s_l[kWarps][8], s_wide[kWarps];
  __shared__ int s_list[256];
  __shared__ int s_count;
  ExactShared &sh = u.exact;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g0 = blockIdx.x, part = blockIdx.y;
  const int row_tile = shape.row_tile, j_lo = blockIdx.z * CH;
  if (tid == 0) s_count = 0;
  grid_dep_wait();
  const SplitRecord rec = sp.records[g0];
  const size_t size = piece_floats(row_tile, D);
  const int n = rec.n;
  const float *base = sp.pieces + static_cast<size_t>(g0) * 2 * size;  // piece 0 in slot 1, the others in slot 0
  auto piece = [&](int i) { return base + (static_cast<size_t>(i) * 2 + (i == 0 ? 1 : 0)) * size; };
  // the class of channel j: the largest of its pieces'
  auto widest = [&](int j) {
    float most = 0.f;
    for (int i = 0; i < n; ++i) most = fmaxf(most, piece(i)[piece_classes(row_tile, D) + j]);
    return static_cast<int>(most);
  };
  if (part * 8 < rec.rows && n > 0) {
    const int r8 = lane & 7, c0 = lane >> 3, rr = part * 8 + r8, c4 = j_lo / 4 + c0;
    const bool on = rr < rec.rows;
    // this warp's pieces, its rows' sums against the largest maximum among them
    float m = -INFINITY, l = 0.f, wide = 0.f, acc[C][4];
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c][0] = acc[c][1] = acc[c][2] = acc[c][3] = 0.f;
#pragma unroll(32 / C)
    for (int i = warp; i < n; i += kWarps) {
      const float *p = piece(i);
      const float2 st = on ? *reinterpret_cast<const float2 *>(p + row_tile * D + 2 * rr) : make_float2(-INFINITY, 0.f);
      float4 v[C];
#pragma unroll
      for (int c = 0; c < C; ++c)
        v[c] = on ? *reinterpret_cast<const float4 *>(p + piece_at(rr, c4 + 4 * c, D)) : make_float4(0.f, 0.f, 0.f, 0.f);
      const float4 wd = *reinterpret_cast<const float4 *>(p + piece_wide(row_tile, D));
      wide += (wd.x + wd.y) + (wd.z + wd.w);
      const float top = fmaxf(m, st.x);
      // roots of the weights, applied twice
      const float r0 = m == -INFINITY ? (l != l ? 1.f : 0.f) : weight_root(m - top);
      const float r1 = st.x == -INFINITY ? (st.y != st.y ? 1.f : 0.f) : weight_root(st.x - top);  // NaN scores have no maximum
      m = top;
      l = fmaf(st.y * r1, r1, l * r0 * r0);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        acc[c][0] = fmaf(v[c].x * r1, r1, acc[c][0] * r0 * r0);
        acc[c][1] = fmaf(v[c].y * r1, r1, acc[c][1] * r0 * r0);
        acc[c][2] = fmaf(v[c].z * r1, r1, acc[c][2] * r0 * r0);
        acc[c][3] = fmaf(v[c].w * r1, r1, acc[c][3] * r0 * r0);
      }
    }
    if (c0 == 0) {
      s_m[warp][r8] = m;
      s_l[warp][r8] = l;
    }
    if (lane == 0) s_wide[warp] = wide;
#pragma unroll
    for (int c = 0; c < C; ++c)
      *reinterpret_cast<float4 *>(&u.part[warp][r8][4 * (c0 + 4 * c)]) = make_float4(acc[c][0], acc[c][1], acc[c][2], acc[c][3]);
    __syncthreads();
    // warp: rows 2 warp, 2 warp + 1; lane: CH / 32 channels side by side
    const SeqInfo si = paged_seq(a, rec.s);
    wide = (s_wide[0] + s_wide[1]) + (s_wide[2] + s_wide[3]);
    constexpr int E = CH / 32;
    OutCoef oc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = j_lo + lane * E + e;
      oc[e] = out_coef(a.beta ? __ldg(a.beta + static_cast<long long>(rec.h) * D + j) : 0.f,
                       piece(0)[piece_kinds(row_tile, D) + j], a.beta && wide != 0.f ? widest(j) : 0);
    }
#pragma unroll
    for (int k = 0; k < 8 / kWarps; ++k) {
      const int row = warp * (8 / kWarps) + k, rr2 = part * 8 + row;
      if (rr2 >= rec.rows) break;
      float M = -INFINITY, L = 0.f, x[E];
#pragma unroll
      for (int q = 0; q < kWarps; ++q) M = fmaxf(M, s_m[q][row]);
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = 0.f;
#pragma unroll
      for (int q = 0; q < kWarps; ++q) {
        const float root = s_m[q][row] == -INFINITY ? (s_l[q][row] != s_l[q][row] ? 1.f : 0.f) : weight_root(s_m[q][row] - M);
        L = fmaf(root, root * s_l[q][row], L);
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = fmaf(root, root * u.part[q][row][lane * E + e], x[e]);
      }
      const bool empty = M == -INFINITY && L == 0.f;
      if (L == INFINITY) L = __int_as_float(0x7fffffff);  // finite pieces, a sum past the range: no channel stands
      bool good = true;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        bool ok;
        x[e] = paged_out(oc[e], x[e] * ((a.beta ? kBankUnit : 1.f) / L), &ok);
        if (!ok) x[e] = __int_as_float(0x7fffffff);  // the mark, as bf16
        if (empty) x[e] = 0.f;
        good = good && (ok || empty);
      }
      const int t = (rec.row0 + rr2) / a.group, hq = rec.h * a.group + (rec.row0 + rr2) % a.group;
      const long long orow = (static_cast<long long>(si.q0) + t) * a.Hq + hq;
      __nv_bfloat16 *dst = static_cast<__nv_bfloat16 *>(a.out) + orow * D + j_lo + lane * E;
      if (E == 1) {
        *dst = __float2bfloat16_rn(x[0]);
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 2)
          *reinterpret_cast<__nv_bfloat162 *>(dst + e) = __floats2bfloat162_rn(x[e], x[e + (E > 1 ? 1 : 0)]);
      }
      if (lane == 0 && j_lo == 0 && a.lse != nullptr) a.lse[orow] = empty ? -INFINITY : (M + log2f(L)) * kLn2;
      if (!__all_sync(0xffffffffu, good) && lane == 0) s_list[atomicAdd(&s_count, 1)] = rec.row0 + rr2;
    }
    __syncthreads();
    for (int i = 0; i < s_count; ++i)
      paged_exact_row<FORMAT>(a, rec.s, si, s_list[i] / a.group, rec.h * a.group + s_list[i] % a.group, sh, j_lo, j_lo + CH,
                              true);
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
        paged_exact_row<FORMAT>(a, sg.s, sg.si, s_list[i] / a.group, sg.h * a.group + s_list[i] % a.group, sh, j_lo, j_lo + CH,
                                true);
    }
  }
}

}  // namespace

cudaError_t launch_paged_finish(const PagedReadArgs &a, const PagedSplit &sp, const SplitShape &shape, int grid,
                                cudaStream_t stream) {
  if (shape.row_tile > 256) return cudaErrorInvalidValue;
  const bool few = shape.row_tile <= 16;
  auto go = [&](auto kernel, int channels) {
    return launch_kernel(kernel, dim3(grid, shape.row_tile / 8, a.c.d / channels), dim3(kExactThreads), 0, stream, true, a, sp,
                         shape, grid);
  };
#define FEM_FINISH(F, DD) \
  if (a.c.format == F && a.c.d == DD) return few ? go(paged_finish_kernel<F, DD, 32>, 32) : go(paged_finish_kernel<F, DD, DD>, DD);
  FEM_FINISH(kCacheBf16, 64)
  FEM_FINISH(kCacheBf16, 128)
  FEM_FINISH(kCacheE4m3, 64)
  FEM_FINISH(kCacheE4m3, 128)
#undef FEM_FINISH
  return cudaErrorInvalidValue;
}

cudaError_t launch_paged_exact(const PagedReadArgs &a, int num_sms, cudaStream_t stream) {
  // channels are halved between blocks while those are fewer than four an SM; each then has more threads
  int channels = a.c.d;
  while (channels % 2 == 0 && channels > 8 && static_cast<long long>(a.N) * a.Hq * (a.c.d / channels) < 4ll * num_sms)
    channels /= 2;
  const dim3 grid(a.N, a.Hq, a.c.d / channels);
  if (a.c.format == kCacheBf16) paged_exact_kernel<kCacheBf16><<<grid, kExactThreads, 0, stream>>>(a, channels);
  else if (a.c.format == kCacheE4m3) paged_exact_kernel<kCacheE4m3><<<grid, kExactThreads, 0, stream>>>(a, channels);
  else paged_exact_kernel<kCacheF32><<<grid, kExactThreads, 0, stream>>>(a, channels);
  return cudaGetLastError();
}

}  // namespace fem
