// One output row of the paged read, exact to fp32 rounding, by one block (the
// mathematics in fem_paged.cu).
#pragma once

#include "fem_paged.cuh"

namespace fem {

constexpr int kExactThreads = 128;
constexpr int kExactTile = kExactThreads;  // keys per tile: a thread per key

struct ExactShared {
  float q[256];
  float p[kExactTile];          // the tile's prior weights
  float lp[kExactTile];         // and log weights s_i - m
  float vs[kExactTile];         // value scale of the key's row (e4m3)
  long long row[kExactTile];    // its cache row, -1: the key is not there
  float red[2][kExactThreads / 32];
  int list[kExactThreads];      // the channels to recompute
  int count;
};

// What the other kernels leave in the output of a channel that this path shall have: a NaN, as bf16.
constexpr unsigned short kExactMark = 0x7fff;

// expm1(b x) / b, continuous at b = 0
__device__ __forceinline__ float exact_em1(float b, float x) { return b != 0.f ? expm1f(b * x) / b : x; }

template <int FORMAT>
__device__ __forceinline__ float paged_value(const PagedCacheView &c, long long row, int j, float scale) {
  if (FORMAT == kCacheBf16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(c.v)[row * c.d + j]);
  if (FORMAT == kCacheF32) return static_cast<const float *>(c.v)[row * c.d + j];
  return e4m3x2_to_float2(static_cast<const uint8_t *>(c.v)[row * c.d + j]).x * scale;
}

// q . k of cache row `row`, q in shared memory as fp32
template <int FORMAT>
__device__ __forceinline__ float paged_dot(const PagedCacheView &c, long long row, const float *q) {
  float acc = 0.f;
  if (FORMAT == kCacheF32) {
    const float4 *k = reinterpret_cast<const float4 *>(static_cast<const float *>(c.k) + row * c.d);
    for (int j = 0; j < c.d / 4; ++j) {
      const float4 x = __ldg(k + j);
      acc = fmaf(x.x, q[4 * j], acc);
      acc = fmaf(x.y, q[4 * j + 1], acc);
      acc = fmaf(x.z, q[4 * j + 2], acc);
      acc = fmaf(x.w, q[4 * j + 3], acc);
    }
    return acc;
  }
  const int bytes = FORMAT == kCacheBf16 ? 2 : 1, per = 16 / bytes;
  const uint4 *k = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(c.k) + row * c.d * bytes);
  for (int j = 0; j < c.d / per; ++j) {
    const uint4 x = __ldg(k + j);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    const float *qj = q + j * per;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (FORMAT == kCacheBf16) {
        acc = fmaf(__int_as_float(static_cast<int>(w[u] << 16)), qj[2 * u], acc);
        acc = fmaf(__int_as_float(static_cast<int>(w[u] & 0xffff0000u)), qj[2 * u + 1], acc);
      } else {
        const float2 lo = e4m3x2_to_float2(w[u] & 0xffffu), hi = e4m3x2_to_float2(w[u] >> 16);
        acc = fmaf(lo.x, qj[4 * u], acc);
        acc = fmaf(lo.y, qj[4 * u + 1], acc);
        acc = fmaf(hi.x, qj[4 * u + 2], acc);
        acc = fmaf(hi.y, qj[4 * u + 3], acc);
      }
    }
  }
  return FORMAT == kCacheE4m3 ? acc * paged_scale(__ldg(c.ke + row)) : acc;
}

// State of one channel over some of the keys: the sum of their weights, the largest value and W against it, the
// largest log weight and A against it (fem_paged.cu).
struct ExactState {
  float L, ref, W, top, A;
};
// W against the larger value R
__device__ __forceinline__ float exact_move(const ExactState &x, float b, float R) {
  if (x.ref == R) return x.W;
  return x.L == 0.f ? 0.f : expf(b * (x.ref - R)) * x.W + exact_em1(b, x.ref - R) * x.L;
}
__device__ __forceinline__ ExactState exact_join(const ExactState &x, const ExactState &y, float b) {
  ExactState z;
  z.L = x.L + y.L;
  z.ref = fmaxf(x.ref, y.ref);
  z.W = exact_move(x, b, z.ref) + exact_move(y, b, z.ref);
  z.top = fmaxf(x.top, y.top);
  z.A = z.top == -INFINITY ? x.A + y.A : expf(x.top - z.top) * x.A + expf(y.top - z.top) * y.A;
  return z;
}

// Row t of sequence s (si), query head hq: channels j_lo .. j_hi - 1 into a.out, and
// with the first of them a.lse; `marked`: only those whose output (bf16) holds the mark.  All threads of a block
// of kExactThreads call it together.
//
// A channel has as many threads as there are for it, up to a warp, and they share its keys out: a row of 8192
// keys that wants one channel takes some 50 us, all 128 by a thread each ten times that.
template <int FORMAT>
__device__ void paged_exact_row(const PagedReadArgs &a, int s, const SeqInfo &si, int t, int hq, ExactShared &sh,
                                int j_lo, int j_hi, bool marked) {
  const PagedCacheView &c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = c.d, h = hq / a.group;
  const long long qrow = static_cast<long long>(si.q0) + t, orow = qrow * a.Hq + hq;
  const long long qoff = qrow * a.q_sn + hq * a.q_sh;
  __syncthreads();  // the previous row's readers of sh are done
  if (tid == 0) sh.count = 0;
  for (int j = tid; j < d; j += kExactThreads)
    sh.q[j] = FORMAT == kCacheF32 ? static_cast<const float *>(a.q)[qoff + j]
                                  : __bfloat162float(static_cast<const __nv_bfloat16 *>(a.q)[qoff + j]);
  __syncthreads();
  int n = j_hi - j_lo;
  if (marked) {  // at most kExactThreads of them
    if (tid < n && static_cast<const unsigned short *>(a.out)[orow * d + j_lo + tid] == kExactMark)
      sh.list[atomicAdd(&sh.count, 1)] = j_lo + tid;
    __syncthreads();
    n = sh.count;
    if (n == 0) return;
  }
  int shift = 0;  // log2 of a channel's threads
  while (shift < 5 && (n << (shift + 1)) <= kExactThreads) ++shift;
  const int step = 1 << shift, split = tid & (step - 1);
  const int limit = paged_limit(si, t, a.causal);
  float m = -INFINITY, L = 0.f;
  // up to two channels per thread (d <= 256)
  float beta[2];
  int ch[2];
  ExactState st[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = (tid >> shift) + u * (kExactThreads >> shift);
    ch[u] = i < n ? (marked ? sh.list[i] : j_lo + i) : -1;
    beta[u] = a.beta != nullptr && ch[u] >= 0 ? a.beta[static_cast<long long>(h) * d + ch[u]] : 0.f;
    st[u] = {0.f, -INFINITY, 0.f, -INFINITY, 0.f};
  }
  for (int k0 = 0; k0 < limit; k0 += kExactTile) {
    const int i = k0 + tid;
    float sc = -INFINITY;
    long long row = -1;
    if (i < limit) {
      const int page = paged_page(a, s, i);
      if (page >= 0) {
        row = paged_row(c, page, h, i);
        sc = paged_dot<FORMAT>(c, row, sh.q) * a.scale;
        if (FORMAT == kCacheE4m3) sh.vs[tid] = paged_scale(__ldg(c.ve + row));
      }
    }
    sh.row[tid] = row;
    float mx = sc;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    if (lane == 0) sh.red[0][warp] = mx;
    __syncthreads();
    const float m_new = fmaxf(fmaxf(fmaxf(sh.red[0][0], sh.red[0][1]), fmaxf(sh.red[0][2], sh.red[0][3])), m);
    // nothing but -inf so far: no weight to add (m_new is -inf also for a row of NaN, which goes on)
    const float lp = row < 0 ? -INFINITY : sc - (m_new == -INFINITY ? 0.f : m_new);
    const float p = row < 0 ? 0.f : expf(lp);
    sh.lp[tid] = lp;
    sh.p[tid] = p;
    float sum = p;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sh.red[1][warp] = sum;
    __syncthreads();
    const float alpha = m == m_new ? 1.f : expf(m - m_new);  // 0 for the first weight
    const float dm = m == m_new ? 0.f : m - m_new;
    const int cnt = min(limit - k0, kExactTile);
    L = fmaf(L, alpha, (sh.red[1][0] + sh.red[1][1]) + (sh.red[1][2] + sh.red[1][3]));
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int j = ch[u];
      if (j < 0) continue;
      const float b = beta[u];
      ExactState &x = st[u];
      // log weights are kept relative to m: the old maximum moves with it (-inf: nothing yet)
      x.L *= alpha;
      x.W *= alpha;
      if (x.top != -INFINITY) x.top += dm;
      // the tile's largest value and log weight, then its sums against them (the values come twice, from L1
      // the second time; without a branch on each key the loads of several keys are under way at once)
      float vmax = -INFINITY, xmax = -INFINITY;
#pragma unroll 8
      for (int kk = split; kk < cnt; kk += step) {
        const long long r = sh.row[kk];
        if (r >= 0) {
          const float v = paged_value<FORMAT>(c, r, j, FORMAT == kCacheE4m3 ? sh.vs[kk] : 1.f);
          vmax = fmaxf(vmax, v);
          xmax = fmaxf(xmax, fmaf(b, v, sh.lp[kk]));
        }
      }
      if (vmax > x.ref) {
        x.W = exact_move(x, b, vmax);
        x.ref = vmax;
      }
      if (xmax > x.top) {
        x.A *= expf(x.top - xmax);
        x.top = xmax;
      }
      const float t0 = x.top == -INFINITY ? 0.f : x.top;
#pragma unroll 8
      for (int kk = split; kk < cnt; kk += step) {
        const long long r = sh.row[kk];
        if (r >= 0) {
          const float v = paged_value<FORMAT>(c, r, j, FORMAT == kCacheE4m3 ? sh.vs[kk] : 1.f);
          x.W = fmaf(sh.p[kk], exact_em1(b, v == x.ref ? 0.f : v - x.ref), x.W);
          x.A += expf(fmaf(b, v, sh.lp[kk]) - t0);
          x.L += sh.p[kk];
        }
      }
    }
    m = m_new;
    __syncthreads();
  }
  const bool empty = m == -INFINITY && L == 0.f;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    for (int o = 1; o < step; o <<= 1) {
      ExactState y;
      y.L = __shfl_xor_sync(0xffffffffu, st[u].L, o);
      y.ref = __shfl_xor_sync(0xffffffffu, st[u].ref, o);
      y.W = __shfl_xor_sync(0xffffffffu, st[u].W, o);
      y.top = __shfl_xor_sync(0xffffffffu, st[u].top, o);
      y.A = __shfl_xor_sync(0xffffffffu, st[u].A, o);
      st[u] = split & o ? exact_join(y, st[u], beta[u]) : exact_join(st[u], y, beta[u]);
    }
    const int j = ch[u];
    if (j < 0 || split != 0) continue;
    float o = 0.f;
    if (!empty) {
      const ExactState &x = st[u];
      const float b = beta[u], y = b * x.W / L;
      if (b == 0.f) o = x.ref + x.W / L;
      else if (y > -0.5f) o = x.ref + log1pf(y) / b;
      else o = (x.top + logf(x.A) - logf(L)) / b;
    }
    if (FORMAT == kCacheF32) static_cast<float *>(a.out)[orow * d + j] = o;
    else static_cast<__nv_bfloat16 *>(a.out)[orow * d + j] = __float2bfloat16_rn(o);
  }
  if (a.lse != nullptr && tid == 0 && j_lo == 0) a.lse[orow] = empty ? -INFINITY : m + logf(L);
}

}  // namespace fem
