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
};

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

// Row t of sequence s (si), query head hq: channels j_lo .. j_hi - 1 into a.out, and
// with the first of them a.lse.  All threads of a block of kExactThreads call it
// together.
template <int FORMAT>
__device__ void paged_exact_row(const PagedReadArgs &a, int s, const SeqInfo &si, int t, int hq, ExactShared &sh,
                                int j_lo, int j_hi) {
  const PagedCacheView &c = a.c;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, d = c.d, h = hq / a.group;
  const long long qrow = static_cast<long long>(si.q0) + t;
  const long long qoff = qrow * a.q_sn + hq * a.q_sh;
  __syncthreads();  // the previous row's readers of sh are done
  for (int j = tid; j < d; j += kExactThreads)
    sh.q[j] = FORMAT == kCacheF32 ? static_cast<const float *>(a.q)[qoff + j]
                                  : __bfloat162float(static_cast<const __nv_bfloat16 *>(a.q)[qoff + j]);
  __syncthreads();
  const int limit = paged_limit(si, t, a.causal);
  float m = -INFINITY, L = 0.f;
  // two channels per thread (d <= 256)
  float beta[2], top[2] = {-INFINITY, -INFINITY}, A[2] = {0.f, 0.f}, ref[2] = {-INFINITY, -INFINITY}, W[2] = {0.f, 0.f};
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int j = tid + u * kExactThreads;
    beta[u] = (a.beta != nullptr && j < d) ? a.beta[static_cast<long long>(h) * d + j] : 0.f;
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
    __syncthreads();
    const float alpha = m == m_new ? 1.f : expf(m - m_new);  // 0 for the first weight
    const float dm = m == m_new ? 0.f : m - m_new;
    const int cnt = min(limit - k0, kExactTile);
    const float L_old = L * alpha;
    float L_new = L_old;
    for (int kk = 0; kk < cnt; ++kk) L_new += sh.p[kk];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int j = tid + u * kExactThreads;
      if (j < j_lo || j >= j_hi) continue;
      const float b = beta[u];
      // log weights are kept relative to m: the old maximum moves with it (-inf: nothing yet)
      W[u] *= alpha;
      if (top[u] != -INFINITY) top[u] += dm;
      // the tile's largest value and log weight, then its sums against them (the values come twice, from L1
      // the second time; without a branch on each key the loads of several keys are under way at once)
      float vmax = -INFINITY, xmax = -INFINITY;
#pragma unroll 8
      for (int kk = 0; kk < cnt; ++kk) {
        const long long r = sh.row[kk];
        if (r >= 0) {
          const float v = paged_value<FORMAT>(c, r, j, FORMAT == kCacheE4m3 ? sh.vs[kk] : 1.f);
          vmax = fmaxf(vmax, v);
          xmax = fmaxf(xmax, fmaf(b, v, sh.lp[kk]));
        }
      }
      if (vmax > ref[u]) {
        if (L_old > 0.f)
          W[u] = (ref[u] == -INFINITY ? 0.f : expf(b * (ref[u] - vmax)) * W[u]) + exact_em1(b, ref[u] - vmax) * L_old;
        ref[u] = vmax;
      }
      if (xmax > top[u]) {
        A[u] *= expf(top[u] - xmax);
        top[u] = xmax;
      }
      const float t0 = top[u] == -INFINITY ? 0.f : top[u];
#pragma unroll 8
      for (int kk = 0; kk < cnt; ++kk) {
        const long long r = sh.row[kk];
        if (r >= 0) {
          const float v = paged_value<FORMAT>(c, r, j, FORMAT == kCacheE4m3 ? sh.vs[kk] : 1.f);
          W[u] = fmaf(sh.p[kk], exact_em1(b, v == ref[u] ? 0.f : v - ref[u]), W[u]);
          A[u] += expf(fmaf(b, v, sh.lp[kk]) - t0);
        }
      }
    }
    L = L_new;
    m = m_new;
    __syncthreads();
  }
  const bool empty = m == -INFINITY && L == 0.f;
  const long long orow = qrow * a.Hq + hq;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int j = tid + u * kExactThreads;
    if (j < j_lo || j >= j_hi) continue;
    float o = 0.f;
    if (!empty) {
      const float b = beta[u], x = b * W[u] / L;
      if (b == 0.f) o = ref[u] + W[u] / L;
      else if (x > -0.5f) o = ref[u] + log1pf(x) / b;
      else o = (top[u] + logf(A[u]) - logf(L)) / b;
    }
    if (FORMAT == kCacheF32) static_cast<float *>(a.out)[orow * d + j] = o;
    else static_cast<__nv_bfloat16 *>(a.out)[orow * d + j] = __float2bfloat16_rn(o);
  }
  if (a.lse != nullptr && tid == 0 && j_lo == 0) a.lse[orow] = empty ? -INFINITY : m + logf(L);
}

}  // namespace fem
