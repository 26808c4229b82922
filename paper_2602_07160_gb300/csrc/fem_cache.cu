// Writing a paged cache and reading it back (layout and format in fem_paged.cuh).
//
// Both are bound by memory: every element is read once and written once, with
// no arithmetic to speak of.  The rows are short (d elements of one token and
// head), so a group of G lanes takes a row with 16-byte accesses, and the
// row's largest magnitude (the e4m3 scale) is a butterfly over the group.
#include <cuda_fp8.h>

#include "fem_launch.h"
#include "fem_paged.cuh"

namespace fem {

namespace {

struct CacheWrite {
  PagedCacheView c;
  const void *k, *v;
  long long k_sn, k_sh, v_sn, v_sh;  // element strides over tokens and heads
  const long long *slots;
  int N;
  unsigned *err;
};

// Scale exponent of a row with largest magnitude amax (finite): the smallest e
// with amax <= 448 2^e.  amax = f 2^x with 1 <= f < 2 and 448 = 1.75 2^8.
__device__ __forceinline__ int scale_exponent(float amax) {
  const int bits = __float_as_int(amax);
  const int x = (bits >> 23) - 127;
  const int e = (bits & 0x7fffff) <= 0x600000 ? x - 8 : x - 7;
  return min(max(e, kScaleExpMin), kScaleExpMax);
}

// G lanes per row, 8 elements per lane at a time (bf16 and e4m3), 4 (fp32).
template <int G, int FORMAT>
__global__ void __launch_bounds__(256) cache_write_kernel(const CacheWrite a) {
  constexpr int E = FORMAT == kCacheF32 ? 4 : 8;
  const int lane = threadIdx.x % G;
  const int H = a.c.H, d = a.c.d, page_mask = (1 << a.c.page_shift) - 1;
  const long long rows = 2ll * a.N * H, n_slots = static_cast<long long>(a.c.num_pages) << a.c.page_shift;
  const long long step = static_cast<long long>(gridDim.x) * (256 / G);
  // every lane of a warp runs the same number of rounds: the butterfly below names all of them
  const long long first = static_cast<long long>(blockIdx.x) * (256 / G) + threadIdx.x / G;
  for (long long base = static_cast<long long>(blockIdx.x) * (256 / G), r = first; base < rows; base += step, r += step) {
    bool on = r < rows;
    const int n = on ? static_cast<int>(r / (2 * H)) : 0, rem = on ? static_cast<int>(r - 2ll * H * n) : 0;
    const bool is_v = rem >= H;
    const int h = is_v ? rem - H : rem;
    const long long slot = on ? a.slots[n] : -1;
    if (slot >= n_slots && lane == 0) atomicOr(a.err, kErrPageRange);
    on = on && slot >= 0 && slot < n_slots;
    const long long src = is_v ? n * a.v_sn + h * a.v_sh : n * a.k_sn + h * a.k_sh;
    const int page = static_cast<int>(slot >> a.c.page_shift);
    const long long row = on ? paged_row(a.c, page, h, static_cast<int>(slot & page_mask)) : 0;
    const int j = lane * E;
    const bool has = on && j < d;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (has) {
      if (FORMAT == kCacheF32)
        x = *reinterpret_cast<const uint4 *>(static_cast<const float *>(is_v ? a.v : a.k) + src + j);
      else
        x = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(is_v ? a.v : a.k) + src + j);
    }
    if (FORMAT == kCacheF32) {
      // d <= 256 in 4-element pieces: two per lane at most (G = 32 covers 128 elements)
      if (has) *reinterpret_cast<uint4 *>(static_cast<float *>(is_v ? a.c.v : a.c.k) + row * d + j) = x;
      if (on && j + G * E < d) {
        const float *s2 = static_cast<const float *>(is_v ? a.v : a.k) + src + j + G * E;
        *reinterpret_cast<uint4 *>(static_cast<float *>(is_v ? a.c.v : a.c.k) + row * d + j + G * E) =
            *reinterpret_cast<const uint4 *>(s2);
      }
    } else if (FORMAT == kCacheBf16) {
      if (has) *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(is_v ? a.c.v : a.c.k) + row * d + j) = x;
    } else {
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
      // magnitudes of bf16 order as their bits; infinities and NaN come last
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
      const bool bad = top >= 0x7f80u;
      const int e = scale_exponent(__int_as_float(static_cast<int>(top << 16)));
      // 2^-e is a normal number for e in [-100, 120]; the products are exact
      const float inv = __int_as_float((127 - e) << 23), lim = e == kScaleExpMax ? 240.f : 448.f;
      uint32_t code[2] = {0, 0};
      if (!bad) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float lo = __int_as_float(static_cast<int>(w[i] << 16)) * inv;
          const float hi = __int_as_float(static_cast<int>(w[i] & 0xffff0000u)) * inv;
          const float2 p = make_float2(fminf(fmaxf(lo, -lim), lim), fminf(fmaxf(hi, -lim), lim));
          code[i / 2] |= static_cast<uint32_t>(__nv_cvt_float2_to_fp8x2(p, __NV_SATFINITE, __NV_E4M3)) << (16 * (i & 1));
        }
      }
      if (has) {
        *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(is_v ? a.c.v : a.c.k) + row * d + j) =
            make_uint2(code[0], code[1]);
        if (lane == 0) (is_v ? a.c.ve : a.c.ke)[row] = static_cast<uint8_t>(bad ? kScaleNan : e + kScaleBias);
      }
    }
  }
}

struct CacheGather {
  PagedCacheView c;
  const int *table, *starts, *offsets;
  int max_pages, S, total;
  void *k, *v;
  unsigned *err;
};

// One block per output position (all heads of k and v).
template <int FORMAT>
__global__ void __launch_bounds__(256) cache_gather_kernel(const CacheGather a) {
  constexpr int E = FORMAT == kCacheF32 ? 4 : 8;
  const int n = blockIdx.x, H = a.c.H, d = a.c.d;
  // the sequence that owns row n: the last s with offsets[s] <= n
  int lo = 0, hi = a.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (__ldg(a.offsets + mid) <= n) lo = mid; else hi = mid;
  }
  const int o0 = __ldg(a.offsets + lo), o1 = __ldg(a.offsets + lo + 1);
  const long long i = static_cast<long long>(__ldg(a.starts + lo)) + (n - o0);
  const long long p = i >> a.c.page_shift;
  int page = -1;
  if (n >= o0 && n < o1 && i >= 0 && p < a.max_pages) page = __ldg(a.table + static_cast<long long>(lo) * a.max_pages + p);
  const bool ok = static_cast<unsigned>(page) < static_cast<unsigned>(a.c.num_pages);
  if (!ok && threadIdx.x == 0) atomicOr(a.err, kErrPageRange);
  const int per = d / E, pieces = 2 * H * per;
  for (int t = threadIdx.x; t < pieces; t += 256) {
    const int r = t / per, j = (t - r * per) * E;
    const bool is_v = r >= H;
    const int h = is_v ? r - H : r;
    const long long row = ok ? paged_row(a.c, page, h, static_cast<int>(i & ((1 << a.c.page_shift) - 1))) : 0;
    const long long dst = (static_cast<long long>(n) * H + h) * d + j;
    uint4 y = make_uint4(0, 0, 0, 0);
    if (ok) {
      if (FORMAT == kCacheE4m3) {
        const uint2 x = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(is_v ? a.c.v : a.c.k) + row * d + j);
        const float s = paged_scale((is_v ? a.c.ve : a.c.ke)[row]);
        const uint32_t w[4] = {x.x & 0xffffu, x.x >> 16, x.y & 0xffffu, x.y >> 16};
        uint32_t o[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float2 f = e4m3x2_to_float2(w[u]);
          const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * s, f.y * s);
          o[u] = *reinterpret_cast<const uint32_t *>(&b);
        }
        y = make_uint4(o[0], o[1], o[2], o[3]);
      } else if (FORMAT == kCacheBf16) {
        y = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(is_v ? a.c.v : a.c.k) + row * d + j);
      } else {
        y = *reinterpret_cast<const uint4 *>(static_cast<const float *>(is_v ? a.c.v : a.c.k) + row * d + j);
      }
    }
    if (FORMAT == kCacheF32)
      *reinterpret_cast<uint4 *>(static_cast<float *>(is_v ? a.v : a.k) + dst) = y;
    else
      *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(is_v ? a.v : a.k) + dst) = y;
  }
}

template <int FORMAT>
cudaError_t launch_write_f(const CacheWrite &a, int num_sms, cudaStream_t s) {
  const int per = a.c.d / (FORMAT == kCacheF32 ? 4 : 8);
  int G = 2;
  while (G < per && G < 32) G *= 2;
  const long long rows = 2ll * a.N * a.c.H, blocks = (rows + 256 / G - 1) / (256 / G);
  const int grid = static_cast<int>(blocks < 32ll * num_sms ? blocks : 32ll * num_sms);
  switch (G) {
    case 2: cache_write_kernel<2, FORMAT><<<grid, 256, 0, s>>>(a); break;
    case 4: cache_write_kernel<4, FORMAT><<<grid, 256, 0, s>>>(a); break;
    case 8: cache_write_kernel<8, FORMAT><<<grid, 256, 0, s>>>(a); break;
    case 16: cache_write_kernel<16, FORMAT><<<grid, 256, 0, s>>>(a); break;
    default: cache_write_kernel<32, FORMAT><<<grid, 256, 0, s>>>(a); break;
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_write(const PagedCacheView &c, const void *k, const void *v, long long k_sn, long long k_sh,
                               long long v_sn, long long v_sh, const long long *slots, int N, unsigned *err,
                               int num_sms, cudaStream_t stream) {
  const CacheWrite a = {c, k, v, k_sn, k_sh, v_sn, v_sh, slots, N, err};
  if (c.format == kCacheBf16) return launch_write_f<kCacheBf16>(a, num_sms, stream);
  if (c.format == kCacheE4m3) return launch_write_f<kCacheE4m3>(a, num_sms, stream);
  return launch_write_f<kCacheF32>(a, num_sms, stream);
}

cudaError_t launch_cache_gather(const PagedCacheView &c, const int *table, int max_pages, const int *starts,
                                const int *offsets, int S, int total, void *k, void *v, unsigned *err,
                                cudaStream_t stream) {
  const CacheGather a = {c, table, starts, offsets, max_pages, S, total, k, v, err};
  if (c.format == kCacheBf16) cache_gather_kernel<kCacheBf16><<<total, 256, 0, stream>>>(a);
  else if (c.format == kCacheE4m3) cache_gather_kernel<kCacheE4m3><<<total, 256, 0, stream>>>(a);
  else cache_gather_kernel<kCacheF32><<<total, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace fem
