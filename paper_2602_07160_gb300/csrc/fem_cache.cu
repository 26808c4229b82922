// Writing a paged cache and reading it back (layout and format in fem_paged.cuh).
//
// Both are bound by memory: every element is read once and written once, and
// the quantisation's arithmetic is kept under the copies.  The rows are short (d
// elements of one token and head), so a group of G lanes takes a row with 16-byte
// accesses, and the row's largest magnitude (the e4m3 scale) is a butterfly over
// the group.
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

// G lanes per row.  A group takes write_rows rows of one token (of its keys' heads, then its values'), whose loads, 64
// bytes a lane, leave together.  8192 tokens of 16 heads of 128 into e4m3 take 19.3 us, 5.2 TB/s (4 rows 20.5 us, one
// 20.6, 8 24.4; half the elements to a lane 21.1).  With a comparison and a clamp per element, where words of two
// elements do and no clamp is needed, the integer pipe was busy for 73 % of 24.0 us.
__host__ __device__ constexpr int write_rows(int format) { return format == kCacheE4m3 ? 2 : 4; }

template <int G, int FORMAT>
__global__ void __launch_bounds__(256) cache_write_kernel(const CacheWrite a) {
  // elements per lane and step, bytes of one
  constexpr int E = FORMAT == kCacheF32 ? 4 : FORMAT == kCacheBf16 ? 8 : 16, kIn = FORMAT == kCacheF32 ? 4 : 2;
  // 16-byte pieces of a lane, and the elements between them: fp32 rows of up to 256 take two steps; 16 elements side by
  // side become 16 bytes of codes
  constexpr int kRows = write_rows(FORMAT), kPieces = FORMAT == kCacheBf16 ? 1 : 2, kStep = FORMAT == kCacheE4m3 ? 8 : G * E;
  const int lane = threadIdx.x % G, n = blockIdx.x * (256 / G) + threadIdx.x / G, j = lane * E;
  const int H = a.c.H, d = a.c.d, page_mask = (1 << a.c.page_shift) - 1;
  const long long n_slots = static_cast<long long>(a.c.num_pages) << a.c.page_shift;
  // every lane of a warp goes on: the butterfly below names all of them
  const long long slot = n < a.N ? __ldg(a.slots + n) : -1;
  if (slot >= n_slots && lane == 0) atomicOr(a.err, kErrPageRange);
  const bool on = slot >= 0 && slot < n_slots;
  const int page = on ? static_cast<int>(slot >> a.c.page_shift) : 0, inside = static_cast<int>(slot & page_mask);
  uint4 x[kRows][kPieces];
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int row = blockIdx.y * kRows + u, h = row < H ? row : row - H;
    const long long src = row < H ? n * a.k_sn + h * a.k_sh : n * a.v_sn + h * a.v_sh;
    const uint8_t *p = static_cast<const uint8_t *>(row < H ? a.k : a.v) + (src + j) * kIn;
#pragma unroll
    for (int q = 0; q < kPieces; ++q)
      x[u][q] = on && row < 2 * H && j + q * kStep < d ? __ldcs(reinterpret_cast<const uint4 *>(p + q * kStep * kIn))
                                                      : make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int u = 0; u < kRows; ++u) {
    const int row = blockIdx.y * kRows + u, h = row < H ? row : row - H;
    const bool put = on && row < 2 * H && j < d;
    const long long at = paged_row(a.c, page, row < 2 * H ? h : 0, inside);
    if (FORMAT != kCacheE4m3) {
      uint8_t *dst = static_cast<uint8_t *>(row < H ? a.c.k : a.c.v) + (at * d + j) * kIn;
#pragma unroll
      for (int q = 0; q < kPieces; ++q)
        if (put && j + q * kStep < d) *reinterpret_cast<uint4 *>(dst + q * kStep * kIn) = x[u][q];
    } else {
      const uint4 y = x[u][0], z = x[u][kPieces - 1];
      const uint32_t w[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
      // magnitudes of bf16 order as their bits, two to a word; infinities and NaN come last
      constexpr uint32_t kMag = 0x7fff7fffu;
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) top = __vimax3_u16x2(top, w[i] & kMag, w[i + 1] & kMag);
#pragma unroll
      for (int o = G / 2; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, o));
      top = max(top & 0xffffu, top >> 16);
      const bool bad = top >= 0x7f80u;
      const int e = scale_exponent(__int_as_float(static_cast<int>(top << 16)));
      // 2^-e is a normal number for e in [-100, 120]; the products are exact, and none is over 448
      const float inv = __int_as_float((127 - e) << 23);
      uint32_t code[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t c[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint32_t x2 = w[2 * i + u];
          const float2 f = make_float2(__int_as_float(static_cast<int>(x2 << 16)), __int_as_float(static_cast<int>(x2 & 0xffff0000u)));
          c[u] = __nv_cvt_float2_to_fp8x2(__fmul2_rn(f, make_float2(inv, inv)), __NV_SATFINITE, __NV_E4M3);
        }
        code[i] = bad ? 0u : __byte_perm(c[0], c[1], 0x5410);
      }
      if (e == kScaleExpMax) {  // 256 2^120 would read back as an infinity: codes stop at 240
#pragma unroll
        for (int i = 0; i < 4; ++i) code[i] = __vminu4(code[i] & 0x7f7f7f7fu, 0x77777777u) | (code[i] & 0x80808080u);
      }
      if (put) {
        *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(row < H ? a.c.k : a.c.v) + at * d + j) =
            make_uint4(code[0], code[1], code[2], code[3]);
        if (lane == 0) (row < H ? a.c.ke : a.c.ve)[at] = static_cast<uint8_t>(bad ? kScaleNan : e + kScaleBias);
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

// A block takes kGatherRows output rows (positions, all heads of k and v), 16 bytes of the cache per piece,
// kGatherUnroll pieces per thread under way at once: reading 4 sequences of up to 8192 positions, 16 heads of 128,
// back from e4m3 takes 62.7 us, 5.9 TB/s (4.5 with a position per block and two pieces).
constexpr int kGatherRows = 8, kGatherUnroll = 4;

template <int FORMAT>
__global__ void __launch_bounds__(256) cache_gather_kernel(const CacheGather a) {
  constexpr int E = FORMAT == kCacheE4m3 ? 16 : FORMAT == kCacheBf16 ? 8 : 4;  // elements of a piece
  constexpr int kOut = FORMAT == kCacheE4m3 ? 2 : 1;                           // 16-byte pieces they become
  __shared__ int s_page[kGatherRows], s_inside[kGatherRows];
  const int H = a.c.H, d = a.c.d, first = blockIdx.x * kGatherRows, rows = min(kGatherRows, a.total - first);
  if (threadIdx.x < rows) {
    // the sequence that owns row n: the last s with offsets[s] <= n
    const int n = first + threadIdx.x;
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
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(a.c.num_pages)) {
      page = -1;
      atomicOr(a.err, kErrPageRange);
    }
    s_page[threadIdx.x] = page;
    s_inside[threadIdx.x] = static_cast<int>(i & ((1 << a.c.page_shift) - 1));
  }
  __syncthreads();
  const unsigned per = d / E, row_pieces = 2u * H * per, pieces = row_pieces * rows;
  for (unsigned t0 = threadIdx.x; t0 < pieces; t0 += 256 * kGatherUnroll) {
    uint4 x[kGatherUnroll];
    float scale[kGatherUnroll];
    uint4 *dst[kGatherUnroll];
#pragma unroll
    for (int u = 0; u < kGatherUnroll; ++u) {
      const unsigned t = t0 + 256 * u;
      dst[u] = nullptr;
      x[u] = make_uint4(0, 0, 0, 0);
      if (t >= pieces) continue;
      const unsigned n = t / row_pieces, in = t - n * row_pieces, r = in / per, j = (in - r * per) * E;
      const bool is_v = r >= static_cast<unsigned>(H);
      const int h = is_v ? r - H : r, page = s_page[n];
      const long long at = (static_cast<long long>(first + n) * H + h) * d + j;
      dst[u] = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(is_v ? a.v : a.k) + at * (FORMAT == kCacheF32 ? 4 : 2));
      if (page < 0) {
        scale[u] = 1.f;
        continue;
      }
      const long long row = paged_row(a.c, page, h, s_inside[n]);
      x[u] = __ldcs(reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(is_v ? a.c.v : a.c.k) + (row * d + j) * (16 / E)));
      if (FORMAT == kCacheE4m3) scale[u] = paged_scale(__ldg((is_v ? a.c.ve : a.c.ke) + row));
    }
#pragma unroll
    for (int u = 0; u < kGatherUnroll; ++u) {
      if (dst[u] == nullptr) continue;
      if (FORMAT != kCacheE4m3) {
        __stcs(dst[u], x[u]);
        continue;
      }
      const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
      uint32_t o[8];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 f = e4m3x2_to_float2(w[q] & 0xffffu), g = e4m3x2_to_float2(w[q] >> 16);
        const __nv_bfloat162 lo = __floats2bfloat162_rn(f.x * scale[u], f.y * scale[u]);
        const __nv_bfloat162 hi = __floats2bfloat162_rn(g.x * scale[u], g.y * scale[u]);
        o[2 * q] = *reinterpret_cast<const uint32_t *>(&lo);
        o[2 * q + 1] = *reinterpret_cast<const uint32_t *>(&hi);
      }
#pragma unroll
      for (int q = 0; q < kOut; ++q) __stcs(dst[u] + q, make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]));
    }
  }
}

template <int FORMAT>
cudaError_t launch_write_f(const CacheWrite &a, cudaStream_t s) {
  const int per = a.c.d / (FORMAT == kCacheF32 ? 4 : FORMAT == kCacheBf16 ? 8 : 16);
  int G = 2;
  while (G < per && G < 32) G *= 2;
  const dim3 grid((a.N + 256 / G - 1) / (256 / G), (2 * a.c.H + write_rows(FORMAT) - 1) / write_rows(FORMAT));
  switch (G) {
    case 2: cache_write_kernel<2, FORMAT><<<grid, 256, 0, s>>>(a); break;
    case 4: cache_write_kernel<4, FORMAT><<<grid, 256, 0, s>>>(a); break;
    case 8: cache_write_kernel<8, FORMAT><<<grid, 256, 0, s>>>(a); break;
    case 16: cache_write_kernel<16, FORMAT><<<grid, 256, 0, s>>>(a); break;
    default: cache_write_kernel<FORMAT == kCacheE4m3 ? 16 : 32, FORMAT><<<grid, 256, 0, s>>>(a); break;  // e4m3: 16 at most
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_cache_write(const PagedCacheView &c, const void *k, const void *v, long long k_sn, long long k_sh,
                               long long v_sn, long long v_sh, const long long *slots, int N, unsigned *err,
                               cudaStream_t stream) {
  const CacheWrite a = {c, k, v, k_sn, k_sh, v_sn, v_sh, slots, N, err};
  if (c.format == kCacheBf16) return launch_write_f<kCacheBf16>(a, stream);
  if (c.format == kCacheE4m3) return launch_write_f<kCacheE4m3>(a, stream);
  return launch_write_f<kCacheF32>(a, stream);
}

cudaError_t launch_cache_gather(const PagedCacheView &c, const int *table, int max_pages, const int *starts,
                                const int *offsets, int S, int total, void *k, void *v, unsigned *err,
                                cudaStream_t stream) {
  const int blocks = (total + kGatherRows - 1) / kGatherRows;
  const CacheGather a = {c, table, starts, offsets, max_pages, S, total, k, v, err};
  if (c.format == kCacheBf16) cache_gather_kernel<kCacheBf16><<<blocks, 256, 0, stream>>>(a);
  else if (c.format == kCacheE4m3) cache_gather_kernel<kCacheE4m3><<<blocks, 256, 0, stream>>>(a);
  else cache_gather_kernel<kCacheF32><<<blocks, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace fem
