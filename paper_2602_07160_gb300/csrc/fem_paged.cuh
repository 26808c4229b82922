// The paged key/value cache: its layout, addressing and 8-bit format, shared by
// the kernels that write it, read it back and read over it.
//
// A cache holds k and v as [pages, H, page_size, d]: the keys of one head in one
// page are contiguous.  A sequence's position i lives in page table[i / page_size],
// row i % page_size.  In the e4m3 format every (token, head) row of d codes has
// one power-of-two scale 2^e, stored as the byte e + 127 (255: the row held a
// value that is not finite, and reads back NaN).  A code times a power of two
// is a bf16 value exactly, so a row read back, and a row handed to the tensor
// cores, lose nothing beyond the code's own rounding.
#pragma once

#include "fem_common.cuh"

namespace fem {

enum : int { kCacheBf16 = 0, kCacheE4m3 = 1, kCacheF32 = 2 };

constexpr int kScaleExpMin = -100;  // smallest scale exponent: 2^-100 times the least code is a normal bf16
constexpr int kScaleExpMax = 120;   // largest: reached by magnitudes from 2^127 up
constexpr int kScaleBias = 127;
constexpr int kScaleNan = 255;

struct PagedCacheView {
  void *k, *v;
  uint8_t *ke, *ve;  // scale exponents [pages, H, page_size] (e4m3), else null
  int format, num_pages, H, page_shift, d;
};

// One read of new tokens over the cache.  Sequence s owns the query rows
// q_off[s] .. q_off[s+1] - 1 and the positions 0 .. ctx[s] - 1.
struct PagedReadArgs {
  PagedCacheView c;
  const void *q;
  long long q_sn, q_sh;  // element strides of q over tokens and heads
  const float *beta;     // [H, d], or null: the prior mean of every channel
  const int *q_off, *ctx, *table;
  int max_pages, S, N, Hq, group, causal;
  float scale;  // 1 / sqrt(d)
  void *out;    // [N, Hq, d], q's type
  float *lse;   // [N, Hq] or null
  unsigned *err;
};

struct SeqInfo {
  int q0, n, ctx;
};

// Sequence s's rows and length, held inside the buffers whatever the device arrays say: a range that
// leaves them sets kErrPageRange and is cut.
__device__ __forceinline__ SeqInfo paged_seq(const PagedReadArgs &a, int s) {
  const int q0 = __ldg(a.q_off + s), q1 = __ldg(a.q_off + s + 1), ctx = __ldg(a.ctx + s);
  SeqInfo r;
  r.q0 = min(max(q0, 0), a.N);
  r.n = max(min(q1, a.N) - r.q0, 0);
  // (2^30 positions, more than the memory holds, keep every sum of positions in 32 bits)
  const long long cap = min(static_cast<long long>(a.max_pages) << a.c.page_shift, 1ll << 30);
  r.ctx = static_cast<int>(min(static_cast<long long>(max(ctx, 0)), cap));
  if (r.q0 != q0 || r.n != q1 - q0 || r.ctx != ctx) atomicOr(a.err, kErrPageRange);
  return r;
}

// The sequence that owns a query row, if any does: the last s with q_off[s] <= row.
__device__ __forceinline__ int paged_owner(const PagedReadArgs &a, int row) {
  int lo = 0, hi = a.S;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (__ldg(a.q_off + mid) <= row) lo = mid; else hi = mid;
  }
  return lo;
}

// Keys that row t (of n) of a sequence sees: positions 0 .. limit - 1.
__device__ __forceinline__ int paged_limit(const SeqInfo &si, int t, int causal) {
  return causal ? max(si.ctx - si.n + t + 1, 0) : si.ctx;
}

// Page of a sequence's position i, or -1 where the table names none (recorded).
__device__ __forceinline__ int paged_page(const PagedReadArgs &a, int s, int i) {
  const int p = __ldg(a.table + static_cast<long long>(s) * a.max_pages + (i >> a.c.page_shift));
  if (static_cast<unsigned>(p) >= static_cast<unsigned>(a.c.num_pages)) {
    atomicOr(a.err, kErrPageRange);
    return -1;
  }
  return p;
}

// Row index (of d elements) of position i of head h in page p.
__device__ __forceinline__ long long paged_row(const PagedCacheView &c, int p, int h, int i) {
  return ((static_cast<long long>(p) * c.H + h) << c.page_shift) + (i & ((1 << c.page_shift) - 1));
}

// 2^e of a stored scale byte (255: NaN).  The byte is biased like an fp32
// exponent, and every written byte (27 .. 247) is one of a normal number.
__device__ __forceinline__ float paged_scale(unsigned byte) {
  return byte == kScaleNan ? __int_as_float(0x7fffffff) : __int_as_float(static_cast<int>(byte << 23));
}

// Two e4m3 codes (low 16 bits of x) as floats, exactly.
__device__ __forceinline__ float2 e4m3x2_to_float2(uint32_t x) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(static_cast<uint16_t>(x)));
  return __half22float2(*reinterpret_cast<const __half2 *>(&h));
}

}  // namespace fem
