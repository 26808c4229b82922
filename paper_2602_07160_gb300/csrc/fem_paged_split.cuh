// How the paged read's work is split over CTAs, the value bank's coefficients,
// and the state a CTA leaves of a piece: shared by the kernels that read and
// the one that joins their pieces.
//
// Work is counted in key tiles.  An item is (sequence, key/value head, tile of
// query rows), the rows of a head's group interleaved: row r is token r / group,
// query head h group + r % group.  Items stand in a line, sequence by sequence,
// each as long as its key tiles; CTA g of G takes the stretch [g W / G, (g+1) W / G)
// of the line's W tiles.  So every CTA has the same number of tiles whatever the
// sequences' lengths, and one long sequence is spread over the whole GPU; an
// item that a stretch's end cuts is joined afterwards from its pieces.
//
// Value bank.  The read mixes the prior weights P = 2^(s - m) against a bank
// E(v), in bf16 with fp32 sums, a = sum P E / sum P.  Channel j of a sequence
// and head is read from its first kSampleKeys values v:
//   linear   (beta max|v| <= 2)  E = expm1(beta v) / beta,  o = log1p(beta a) / beta
//   shifted  (else)              E = exp(beta (v - max v)), o = max v + log(a) / beta
// Linear keeps small beta free of cancellation (beta = 0: E = v).  bf16 has
// fp32's range, so the shift needs no running update: later values may lie far
// from the sample's, and a result the ranges could have spoilt is seen in a
// (paged_out) and its row recomputed exactly.
#pragma once

#include "fem_paged.cuh"

namespace fem {

constexpr int kSampleKeys = 16;
constexpr float kLinearReach = 2.f;     // beta max|v| up to which a channel is linear
constexpr float kSmallX = 0.015625f;    // |beta v| under which expm1(beta v) is its series (x^2/6 below 2^-14)
// What the range of bf16 and fp32 may cost: a term whose weight or bank underflows is lost.  It is
// at most 2^-126 times the other factor's largest: 2^8 (P) or the largest |E| met.  While that is at
// most 2^kWideLog2, the lost terms of 2^20 keys stay under 2^-76, against a >= 2^-66.
constexpr float kWideE = 1073741824.f;        // 2^30
constexpr float kLeastA = 1.3552527e-20f;     // 2^-66
constexpr float kMostA = 1.2980742e33f;       // 2^110
constexpr float kLeastLinear = 0.25f;         // 1 + beta a: less cancels more than two bits

// E(v) = |v| < theta ? v + hb v^2 : ia 2^(b v + s) + ic
struct BankCoef {
  float b, s, ia, ic, hb, theta;
};

__device__ __forceinline__ BankCoef bank_coef(float beta, float vmax, float vabs) {
  BankCoef c;
  c.b = beta * kLog2e;
  c.hb = 0.5f * beta;
  const bool linear = !(beta * vabs > kLinearReach);
  if (linear) {
    c.s = 0.f;
    c.ia = beta > 0.f ? 1.f / beta : 0.f;
    c.ic = -c.ia;
    c.theta = beta > 0.f ? kSmallX / beta : INFINITY;
  } else {
    c.s = -c.b * vmax;
    c.ia = 1.f;
    c.ic = 0.f;
    c.theta = 0.f;
  }
  return c;
}

__device__ __forceinline__ float bank_value(const BankCoef &c, float v) {
  const float e = fmaf(ex2_approx(fmaf(c.b, v, c.s)), c.ia, c.ic);
  return fabsf(v) < c.theta ? fmaf(c.hb * v, v, v) : e;
}

// The read from a; `shift` is the coefficient s of a shifted channel, NaN of a linear one.  ok: false
// where the ranges could have spoilt it.
__device__ __forceinline__ float paged_out(float beta, float shift, float a, bool wide, bool *ok) {
  if (shift != shift) {
    const float x = beta * a;
    *ok = !wide && x > kLeastLinear - 1.f && x < kMostA && fabsf(a) < kMostA;
    return fabsf(x) < 1e-4f ? a * fmaf(-0.5f, x, 1.f) : log1pf(x) / beta;
  }
  *ok = a > (wide ? kWideE : kLeastA) && a < kMostA;
  return (log2f(a) - shift) / (beta * kLog2e);
}

// ---------------------------------------------------------------------------
// The line of work
// ---------------------------------------------------------------------------
struct SplitShape {
  int row_tile, key_tile;  // rows and keys of a tile
  int least;               // key tiles a CTA takes at least
};

// Row tiles and key tiles of a sequence; a sequence without rows has none, and
// one with rows has at least one key tile, so that its rows are written.
__device__ __forceinline__ int seq_row_tiles(const SeqInfo &si, int group, const SplitShape &sh) {
  return (si.n * group + sh.row_tile - 1) / sh.row_tile;
}
__device__ __forceinline__ int seq_key_tiles(const SeqInfo &si, const SplitShape &sh) {
  return max((si.ctx + sh.key_tile - 1) / sh.key_tile, 1);
}
__device__ __forceinline__ long long seq_tiles(const PagedReadArgs &a, const SeqInfo &si, const SplitShape &sh) {
  return static_cast<long long>(a.c.H) * seq_row_tiles(si, a.group, sh) * seq_key_tiles(si, sh);
}

// CTAs that take part, and CTA g's first tile.
__device__ __forceinline__ int split_ctas(long long W, int grid, const SplitShape &sh) {
  const long long most = (W + sh.least - 1) / sh.least;
  return static_cast<int>(most < grid ? most : grid);
}
__device__ __forceinline__ long long split_start(long long W, int G, int g) { return W * g / G; }
// the CTA that has tile x
__device__ __forceinline__ int split_owner(long long W, int G, long long x) {
  return static_cast<int>(((x + 1) * G - 1) / W);
}

template <int THREADS>
struct SplitScan {
  long long warp[THREADS / 32];
  long long prefix;
  int s;
};

// Tiles of all sequences.  All THREADS threads of the block.
template <int THREADS>
__device__ long long split_total(const PagedReadArgs &a, const SplitShape &shape, SplitScan<THREADS> &sc) {
  long long w = 0;
  for (int s = threadIdx.x; s < a.S; s += THREADS) w += seq_tiles(a, paged_seq(a, s), shape);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sc.warp[threadIdx.x >> 5] = w;
  __syncthreads();
  w = 0;
#pragma unroll
  for (int i = 0; i < THREADS / 32; ++i) w += sc.warp[i];
  return w;
}

// The sequence that holds tile x (0 <= x < total), and the tiles before that sequence.
template <int THREADS>
__device__ void split_locate(const PagedReadArgs &a, const SplitShape &shape, long long x, SplitScan<THREADS> &sc,
                             int *s_out, long long *prefix_out) {
  long long before = 0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int base = 0; base < a.S; base += THREADS) {
    const int s = base + threadIdx.x;
    const long long w = s < a.S ? seq_tiles(a, paged_seq(a, s), shape) : 0;
    long long inc = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 31) sc.warp[warp] = inc;
    __syncthreads();
    long long off = before, all = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
      if (i < warp) off += sc.warp[i];
      all += sc.warp[i];
    }
    if (x >= off + inc - w && x < off + inc) {
      sc.s = s;
      sc.prefix = off + inc - w;
    }
    before += all;
    if (x < before) break;  // the same for every thread
  }
  __syncthreads();
  *s_out = sc.s;
  *prefix_out = sc.prefix;
}

// ---------------------------------------------------------------------------
// Pieces.  CTA g's slot 0 holds the piece at its stretch's start that continues
// an item of an earlier CTA, slot 1 the piece that begins an item it does not
// end.  A piece: per row the accumulators [D] (not normalised), then per row
// {m, L} (log2 units), then the shifts [D] (NaN: linear), then whether |E| went wide.
// ---------------------------------------------------------------------------
__host__ __device__ constexpr size_t piece_floats(int rows, int D) {
  return static_cast<size_t>(rows) * D + 2 * rows + D + 4;
}

// Per output row, what is left to do after the reading kernel.
enum : uint8_t { kRowDone = 0, kRowExact = 1, kRowSplit = 2 };

struct PagedSplit {
  float *pieces;  // two slots per CTA
  uint8_t *todo;  // [N, Hq]
};

}  // namespace fem
