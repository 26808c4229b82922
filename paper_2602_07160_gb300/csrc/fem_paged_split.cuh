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
// and head goes by its first kSampleKeys values v (where those are all zero, by its
// last ones):
//   tiny     (beta max|v| <= 2^-12)  E = D v,                    o = a / D
//   linear   (beta max|v| <= 0.7)    E = expm1(beta v),          o = log1p(a) / beta
//   shifted  (else)                  E = exp(beta (v - c)),      o = c + log(a) / beta,  c about max v
// Tiny and linear keep small beta free of cancellation: E = v leaves out
// beta v^2 / 2, at most 2^-9 |v| where it is let through, and expm1 by
// subtraction is off by 2^-22, 2^-10 of the largest E.  (beta = 0 is tiny.)
// bf16 has fp32's range, so the shift needs no running update: later values may
// lie far from the sample's (at beta = 20 normal values reach E = 2^80), and a
// result that could spoil is seen in a and in its channel's largest |E|
// (paged_out), and its row recomputed exactly.
#pragma once

#include "fem_paged.cuh"

namespace fem {

constexpr int kSampleKeys = 16;
constexpr float kLinearReach = 0.7f;           // beta max|v| up to which a channel is linear: there both forms round to
                                               // 2^-9 / (1/2 beta), the linear one at v = -max|v|, the other at any v
constexpr float kTinyReach = 0.000244140625f;  // 2^-12: up to which it is tiny
// What the range of bf16 and fp32 may cost: a term whose weight or bank underflows is lost.  It is
// at most 2^-126 times the other factor's largest: 2^8 (P) or the largest |E| among the keys of such a weight.
// While that is at most 2^30, the lost terms of 2^20 keys stay under 2^-76, against a >= 2^-66; where
// it is more, the channel's class c (2^30 to 2^(30 + 6 c)) raises the bound on a by as much.  The kernel of
// many rows knows the largest |E| of every key tile; the kernel of few rows looks for it in the tiles that
// hold a weight under 2^kDeepP of the maximum at that time.  What earlier tiles, another warp or another CTA
// summed against a smaller maximum, however large its |E| or its weights, is moved to the larger one without such
// a loss (weight_root).  One
// class for a whole head would send every channel of small beta to the exact path because of one of
// large beta: reads of 4096 keys at beta 0.05 to 20 took 28 ms in place of 0.37.
constexpr float kMostShift = 32000.f;  // of a shifted channel's s (beyond it the exact path takes over)
// The bank is held times 2^-29 (of E as written above): 2^30, where class 0 ends, then sets the highest bit of
// the exponent, which the OR of a channel's E tells, at half the cost of a maximum.
constexpr int kBankShift = -29;
constexpr float kBankScale = 1.8626451e-9f;  // 2^-29
constexpr float kBankUnit = 536870912.f;     // 2^29
constexpr int kWidest = 15;                 // the class of |E| from 2^114 on, infinities and NaN
constexpr int kWideLinear = 7;              // a linear channel's last class: lost terms under 2^-34, its a from 2^-12
constexpr float kLeastA = 1.3552527e-20f;   // 2^-66
constexpr float kMostA = 1.2980742e33f;     // 2^110
constexpr float kDeepP = -100.f;            // log2 of a weight below which its term may be lost (the kernel of few rows)
constexpr float kLeastLinear = 0.125f;      // x = 1 + a of a linear channel: there a rounding of E (2^-9, as |E| < 1) is
                                            // 2^-9 / (beta x) = 2^-9 |v| / (-x log x) in the result, under 2^-7 |v|;
                                            // and v is three times the sample's largest at least, seldom even in rows of one key

// Scale D of a tiny channel, a power of two: |E| reaches 2^30 where beta |v| reaches 2^-8 (to a factor 2), or, where
// beta is under 2^-38, |v| 2^30.
__device__ __forceinline__ float tiny_scale(float beta) {
  // 2^38 times beta without its fraction
  return fmaxf(__int_as_float(__float_as_int(beta * 274877906944.f) & 0x7f800000), 1.f);
}

// The root of 2^x, x <= 0, by which a sum is multiplied twice when a maximum rises by -x: 2^x itself is 0 from 126
// on, where a sum of up to 2^127 still matters.  With the root no lower than 2^-126, what is lost or left over is
// under 2^-124 of what is held, 2^-95 of E, against a >= 2^-66.
__device__ __forceinline__ float weight_root(float x) { return ex2_approx(fmaxf(0.5f * x, -126.f)); }

// 2^-29 E(v) = 2^(b v + s) + ic + d v, with b = beta log2 e: shifted {b, -b max v rounded to a whole number, less 29, 0, 0},
// linear {b, -29, -2^-29, 0}, tiny {0, -1000, 0, 2^-29 D}
struct BankCoef {
  float b, s, ic, d;
};

// A channel whose first values are all zero (tokens without a value of their own, as at the start of many
// sequences) goes by the last kSampleKeys of those after them.  Taken as of order one, values of 0.01 at beta 2
// would be read to 2^-9 / beta, a tenth of them.  (Where the last ones are zero too, channels of padding say, order
// one it is.)
__device__ __forceinline__ int sample_last(int ctx) { return max(ctx - kSampleKeys, kSampleKeys); }
// Page of such a position, or -1; the read of its own key tile records what is not there.  (Recorded here too, the
// bank's warps of the kernel of many rows spill 300 bytes and more: a prompt of 8192 295 us, 283 without.)
__device__ __forceinline__ int sample_page(const PagedReadArgs &a, int s, int i) {
  const int p = __ldg(a.table + static_cast<long long>(s) * a.max_pages + (i >> a.c.page_shift));
  return static_cast<unsigned>(p) < static_cast<unsigned>(a.c.num_pages) ? p : -1;
}

__device__ __forceinline__ BankCoef bank_coef(float beta, float vmax, float vabs) {
  const float x = beta * (vabs > 0.f ? vabs : 1.f);
  BankCoef c;
  c.b = beta * kLog2e;
  c.s = kBankShift;
  c.ic = -kBankScale;
  c.d = 0.f;
  if (x <= kTinyReach) {
    c.b = 0.f;
    c.s = -1000.f;
    c.ic = 0.f;
    c.d = tiny_scale(beta) * kBankScale;
  } else if (!(x <= kLinearReach)) {
    c.s = fminf(fmaxf(-rintf(c.b * vmax), -kMostShift), kMostShift) + kBankShift;
    c.ic = 0.f;
  }
  return c;
}
// The channel's kind, and a shifted one's s (a whole number, of E), in one float: NaN linear, infinity tiny.
__device__ __forceinline__ float bank_kind(const BankCoef &c) {
  return c.d != 0.f ? INFINITY : c.ic == 0.f ? c.s - kBankShift : __int_as_float(0x7fffffff);
}

// The same in 16 bits.
__device__ __forceinline__ short kind_pack(float kind) {
  return kind == INFINITY ? 32766 : kind != kind ? 32767 : static_cast<short>(kind);
}
__device__ __forceinline__ float kind_unpack(short k) {
  return k == 32766 ? INFINITY : k == 32767 ? __int_as_float(0x7fffffff) : static_cast<float>(k);
}

// The class of a largest |E| by the exponent field of what is held.
__device__ __forceinline__ int wide_class(int field) {
  return field < 128 ? 0 : min(kWidest, 1 + (field - 128) / 6);
}

// 2^-29 E of two values; coefficients of both
__device__ __forceinline__ float2 bank_pair(const float2 b, const float2 s, const float2 ic, const float2 d, const float2 v,
                                            bool tiny = true) {
  const float2 x = __ffma2_rn(b, v, s);
  const float2 e = __fadd2_rn(make_float2(ex2_approx(x.x), ex2_approx(x.y)), ic);
  return tiny ? __ffma2_rn(d, v, e) : e;
}

// The read from a, o = |a| g < 2^-6 and w != 0 ? a w (1 - g (a/2 - a^2/3)) : lg2(a + g) z + y:
//   tiny {g 0, w 1/D}, linear {g 1, w 1/beta, z 1/b, y 0}, shifted {g 0, w 0, z 1/b, y -s/b}
// (log1p's series is good to 2^-18 where it is used, lg2's 2^-22 to 2^-16 elsewhere.)  It stands when
// lo < a + g < 2^110; otherwise the ranges could have spoilt it.  No branch: the kinds of a row's
// channels are mixed.
struct OutCoef {
  float g, z, y, w, lo;
};
__device__ __forceinline__ OutCoef out_coef(float beta, float kind, int wide) {
  const float ib = rcp_approx(beta * kLog2e);
  OutCoef c;
  const bool tiny = kind == INFINITY, linear = kind != kind;
  c.g = linear ? 1.f : 0.f;
  c.z = tiny ? 0.f : ib;
  c.y = tiny || linear ? 0.f : -kind * ib;
  c.w = tiny ? 1.f / tiny_scale(beta) : linear ? ib * kLog2e : 0.f;
  // a tiny channel's |E| over 2^30 says that it is none
  const float least = kLeastA * __int_as_float((127 + 6 * wide) << 23);
  c.lo = tiny ? (wide ? INFINITY : -kMostA) : linear ? (wide > kWideLinear ? INFINITY : kLeastLinear) : (wide == kWidest ? INFINITY : least);
  return c;
}
__device__ __forceinline__ float paged_out(const OutCoef &c, float a, bool *ok) {
  const float x = a + c.g;
  *ok = x > c.lo && x < kMostA;
  const float log = fmaf(lg2_approx(x), c.z, c.y);
  const float series = a * c.w * fmaf(c.g * a, fmaf(a, 1.f / 3.f, -0.5f), 1.f);
  return fabsf(a) * c.g < 0.015625f && c.w != 0.f ? series : log;
}

// ---------------------------------------------------------------------------
// The line of work
// ---------------------------------------------------------------------------
struct SplitShape {
  int row_tile, key_shift;  // rows of a tile, log2 of its keys
  int tok;                  // tokens of a row tile (whole tokens), or 0: rows packed without regard to tokens
  int least;                // key tiles a CTA takes at least
  int fixed;                // what beginning an item costs, in key tiles: the line counts them before its tiles
  int whole;                // items of up to so many key tiles are not cut: the CTA that has their start has them
};

// Row tiles of a sequence, for each of its heads; a sequence without rows has none.
__host__ __device__ __forceinline__ int seq_row_tiles(const SeqInfo &si, int group, const SplitShape &sh) {
  return sh.tok ? (si.n + sh.tok - 1) / sh.tok : (si.n * group + sh.row_tile - 1) / sh.row_tile;
}
// Key tiles of row tile r: those its last row sees (tiles of whole tokens), or all.  At least one, so
// that rows which see nothing are written.
__host__ __device__ __forceinline__ int row_key_tiles(const SeqInfo &si, int r, int causal, const SplitShape &sh) {
  int keys = si.ctx;
  if (sh.tok && causal) {
    const int last = (r + 1) * sh.tok;
    keys = si.ctx - si.n + (last < si.n ? last : si.n);
  }
  const int tiles = (keys + (1 << sh.key_shift) - 1) >> sh.key_shift;
  return tiles > 1 ? tiles : 1;
}
// Key tiles of row tiles 0 .. R - 1 of one head (R at most `all`, the sequence's), and the items' fixed costs.
__host__ __device__ __forceinline__ long long head_key_tiles(const SeqInfo &si, int R, int all, int causal,
                                                             const SplitShape &sh) {
  if (R <= 0) return 0;
  if (!(sh.tok && causal)) return static_cast<long long>(R) * (row_key_tiles(si, 0, 0, sh) + sh.fixed);
  // sum of ceil((c + i tok) / T), i = 0 .. n - 1, over the tiles of tok whole tokens; the sequence's
  // last tile may hold fewer
  long long sum = static_cast<long long>(R) * sh.fixed;
  int n = R, i0 = 0;
  if (R == all) {
    sum += row_key_tiles(si, R - 1, causal, sh);
    n = R - 1;
  }
  const int base = si.ctx - si.n, step = sh.tok, shift = sh.key_shift, T = 1 << shift;
  if (base + step < 1) {  // leading tiles that see nothing count one each
    i0 = -base / step;
    if (i0 > n) i0 = n;
    while (i0 < n && base + (i0 + 1) * step < 1) ++i0;
    sum += i0;
  }
  n -= i0;
  // ceil(x / T) = floor((x + T - 1) / T); floor sum = (sum of x - sum of x mod T) / T.  The residues have
  // the period P = T / gcd(tok, T), a full period's being g times 0 .. P - 1 plus b mod g (T is a power
  // of two, and so are g and P).
  const long long b = static_cast<long long>(base) + static_cast<long long>(i0 + 1) * step + T - 1;
  int lg = 0;
  while (lg < shift && !((step >> lg) & 1)) ++lg;
  const int gcd = 1 << lg, P = T >> lg, rem = n & (P - 1);
  const long long full = n >> (shift - lg);
  long long res = full * (static_cast<long long>(P) * (b & (gcd - 1)) + static_cast<long long>(gcd) * P * (P - 1) / 2);
  for (int i = 0; i < rem; ++i) res += (b + static_cast<long long>(i) * step) & (T - 1);
  const long long x = n * b + static_cast<long long>(step) * n * (n - 1) / 2;
  return sum + ((x - res) >> shift);
}
__device__ __forceinline__ long long seq_tiles(const PagedReadArgs &a, const SeqInfo &si, const SplitShape &sh) {
  const int R = seq_row_tiles(si, a.group, sh);
  return a.c.H * head_key_tiles(si, R, R, a.causal, sh);
}

// CTA g's first tile of W (below 2^31) split over G: floor(W g / G).
__host__ __device__ __forceinline__ unsigned split_start(unsigned W, unsigned G, unsigned g) {
  return W / G * g + W % G * g / G;
}
// The CTA that has tile x.
__host__ __device__ __forceinline__ int split_owner(unsigned W, unsigned G, unsigned x) {
  return static_cast<int>((static_cast<unsigned long long>(x + 1) * G - 1) / W);
}

// An item and the key tiles kt0 .. kt1 - 1 of it (kt_all in the whole item).
struct SplitSeg {
  SeqInfo si;
  int s, h, r;  // sequence, head, row tile
  int kt0, kt1, kt_all;
  unsigned x_end;  // the line's tile after the item's last
};

// Walks a CTA's stretch, item by item.
struct SplitWalk {
  unsigned x, left;  // next tile, tiles to go
  unsigned W, G;     // the line's tiles, CTAs that take part
  SeqInfo si;
  int s, h, r, R;
  int at;  // the next tile's place in the item's stretch of the line (its fixed cost, then its key tiles)
  __device__ __forceinline__ bool next(const PagedReadArgs &a, const SplitShape &sh, SplitSeg &g) {
    while (left) {
      g.si = si;
      g.s = s;
      g.h = h;
      g.r = r;
      g.kt_all = row_key_tiles(si, r, a.causal, sh);
      const unsigned rest = g.kt_all + sh.fixed - at, take = min(rest, left);
      g.kt0 = max(at - sh.fixed, 0);
      g.kt1 = at + static_cast<int>(take) - sh.fixed;
      if (g.kt_all <= sh.whole) {
        g.kt0 = 0;
        g.kt1 = at == 0 ? g.kt_all : 0;
      }
      g.x_end = x + rest;
      x += take;
      left -= take;
      at = 0;
      if (left && ++r == R) {
        r = 0;
        if (++h == a.c.H) {
          h = 0;
          do {  // the next sequence with rows: there is one, as tiles are left
            si = paged_seq(a, ++s);
            R = seq_row_tiles(si, a.group, sh);
          } while (R == 0);
        }
      }
      // else the stretch ends inside the item's fixed cost (the next CTA begins it), or begins inside an item
      // that is not cut
      if (g.kt1 > 0) return true;
    }
    return false;
  }
};

template <int THREADS>
struct SplitScan {
  long long warp[THREADS / 32];
  int s, h, r, at;
};

// The stretch of CTA `cta` of a grid of `grid`; false where it has none.  All THREADS threads of the block.
template <int THREADS>
__device__ bool split_begin(const PagedReadArgs &a, const SplitShape &shape, int cta, int grid, SplitScan<THREADS> &sc,
                            SplitWalk &walk) {
  constexpr int kWarps = THREADS / 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // inclusive sums of the tiles of sequences base .. base + THREADS - 1 (thread = sequence)
  auto scan = [&](long long w, long long &all) {
    long long inc = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    __syncthreads();
    if (lane == 31) sc.warp[warp] = inc;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < warp) inc += sc.warp[i];
      all += sc.warp[i];
    }
    return inc;
  };
  SeqInfo si = {0, 0, 0};
  if (threadIdx.x < a.S) si = paged_seq(a, threadIdx.x);
  long long w = seq_tiles(a, si, shape), all, W;
  long long inc = scan(w, all);
  W = all;
  for (int base = THREADS; base < a.S; base += THREADS) {  // more sequences than threads
    const int s = base + threadIdx.x;
    scan(s < a.S ? seq_tiles(a, paged_seq(a, s), shape) : 0, all);
    W += all;
  }
  if (W <= 0) return false;
  if (W >= (1ll << 31)) {  // hours of work: lengths that are not meant
    if (threadIdx.x == 0) atomicOr(a.err, kErrPageRange);
    return false;
  }
  const long long most = (W + shape.least - 1) / shape.least;
  walk.W = static_cast<unsigned>(W);
  walk.G = static_cast<unsigned>(most < grid ? most : grid);
  if (cta >= static_cast<int>(walk.G)) return false;
  walk.x = split_start(walk.W, walk.G, cta);
  walk.left = split_start(walk.W, walk.G, cta + 1) - walk.x;
  long long before = 0;
  int s = threadIdx.x;
  for (int base = 0;; base += THREADS) {
    if (base > 0) {
      s = base + threadIdx.x;
      si = {0, 0, 0};
      if (s < a.S) si = paged_seq(a, s);
      w = seq_tiles(a, si, shape);
      inc = scan(w, all) + before;
    } else if (a.S > THREADS) {
      inc = scan(w, all);  // all: of this round again
    }
    if (walk.x >= inc - w && walk.x < inc) {
      // this thread's sequence holds the stretch's first tile
      const int R = seq_row_tiles(si, a.group, shape);
      const unsigned per = static_cast<unsigned>(head_key_tiles(si, R, R, a.causal, shape));
      const unsigned local = static_cast<unsigned>(walk.x - (inc - w));
      const unsigned h = local / per, in = local - h * per;
      int lo = 0, hi = R;  // the last row tile whose key tiles begin at or before `in`
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (head_key_tiles(si, mid, R, a.causal, shape) <= in) lo = mid; else hi = mid;
      }
      sc.s = s;
      sc.h = static_cast<int>(h);
      sc.r = lo;
      sc.at = static_cast<int>(in - head_key_tiles(si, lo, R, a.causal, shape));
    }
    before += all;
    if (walk.x < before) break;  // the same for every thread
  }
  __syncthreads();
  walk.s = sc.s;
  walk.h = sc.h;
  walk.r = sc.r;
  walk.at = sc.at;
  walk.si = paged_seq(a, walk.s);
  walk.R = seq_row_tiles(walk.si, a.group, shape);
  return true;
}

// ---------------------------------------------------------------------------
// Pieces.  CTA g's slot 0 holds the piece at its stretch's start that continues
// an item of an earlier CTA, slot 1 the piece that begins an item it does not
// end.  A piece: the rows' accumulators [rows][D] (not normalised), in groups of
// 8 rows with 4 channels of the 8 side by side (128 bytes), so that a warp whose
// lanes are rows and one whose lanes are channels both write full lines; then
// per row {m, L} (log2 units), then the channels' kinds [D] and classes of |E|
// [D], then four numbers whose sum is 0 where every class is.
// ---------------------------------------------------------------------------
// Channels 4 c4 .. of row `row`, in floats.
__host__ __device__ constexpr size_t piece_at(int row, int c4, int D) {
  return (static_cast<size_t>(row >> 3) * (D / 4) + c4) * 32 + (row & 7) * 4;
}
__host__ __device__ constexpr size_t piece_floats(int rows, int D) {
  return (static_cast<size_t>(rows) * D + 2 * rows + 2 * D + 4 + 31) / 32 * 32;  // full lines
}
// Where the kinds, the classes and the four numbers begin.
__host__ __device__ constexpr int piece_kinds(int rows, int D) { return rows * D + 2 * rows; }
__host__ __device__ constexpr int piece_classes(int rows, int D) { return rows * D + 2 * rows + D; }
__host__ __device__ constexpr int piece_wide(int rows, int D) { return rows * D + 2 * rows + 2 * D; }

// What a CTA leaves to the kernel that follows: the item it begins and does not end (n pieces, of
// this CTA and the n - 1 after it; none: 0), and whether rows that it finished need the exact path.
struct __align__(32) SplitRecord {
  int n;
  int s, h;        // the item's sequence and head
  int row0, rows;  // its first row among the sequence's (token * group + head of the group), its rows
  int any_exact;
};

struct PagedSplit {
  float *pieces;         // two slots per CTA
  SplitRecord *records;  // per CTA
  uint8_t *exact;        // [N, Hq]: 1 where a finished row needs the exact path (read where a record says so)
};

}  // namespace fem
