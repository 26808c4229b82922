// The gated linear recurrence h_t = e^(-s_t) h_(t-1) + w(s_t) u_t, w = 1 or 1 - e^(-s_t), and its gradients
// (include/fem.h).
//
// Bound by memory: s and u are read once and h written once (backward: s, dh, h and perhaps u read, ds and du
// written).  The time axis is what is left to share out, since channels are independent but may be few.  A step is an
// affine map x -> a x + b of the state, maps compose, and a stretch of steps is a map again.  A CTA walks a line (one
// sequence, one group of channels) tile by tile:
//
//   each thread composes the map of R steps of its channels, which it keeps in registers,
//   the maps of the CTA's threads meet in shared memory,
//   each thread starts from the state before its steps and writes them,
//
// while the next tile's copies are under way.  Where there are too few lines for the GPU they are cut into chunks: a first
// kernel forms the chunks' maps, and the second one starts each chunk from the maps of those before it; s and u are read
// twice, out of L2 where they fit.  (A cluster of CTAs to a line that exchanged maps through each other's shared memory
// needed no second reading, but its step took as long as a tile's work and clusters of 16 left SMs idle: one sequence of
// 131072 steps of 256 channels took 90 us.)  The orders are fixed, so the same inputs give the same bits.  The backward
// pass is the same walk from the last step to the first: with m_t = a_t (dh_t + m_(t+1)) the cotangent that step t sends
// to the state before it, the map of a step is x -> a x + a dh.
#include <algorithm>
#include <cmath>

#include "fem_launch.h"
#include "fem_layer.cuh"

namespace fem {

namespace {

// One or two channels side by side.
template <int V>
struct Vec;
template <>
struct Vec<1> {
  float x;
  __device__ __forceinline__ static Vec all(float v) { return {v}; }
  __device__ __forceinline__ float get(int) const { return x; }
  __device__ __forceinline__ void set(int, float v) { x = v; }
};
template <>
struct Vec<2> {
  float2 x;
  __device__ __forceinline__ static Vec all(float v) { return {make_float2(v, v)}; }
  __device__ __forceinline__ float get(int i) const { return i ? x.y : x.x; }
  __device__ __forceinline__ void set(int i, float v) { (i ? x.y : x.x) = v; }
};
__device__ __forceinline__ Vec<1> fma(Vec<1> a, Vec<1> b, Vec<1> c) { return {fmaf(a.x, b.x, c.x)}; }
__device__ __forceinline__ Vec<2> fma(Vec<2> a, Vec<2> b, Vec<2> c) { return {__ffma2_rn(a.x, b.x, c.x)}; }
__device__ __forceinline__ Vec<1> operator*(Vec<1> a, Vec<1> b) { return {a.x * b.x}; }
__device__ __forceinline__ Vec<2> operator*(Vec<2> a, Vec<2> b) { return {__fmul2_rn(a.x, b.x)}; }
__device__ __forceinline__ Vec<1> operator+(Vec<1> a, Vec<1> b) { return {a.x + b.x}; }
__device__ __forceinline__ Vec<2> operator+(Vec<2> a, Vec<2> b) { return {__fadd2_rn(a.x, b.x)}; }

// V elements of type T as they lie in memory.
template <typename T, int V>
struct Word;
template <>
struct Word<__nv_bfloat16, 2> {
  uint32_t w;
  __device__ __forceinline__ Vec<2> get() const { return {make_float2(bf16_lo(w), bf16_hi(w))}; }
  __device__ __forceinline__ static Word of(Vec<2> v) { return {bf16_pack(v.x.x, v.x.y)}; }
};
template <>
struct Word<__nv_bfloat16, 1> {
  uint16_t w;
  __device__ __forceinline__ Vec<1> get() const { return {__uint_as_float(static_cast<uint32_t>(w) << 16)}; }
  __device__ __forceinline__ static Word of(Vec<1> v) { return {__bfloat16_as_ushort(__float2bfloat16_rn(v.x))}; }
};
template <>
struct Word<float, 1> {
  float w;
  __device__ __forceinline__ Vec<1> get() const { return {w}; }
  __device__ __forceinline__ static Word of(Vec<1> v) { return {v.x}; }
};
template <>
struct Word<float, 2> {
  float2 w;
  __device__ __forceinline__ Vec<2> get() const { return {w}; }
  __device__ __forceinline__ static Word of(Vec<2> v) { return {v.x}; }
};

// a = e^(-s) and w = 1 - a.  For s in [0, 1/8) w = s p(s), p the cubic with p(0) = 1 that is off least over the interval
// (by 8e-8 of w; coefficients by linear programming on the condition itself), and a is 1 - w, off by 0.5 units of 2^-24 for
// slow rates and 0.75 near 1/8: the error of a decay counts as often as its horizon has steps, which is what limits slow
// ones (a constant input's mean is 2e-4 low at s = 1e-4, 1.3e-2 at 1e-6).  Elsewhere a is 2^(-s log2 e), off by 2 ulp and,
// by its rounded exponent, s units of 2^-24.
template <int V>
__device__ __forceinline__ void decay(Vec<V> s, Vec<V> &a, Vec<V> &w) {
  using F = Vec<V>;
  F p = fma(s, F::all(-0.04012613f), F::all(0.16660093f));
  p = fma(s, p, F::all(-0.4999999f));
  p = fma(s, p, F::all(1.f));
  const F near_w = s * p, t = s * F::all(-kLog2e);
  F x;
  bool near[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    near[i] = __float_as_uint(s.get(i)) < 0x3e000000u;  // 1/8; negative numbers and NaN are above
    x.set(i, near[i] ? near_w.get(i) : ex2_approx(t.get(i)));
  }
  const F y = fma(x, F::all(-1.f), F::all(1.f));
#pragma unroll
  for (int i = 0; i < V; ++i) {
    a.set(i, near[i] ? y.get(i) : x.get(i));
    w.set(i, near[i] ? x.get(i) : y.get(i));
  }
}

// Rows lo .. hi - 1 of sequence q; false where its offsets leave the array.
__device__ __forceinline__ bool sequence(const RecurArgs &a, int q, long long &lo, long long &hi) {
  if (!a.offsets) {
    lo = static_cast<long long>(q) * a.T;
    hi = lo + a.T;
    return true;
  }
  lo = __ldg(a.offsets + q);
  hi = __ldg(a.offsets + q + 1);
  return lo >= 0 && hi >= lo && hi <= a.N;
}

// Row of the state arrays, -1: none.  false where it leaves the array.
__device__ __forceinline__ bool state_row(const RecurArgs &a, int q, int &row) {
  row = a.state_rows ? __ldg(a.state_rows + q) : q;
  if (row < 0) row = -1;
  if (row < a.num_states) return true;
  row = -1;
  return false;
}

// `there` of V channels of a state; the others are 0.
template <int V>
__device__ __forceinline__ Vec<V> load_state(const float *p, long long at, int there) {
  Vec<V> x;
#pragma unroll
  for (int i = 0; i < V; ++i) x.set(i, i < there ? p[at + i] : 0.f);
  return x;
}

// The map x -> a x + b of a stretch of steps.
template <int V>
struct __align__(8 * V) Map {
  Vec<V> a, b;
};

// 16 bytes from global to shared memory, of which `bytes` are read and the rest is zero.
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

template <int V>
__device__ __forceinline__ Vec<V> shift_up(Vec<V> v, int lanes) {
  Vec<V> o;
#pragma unroll
  for (int i = 0; i < V; ++i) o.set(i, __shfl_up_sync(0xffffffffu, v.get(i), lanes));
  return o;
}
template <int V>
__device__ __forceinline__ Map<V> shift_up(Map<V> m, int lanes) { return {shift_up(m.a, lanes), shift_up(m.b, lanes)}; }
// `first`, then `then`.
template <int V>
__device__ __forceinline__ Map<V> after(const Map<V> &first, const Map<V> &then) {
  return {first.a * then.a, fma(then.a, first.b, then.b)};
}

constexpr int kWarps = 4;  // of a CTA that has a chunk
// Steps of a thread in a tile: what registers allow, and in fp32 as many bytes of shared memory.
template <typename T, bool BWD>
constexpr int kSteps = (BWD ? 8 : 16) * 2 / static_cast<int>(sizeof(T));
template <typename T>
constexpr int kMapSteps = 16 / static_cast<int>(sizeof(T));

template <typename T, int V, int L, int W, bool MEAN, bool BWD, int GRAIN>
struct Tag;

// The chunk of a line that a CTA has: steps [k0, k0 + n) of the sequence's `all` in the order of the walk; step k is row
// lo + k, backward hi - 1 - k.
struct Chunk {
  long long lo, hi, all, k0, n;
  int line, q, c0, row, index, count;  // of the chunks that the sequence has
  bool ok;
};

// per: steps of a chunk, at least; more where a sequence is longer than the bound that the chunks were counted by.
// First all lines' first chunks: those that short sequences lack come last, when the GPU is filled evenly (seven sequences
// of 50 to 5000 steps of 1001 channels of fp32: 53 us, line after line 57).
template <bool BWD, int CH, int TR>
__device__ __forceinline__ Chunk chunk_of(const RecurArgs &a, int groups, int chunks, int per) {
  Chunk k;
  const int lines = a.S * groups;
  k.line = blockIdx.x % lines;
  k.index = blockIdx.x / lines;
  k.q = k.line / groups;
  k.c0 = k.line % groups * CH;
  k.ok = sequence(a, k.q, k.lo, k.hi);
  if (!k.ok) {
    if (threadIdx.x == 0 && k.index == 0) atomicOr(a.err, kErrPageRange);
    return k;
  }
  if (!state_row(a, k.q, k.row) && (a.first || a.last) && threadIdx.x == 0 && k.index == 0) atomicOr(a.err, kErrPageRange);
  k.all = k.hi - k.lo;
  long long each = per;
  if (each * chunks < k.all) each = ((k.all + chunks - 1) / chunks + TR - 1) / TR * TR;
  k.count = k.all == 0 ? 1 : static_cast<int>((k.all + each - 1) / each);
  k.k0 = k.index * each;
  k.n = min(each, k.all - k.k0);
  if (k.index >= k.count) k.ok = false;
  return k;
}

// A warp's copies of IN arrays into its part of shared memory: of every array a line of L V channels for each of R steps of
// its G threads, 16 bytes a copy.  Where lines do not start on 16 bytes (GRAIN 4 or 2, what they all start on) they are
// copied with the rest of their first 16 bytes, which are the same allocation's, and nothing past their end, and lie as
// far off 16 bytes in shared memory.  (Five sequences of 5000 steps of 1001 channels of fp32 105 us, eight of 2048 of bf16 38;
// in copies of 4 bytes, and in single loads, a sixth more.)  Results leave in words of GRAIN bytes.
template <typename T, int V, int L, int R, int IN, int STAGES, bool BWD, int GRAIN>
struct Ring {
  static constexpr bool AROUND = GRAIN < 16;
  static constexpr int SIZE = sizeof(T), G = 32 / L, WORD = V * SIZE, LINE = 32 * WORD;
  static constexpr int SPAN = L * WORD, PITCH = SPAN + (AROUND ? 16 : 0), PART = R * G * PITCH, BYTES = STAGES * IN * PART;
  // A lane has PIECES words of GRAIN bytes of an array and tile: SPLIT in a line, where that is longer than 32, then STEP lines on
  static constexpr int PIECES = R * LINE / (32 * GRAIN), PER_LINE = LINE / GRAIN, SPLIT = PER_LINE > 32 ? PER_LINE / 32 : 1, STEP = 32 * SPLIT / PER_LINE;
  static constexpr int AROUNDS = SPAN / 16 + 1;  // copies of a line that starts anywhere
  static constexpr int WAY = BWD ? -SIZE : SIZE;
  char *part;                          // the warp's
  uint32_t to;                         // and as an address in shared memory
  const char *src[IN][AROUND ? 1 : SPLIT];  // where this lane's first copy comes from, tile after tile; AROUND: the warp's first line
  long long st[IN], most[IN];
  uint32_t phase[IN];                  // AROUND: of this thread's first line, tile after tile
  const char *safe;                    // an address to name where nothing is read
  long long k[SPLIT], first, sub, hop; // the words' steps; the warp's first step, steps between its threads, between tiles
  int c[SPLIT], bytes[SPLIT], whole, span;  // the words' byte among the channels, bytes that there are; tiles that need no look; bytes of a line

  // first_sub: of the G threads; sub: steps between their first ones; hop: between tiles
  __device__ __forceinline__ void start(char *smem, const RecurArgs &a, const Chunk &z, int first_sub, long long sub_, long long hop_) {
    const int lane = threadIdx.x & 31;
    part = smem;
    to = smem_u32(smem);
    sub = sub_;
    hop = hop_;
    first = first_sub * sub;
    span = min(SPAN, (a.C - z.c0) * SIZE);
#pragma unroll
    for (int p = 0; p < SPLIT; ++p) {
      const int in_line = (lane + 32 * p) % PER_LINE * GRAIN;
      c[p] = in_line % SPAN;
      k[p] = first + in_line / SPAN * sub + lane / PER_LINE;
      bytes[p] = max(0, min(GRAIN, span - c[p]));
    }
    safe = reinterpret_cast<const char *>(reinterpret_cast<uintptr_t>(a.s) & ~static_cast<uintptr_t>(15));
    whole = 0;
  }
  // the row of the chunk's step k
  __device__ __forceinline__ static long long row(const Chunk &z, long long k) { return BWD ? z.hi - 1 - (z.k0 + k) : z.lo + z.k0 + k; }
  // array i, whose row lags `back` behind the step's; its steps from `most` on (of the chunk) are not there
  __device__ __forceinline__ void array(int i, const void *base, long long stride, int back, const Chunk &z, long long most_) {
    const char *from = static_cast<const char *>(base) + z.c0 * SIZE;
    if constexpr (AROUND) {
      src[i][0] = from + (row(z, first) - back) * stride * SIZE;
      phase[i] = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(src[i][0]) + (threadIdx.x & 31) / L * sub * WAY * stride);
    } else {
#pragma unroll
      for (int p = 0; p < SPLIT; ++p) src[i][p] = from + (row(z, k[p]) - back) * stride * SIZE + c[p];
    }
    st[i] = stride;
    most[i] = most_;
  }
  // tiles that lie wholly in the chunk for a warp whose steps of a tile end `end` behind its first one's
  __device__ __forceinline__ void full(const RecurArgs &a, const Chunk &z, long long end, long long most_) {
    const long long left = most_ - end;
    whole = GRAIN == 2 || z.c0 + L * V > a.C || left < 0 ? 0 : static_cast<int>(left / hop) + 1;
  }
  __device__ __forceinline__ void issue(int tl, int stage) {
    const int lane = threadIdx.x & 31;
    if constexpr (AROUND) {
#pragma unroll
      for (int s = 0; s < IN; ++s) {
        const long long left = most[s] - first - tl * hop;  // steps that there are, from the warp's first one on
#pragma unroll
        for (int j = 0; j < (R * G * AROUNDS + 31) / 32; ++j) {
          const int p = lane + 32 * j, line = p / AROUNDS, piece = p % AROUNDS * 16;
          const int step = line % G * static_cast<int>(sub) + line / G;
          if (R * G * AROUNDS % 32 != 0 && line >= R * G) break;
          const char *at = src[s][0] + static_cast<long long>(step) * (WAY * static_cast<int>(st[s]));
          const int off = static_cast<int>(reinterpret_cast<uintptr_t>(at) & 15);
          const int there = step < left ? max(0, min(16, span + off - piece)) : 0;
          copy_async(to + (stage * IN + s) * PART + line * PITCH + piece, there ? at - off + piece : safe, there);
        }
      }
    } else if (tl < whole) {
#pragma unroll
      for (int s = 0; s < IN; ++s)
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
          copy_async(to + (stage * IN + s) * PART + (32 * j + lane) * 16, src[s][j % SPLIT] + WAY * STEP * (j / SPLIT) * st[s], 16);
    } else {
#pragma unroll
      for (int s = 0; s < IN; ++s)
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
          const char *from = src[s][j % SPLIT] + WAY * STEP * (j / SPLIT) * st[s];
          const int there = k[j % SPLIT] + tl * hop + STEP * (j / SPLIT) < most[s] ? bytes[j % SPLIT] : 0;
          copy_async(to + (stage * IN + s) * PART + (32 * j + lane) * 16, there ? from : safe, there);
        }
    }
#pragma unroll
    for (int s = 0; s < IN; ++s)
#pragma unroll
      for (int p = 0; p < (AROUND ? 1 : SPLIT); ++p) src[s][p] += WAY * hop * st[s];
  }
  // this thread's channels of array `slot` at its step i
  __device__ __forceinline__ Word<T, V> word(int stage, int slot, int i) const {
    const int lane = threadIdx.x & 31;
    const char *line = part + (stage * IN + slot) * PART + (i * G + lane / L) * PITCH + lane % L * WORD;
    if constexpr (AROUND) {
      line += (phase[slot] + static_cast<uint32_t>(i * WAY * static_cast<int>(st[slot]))) & 15;
      if constexpr (WORD == 8) {  // on 4 bytes
        const float *p = reinterpret_cast<const float *>(line);
        return Word<T, V>::of({make_float2(p[0], p[1])});
      }
    }
    return *reinterpret_cast<const Word<T, V> *>(line);
  }
  // after a tile's words
  __device__ __forceinline__ void next() {
    if constexpr (AROUND)
#pragma unroll
      for (int s = 0; s < IN; ++s) phase[s] += static_cast<uint32_t>(WAY * hop * st[s]);
  }
};

// With the maps of the threads before it in the warp; the warp's own to shared memory.
template <int V, int L>
__device__ __forceinline__ void meet(Map<V> &m, Map<V> *s_map) {
  constexpr int G = 32 / L;
  const int lane = threadIdx.x & 31, inner = lane / L;
#pragma unroll
  for (int o = 1; o < G; o *= 2) {
    const Map<V> before = shift_up(m, o * L);
    if (inner >= o) m = after(before, m);
  }
  if (inner == G - 1) s_map[(threadIdx.x >> 5) * L + lane % L] = m;
}

// The maps of the chunks but the last of each line, [line][chunks][L]; in the last one's place the state before the first
// step, since the walk of the last chunk may write the new one over it before the others have begun.  No thread waits for
// another: each walks a stretch of its own.
template <typename T, int V, int L, bool MEAN, bool BWD, int GRAIN>
__global__ void __launch_bounds__(32 * kWarps, 6) recur_maps_kernel(const RecurArgs a, int groups, int chunks, int per, Map<V> *maps) {
  constexpr int W = kWarps, R = kMapSteps<T>, U = 32 / L * W, S = 3;
  using F = Vec<V>;
  using Rg = Ring<T, V, L, R, 2, S, BWD, GRAIN>;
  extern __shared__ __align__(16) char smem[];
  __shared__ Map<V> s_map[W * L];
  grid_dep_launch_dependents();
  const Chunk z = chunk_of<BWD, L * V, kSteps<T, BWD> * U>(a, groups, chunks, per);
  if (!z.ok || z.index == z.count - 1) return;  // such a chunk has a multiple of R U steps
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (z.index == 0 && a.first && threadIdx.x < L) {
    const int c = z.c0 + lane * V;
    const F x = z.row >= 0 ? load_state<V>(a.first, static_cast<long long>(z.row) * a.C + c, min(V, a.C - c)) : F::all(0.f);
    maps[(static_cast<long long>(z.line) * chunks + z.count - 1) * L + lane] = {x, x};
  }
  const long long each = z.n / U;
  Rg ring;
  ring.start(smem + warp * Rg::BYTES, a, z, warp * (32 / L), each, R);
  ring.array(0, a.s, a.s_st, 0, z, z.n);
  if (BWD) ring.array(1, a.dh, a.dh_st, 0, z, z.n);
  else ring.array(1, a.u, a.u_st, 0, z, z.n);
  const int tiles = static_cast<int>(each / R);
  ring.whole = GRAIN == 2 || z.c0 + L * V > a.C ? 0 : tiles;
  for (int tl = 0; tl < S - 1; ++tl) {
    if (tl < tiles) ring.issue(tl, tl);
    copy_commit();
  }
  Map<V> m = {F::all(1.f), F::all(0.f)};
  int stage = 0;
  for (int tl = 0; tl < tiles; ++tl) {
    if (tl + S - 1 < tiles) ring.issue(tl + S - 1, stage == 0 ? S - 1 : stage - 1);
    copy_commit();
    copy_wait<S - 1>();
    __syncwarp();
#pragma unroll
    for (int i = 0; i < R; ++i) {
      F d, w;
      decay<V>(ring.word(stage, 0, i).get(), d, w);
      const F v = ring.word(stage, 1, i).get();
      m.b = BWD ? d * (v + m.b) : fma(d, m.b, MEAN ? w * v : v);
      m.a = m.a * d;
    }
    stage = stage == S - 1 ? 0 : stage + 1;
    ring.next();
    __syncwarp();
  }
  meet<V, L>(m, s_map);
  __syncthreads();
  if (threadIdx.x >= L) return;
  Map<V> whole = s_map[lane];
#pragma unroll
  for (int i = 1; i < W; ++i) whole = after(whole, s_map[i * L + lane]);
  maps[(static_cast<long long>(z.line) * chunks + z.index) * L + lane] = whole;
}

// Walks a chunk, which is the whole line where there is one.  L lanes side by side take V channels each, 32 W / L threads
// behind each other R steps each.
template <typename T, int V, int L, int W, bool MEAN, bool BWD, int GRAIN>
struct Walk {
  static constexpr int R = kSteps<T, BWD>, G = 32 / L, U = G * W, TR = U * R;
  static constexpr int IN = BWD ? (MEAN ? 4 : 3) : 2, OUT = BWD ? 2 : 1;  // arrays read and written
  using Rg = Ring<T, V, L, R, IN, 2, BWD, GRAIN>;
  static constexpr int kMaps = 2 * W * L * sizeof(Map<V>), BYTES = W * Rg::BYTES + kMaps + 2 * L * sizeof(Vec<V>);
};

template <typename T, int V, int L, int W, bool MEAN, bool BWD, int GRAIN>
__global__ void __launch_bounds__(32 * W, 16 / W)
    recur_walk_kernel(const RecurArgs a, int groups, int chunks, int per, const Map<V> *maps) {
  using P = Walk<T, V, L, W, MEAN, BWD, GRAIN>;
  using F = Vec<V>;
  using Wd = Word<T, V>;
  using Rg = typename P::Rg;
  constexpr int R = P::R, G = P::G;
  extern __shared__ __align__(16) char smem[];
  Map<V> *s_map = reinterpret_cast<Map<V> *>(smem + W * Rg::BYTES);  // [2][W][L]: the warps' maps
  F *s_carry = reinterpret_cast<F *>(s_map + 2 * W * L);             // [2][L]: the state before a tile

  const Chunk z = chunk_of<BWD, L * V, P::TR>(a, groups, chunks, per);
  if (!z.ok) {
    if (chunks > 1) grid_dep_wait();
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lc = lane % L, inner = lane / L, sub = warp * G + inner;
  const int c = z.c0 + lc * V;
  const int there = min(V, a.C - c);  // of the thread's channels, 0 and less: none
  const bool end = warp == W - 1 && inner == G - 1;
  const long long state_at = static_cast<long long>(z.row) * a.C + c;
  const int tiles = static_cast<int>((z.n + P::TR - 1) / P::TR);

  Rg ring;
  ring.start(smem + warp * Rg::BYTES, a, z, warp * G, R, P::TR);
  ring.array(0, a.s, a.s_st, 0, z, z.n);
  if (BWD) {
    ring.array(1, a.dh, a.dh_st, 0, z, z.n);
    ring.array(2 % P::IN, a.h, a.h_st, 1, z, min(z.n, z.all - 1 - z.k0));  // what came before a step; before the first one h0 does
    if (MEAN) ring.array(P::IN - 1, a.u, a.u_st, 0, z, z.n);
  } else {
    ring.array(1, a.u, a.u_st, 0, z, z.n);
  }
  ring.full(a, z, P::TR, BWD ? min(z.n, z.all - 1 - z.k0) : z.n);
  char *dst[2][Rg::SPLIT];
#pragma unroll
  for (int p = 0; p < Rg::SPLIT; ++p) {
    const long long r = Rg::row(z, ring.k[p]);
    dst[0][p] = static_cast<char *>(a.out) + (r * a.out_st + z.c0) * static_cast<int>(sizeof(T)) + ring.c[p];
    dst[1][p] = static_cast<char *>(a.du) + (r * a.du_st + z.c0) * static_cast<int>(sizeof(T)) + ring.c[p];
  }
  if (tiles > 0) ring.issue(0, 0);
  copy_commit();

  F carry = a.first && z.row >= 0 && z.count == 1 ? load_state<V>(a.first, state_at, there) : F::all(0.f);
  if (chunks > 1) {
    grid_dep_wait();  // the maps, and whatever ran before them
    if (a.first && z.count > 1) carry = maps[(static_cast<long long>(z.line) * chunks + z.count - 1) * L + lc].a;
    if (z.index > 0) {  // the chunks before this one, a stretch of them a thread
      Map<V> m = {F::all(1.f), F::all(0.f)};
      const Map<V> *o = maps + static_cast<long long>(z.line) * chunks * L + lc;
      const int from = z.index * sub / P::U, to = z.index * (sub + 1) / P::U;
#pragma unroll 8
      for (int i = from; i < to; ++i) m = after(m, o[i * L]);
      meet<V, L>(m, s_map);
      __syncthreads();
#pragma unroll
      for (int i = 0; i < W; ++i) carry = fma(s_map[i * L + lc].a, carry, s_map[i * L + lc].b);
      __syncthreads();
    }
  }

  for (int tl = 0; tl < tiles; ++tl) {
    const int stage = tl & 1;
    if (tl + 1 < tiles) ring.issue(tl + 1, stage ^ 1);  // over the tile before, which this warp has read
    copy_commit();
    copy_wait<1>();
    __syncwarp();
    // the map of the thread's steps: rates of zero behind the end change nothing
    F d[R], w[R];
    Wd v[R], g[BWD ? R : 1], h[BWD ? R : 1];  // u; dh and the states before
    Map<V> m = {F::all(1.f), F::all(0.f)};
#pragma unroll
    for (int i = 0; i < R; ++i) {
      decay<V>(ring.word(stage, 0, i).get(), d[i], w[i]);
      if (BWD) {
        g[i] = ring.word(stage, 1, i);
        h[i] = ring.word(stage, 2 % P::IN, i);
        if (MEAN) v[i] = ring.word(stage, P::IN - 1, i);
        m.b = d[i] * (g[i].get() + m.b);
      } else {
        v[i] = ring.word(stage, 1, i);
        if (MEAN) w[i] = w[i] * v[i].get();
        m.b = fma(d[i], m.b, MEAN ? w[i] : v[i].get());
      }
      m.a = m.a * d[i];
    }
    ring.next();
    meet<V, L>(m, s_map + stage * W * L);
    __syncthreads();
    F x = tl == 0 ? carry : s_carry[(stage ^ 1) * L + lc];
    {
      const Map<V> *o = s_map + stage * W * L + lc;
#pragma unroll 4
      for (int i = 0; i < warp; ++i, o += L) x = fma(o->a, x, o->b);
    }
    if (end) {  // read behind the next tile's barrier
      carry = fma(m.a, x, m.b);
      s_carry[stage * L + lc] = carry;
    }
    if (G > 1) {
      const Map<V> before = shift_up(m, L);
      if (inner > 0) x = fma(before.a, x, before.b);
    }
    // the thread's steps, over the first inputs, which its warp has read, and from there in whole lines
    char *out_p = ring.part + stage * P::IN * Rg::PART;
    const long long k0 = static_cast<long long>(tl) * P::TR;
    auto put = [&](int slot, int i, F y) { *reinterpret_cast<Wd *>(out_p + slot * Rg::PART + i * Rg::LINE + lane * Rg::WORD) = Wd::of(y); };
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (BWD) {
        F before = h[i].get();
        if (a.h0 && z.k0 + k0 + sub * R + i == z.all - 1) before = load_state<V>(a.h0, static_cast<long long>(z.q) * a.C + c, there);
        const F total = g[i].get() + x;
        x = d[i] * total;
        put(0, i, MEAN ? x * fma(before, F::all(-1.f), v[i].get()) : x * (before * F::all(-1.f)));
        put(1, i, MEAN ? w[i] * total : total);
      } else {
        x = fma(d[i], x, MEAN ? w[i] : v[i].get());
        put(0, i, x);
      }
    }
    __syncwarp();
#pragma unroll
    for (int o = 0; o < P::OUT; ++o) {
      const long long st = o ? a.du_st : a.out_st;
#pragma unroll
      for (int j = 0; j < Rg::PIECES; ++j) {
        const char *from = out_p + o * Rg::PART + (lane + 32 * j) * GRAIN;
        constexpr int SPLIT = Rg::SPLIT;
        char *to = dst[o][j % SPLIT] + Rg::WAY * Rg::STEP * (j / SPLIT) * st;
        const bool has = tl < ring.whole || k0 + ring.k[j % SPLIT] + Rg::STEP * (j / SPLIT) < z.n;
        if (has && (tl < ring.whole || ring.bytes[j % SPLIT] == GRAIN)) {
          if (GRAIN == 16) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
          else if (GRAIN == 4) *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(from);
          else *reinterpret_cast<uint16_t *>(to) = *reinterpret_cast<const uint16_t *>(from);
        } else if (has) {
          for (int e = 0; e < ring.bytes[j % SPLIT]; e += sizeof(T)) *reinterpret_cast<T *>(to + e) = *reinterpret_cast<const T *>(from + e);
        }
      }
#pragma unroll
      for (int p = 0; p < Rg::SPLIT; ++p) dst[o][p] += Rg::WAY * P::TR * st;
    }
    __syncwarp();
  }
  if (z.index == z.count - 1 && end && a.last && z.row >= 0)
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < there) a.last[state_at + i] = carry.get(i);
}

// Sequences of few steps: a thread walks V channels of one, four steps' loads under way.
template <typename T, int V, bool MEAN, bool BWD>
__global__ void __launch_bounds__(128) recur_few_kernel(const RecurArgs a, int blocks_c) {
  using F = Vec<V>;
  using Wd = Word<T, V>;
  const int q = blockIdx.x / blocks_c, c = ((blockIdx.x % blocks_c) * 128 + threadIdx.x) * V;
  if (c >= a.C) return;
  long long lo, hi;
  int row;
  if (!sequence(a, q, lo, hi)) {
    if (c == 0) atomicOr(a.err, kErrPageRange);
    return;
  }
  if (!state_row(a, q, row) && (a.first || a.last) && c == 0) atomicOr(a.err, kErrPageRange);
  const long long state_at = static_cast<long long>(row) * a.C + c, n = hi - lo;
  auto at = [&](const void *p, long long st, long long k) {  // step k of the walk
    return reinterpret_cast<const Wd *>(static_cast<const T *>(p) + (BWD ? hi - 1 - k : lo + k) * st + c);
  };
  F x = a.first && row >= 0 ? load_state<V>(a.first, state_at, V) : F::all(0.f);
  constexpr int N = 4;
  for (long long k0 = 0; k0 < n; k0 += N) {
    Wd s[N], u[N], g[N], h[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (k0 + i >= n) break;
      s[i] = *at(a.s, a.s_st, k0 + i);
      if (MEAN || !BWD) u[i] = *at(a.u, a.u_st, k0 + i);
      if (BWD) {
        g[i] = *at(a.dh, a.dh_st, k0 + i);
        if (k0 + i + 1 < n) h[i] = *at(a.h, a.h_st, k0 + i + 1);
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (k0 + i >= n) break;
      F d, w;
      decay<V>(s[i].get(), d, w);
      Wd *out = const_cast<Wd *>(at(a.out, a.out_st, k0 + i));
      if (BWD) {
        F before = F::all(0.f);
        if (k0 + i + 1 < n) before = h[i].get();
        else if (a.h0) before = load_state<V>(a.h0, static_cast<long long>(q) * a.C + c, V);
        const F total = g[i].get() + x;
        x = d * total;
        *out = Wd::of(MEAN ? x * fma(before, F::all(-1.f), u[i].get()) : x * (before * F::all(-1.f)));
        *const_cast<Wd *>(at(a.du, a.du_st, k0 + i)) = Wd::of(MEAN ? w * total : total);
      } else {
        x = fma(d, x, MEAN ? w * u[i].get() : u[i].get());
        *out = Wd::of(x);
      }
    }
  }
  if (a.last && row >= 0)
#pragma unroll
    for (int i = 0; i < V; ++i) a.last[state_at + i] = x.get(i);
}

template <typename T, int V, bool MEAN, bool BWD>
cudaError_t launch_few(const RecurArgs &a, cudaStream_t stream) {
  const int blocks_c = (a.C + 128 * V - 1) / (128 * V);
  recur_few_kernel<T, V, MEAN, BWD><<<static_cast<unsigned>(a.S) * blocks_c, 128, 0, stream>>>(a, blocks_c);
  return cudaGetLastError();
}

// How a call's lines are shared out: `lanes` to a line's channels, CTAs of `warps`, chunks of `per` steps.  No lanes: few
// steps, a thread to a line.
struct Split {
  int lanes, warps, chunks, per;
};

// A line to a CTA where that fills the GPU, 16 warps an SM, to three fifths in its last round (64 or 32 bytes of channels
// a row where there are no more), in CTAs of 8 warps if those fill it better (tiles' last rows counted); otherwise chunks, three to four CTAs an SM.
// Eight sequences of 8192 steps of 2048 channels of bf16, 256 lines: forward 134 us in CTAs of 8 warps, 158 of 4, 195 in
// chunks; backward 243, 303, 317.  One of 131072 steps of 256 channels, 4 lines: forward 60 us in 128 chunks, 71 in 64,
// 69 in 160; backward 82, 102, 99.  By the rule and the best of the others: 4 x 8192 x 768 45 us in chunks and 76, 64 x 1024 x
// 64 11 in chunks and 12, 16 x 4096 x 1024 67 and 80, 8 x 4096 x 4096 130 and 128.  It loses where lines fill a little less than
// three fifths: 32 x 2048 x 333 73 in chunks and 55, 20 x 1030 x 1000 39 and 32.
//
// Few steps fill no tile: a thread walks them alone, 0.2 us a step, where the GPU is not filled four times over, and each
// such filling costs a walk by tiles some 2.4 us.  Forward, bf16, by threads alone and by tiles: 256 channels, 64 sequences of
// 32 steps 5.0 and 3.0 us, 512 of 16 6.5 and 11.8, of 64 19 and 15; 2048 channels, 8 of 8 2.5 and 3.0, of 16 3.3 and 3.0; 64 of 32
// 11 and 13, of 64 20 and 15; 512 of 16 19 and 79, of 64 68 and 90; 4096 channels, 64 of 16 8 and 22, 512 of 64 127 and 174.
Split split_of(const RecurArgs &a, int V, int steps, int num_sms) {
  const double rounds = static_cast<double>(a.S) * a.C / (32 * V) / (4 * num_sms);
  if (a.T <= std::min(64.0, 8 + 13 * rounds)) return {0, 0, 0, 0};
  int lanes = 32;
  while (lanes > 8 && a.C <= lanes * V / 2) lanes /= 2;
  // lines of the full length that there is work for: sequences may be shorter
  const double groups = (a.C + lanes * V - 1) / (lanes * V), lines = std::min<double>(a.S, std::max(1.0, static_cast<double>(a.N) / a.T)) * groups;
  const int tile = 32 / lanes * kWarps * steps;  // rows
  auto fill = [&](int warps) {
    const double round = 16.0 / warps * num_sms, rows = tile / kWarps * warps;
    return lines / (std::ceil(lines / round) * round) * a.T / (std::ceil(a.T / rows) * rows);
  };
  const double four = fill(4), eight = lanes == 32 ? fill(8) : 0;
  const long long per = std::max<long long>(2, static_cast<long long>(std::ceil(lines * a.T / (3.5 * num_sms * tile)))) * tile;
  // a CTA for every chunk that a sequence of the full length would have: not where many sequences are short
  const double most = 262144.0 / (a.S * groups);
  const long long chunks = std::min<long long>((a.T + per - 1) / per, static_cast<long long>(most));
  if (std::max(four, eight) >= 0.6 || chunks < 2) return {lanes, eight > four + 0.05 ? 8 : 4, 1, 0};
  const long long each = std::max(per, ((a.T + chunks - 1) / chunks + tile - 1) / tile * tile);
  return {lanes, kWarps, static_cast<int>((a.T + each - 1) / each), static_cast<int>(each)};
}

template <typename T, int V, int L, int W, bool MEAN, bool BWD, int GRAIN>
cudaError_t launch_walk(const RecurArgs &a, const Split &sp, void *ws, cudaStream_t stream) {
  using P = Walk<T, V, L, W, MEAN, BWD, GRAIN>;
  auto *kernel = recur_walk_kernel<T, V, L, W, MEAN, BWD, GRAIN>;
  const int groups = (a.C + L * V - 1) / (L * V), chunks = sp.chunks;
  const unsigned blocks = static_cast<unsigned>(a.S) * groups * chunks;
  Map<V> *maps = static_cast<Map<V> *>(ws);
  int per_sm = 0;
  cudaError_t e = resident_blocks<Tag<T, V, L, W, MEAN, BWD, GRAIN>>(kernel, 32 * W, P::BYTES, &per_sm);
  if constexpr (W == kWarps) {
    if (e == cudaSuccess && chunks > 1) {
      constexpr int ring = W * Ring<T, V, L, kMapSteps<T>, 2, 3, BWD, GRAIN>::BYTES;
      static_assert(ring <= 48 * 1024 - W * L * static_cast<int>(sizeof(Map<V>)), "no leave to ask for");
      recur_maps_kernel<T, V, L, MEAN, BWD, GRAIN><<<blocks, 32 * W, ring, stream>>>(a, groups, chunks, sp.per, maps);
      e = cudaGetLastError();
    }
  }
  if (e != cudaSuccess) return e;
  return launch_kernel(kernel, dim3(blocks), dim3(32 * W), P::BYTES, stream, chunks > 1, a, groups, chunks,
                       chunks > 1 ? sp.per : 0x7fffff00, static_cast<const Map<V> *>(maps));
}

template <typename T, int V, bool MEAN, bool BWD, int GRAIN>
cudaError_t launch_lanes(const RecurArgs &a, int num_sms, void *ws, cudaStream_t stream) {
  const Split sp = split_of(a, V, kSteps<T, BWD>, num_sms);
  if (sp.lanes == 0) return launch_few<T, sizeof(T) == 4 ? 1 : V, MEAN, BWD>(a, stream);
  if (sp.lanes == 32)
    return sp.warps == 8 ? launch_walk<T, V, 32, 8, MEAN, BWD, GRAIN>(a, sp, ws, stream)
                         : launch_walk<T, V, 32, 4, MEAN, BWD, GRAIN>(a, sp, ws, stream);
  if (sp.lanes == 16) return launch_walk<T, V, 16, 4, MEAN, BWD, GRAIN>(a, sp, ws, stream);
  return launch_walk<T, V, 8, 4, MEAN, BWD, GRAIN>(a, sp, ws, stream);
}

// Whether every row starts on a multiple of `bytes`.
bool starts_at(const RecurArgs &a, int bytes, int size) {
  bool ok = true;
  for (const void *p : {a.s, a.u, a.h, a.dh, static_cast<const void *>(a.out), static_cast<const void *>(a.du)})
    ok = ok && reinterpret_cast<uintptr_t>(p) % bytes == 0;
  for (long long st : {a.s_st, a.u_st, a.h_st, a.dh_st, a.out_st, a.du_st}) ok = ok && st * size % bytes == 0;
  return ok;
}

// Channels to a lane: two, but of bf16 one where not every row starts on a multiple of two.
int channels(const RecurArgs &a, int type) { return type == kTypeF32 || (a.C % 2 == 0 && starts_at(a, 4, 2)) ? 2 : 1; }

template <bool MEAN, bool BWD>
cudaError_t launch_mean(const RecurArgs &a, int type, int num_sms, void *ws, cudaStream_t stream) {
  if (type == kTypeF32)
    return starts_at(a, 16, 4) ? launch_lanes<float, 2, MEAN, BWD, 16>(a, num_sms, ws, stream)
                               : launch_lanes<float, 2, MEAN, BWD, 4>(a, num_sms, ws, stream);
  if (channels(a, type) == 1) return launch_lanes<__nv_bfloat16, 1, MEAN, BWD, 2>(a, num_sms, ws, stream);
  return starts_at(a, 16, 2) ? launch_lanes<__nv_bfloat16, 2, MEAN, BWD, 16>(a, num_sms, ws, stream)
                             : launch_lanes<__nv_bfloat16, 2, MEAN, BWD, 4>(a, num_sms, ws, stream);
}

template <bool BWD>
size_t workspace(const RecurArgs &a, int type, int num_sms) {
  const int V = channels(a, type);
  const Split sp = split_of(a, V, type == kTypeF32 ? kSteps<float, BWD> : kSteps<__nv_bfloat16, BWD>, num_sms);
  if (sp.chunks <= 1) return 0;
  return static_cast<size_t>(a.S) * ((a.C + sp.lanes * V - 1) / (sp.lanes * V)) * sp.chunks * sp.lanes * V * 8;
}

}  // namespace

size_t recur_workspace_bytes(const RecurArgs &a, int type, bool bwd, int num_sms) {
  return bwd ? workspace<true>(a, type, num_sms) : workspace<false>(a, type, num_sms);
}
cudaError_t launch_recur(const RecurArgs &a, int type, bool mean, bool bwd, int num_sms, void *ws, cudaStream_t stream) {
  if (bwd) return mean ? launch_mean<true, true>(a, type, num_sms, ws, stream) : launch_mean<false, true>(a, type, num_sms, ws, stream);
  return mean ? launch_mean<true, false>(a, type, num_sms, ws, stream) : launch_mean<false, false>(a, type, num_sms, ws, stream);
}

}  // namespace fem
