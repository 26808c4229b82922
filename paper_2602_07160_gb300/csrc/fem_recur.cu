// The gated linear recurrence h_t = e^(-s_t) h_(t-1) + w(s_t) u_t, w = 1 or 1 - e^(-s_t), and its gradients
// (include/fem.h).
//
// Bound by memory: s and u are read once and h written once (backward: s, dh, h and perhaps u read, ds and du
// written).  The time axis is what is left to share out, since channels are independent but few.  A step is an affine
// map x -> a x + b of the state, maps compose, and a stretch of steps is a map again, so a line (one sequence, one
// group of channels) is walked by a cluster of CTAs that hold the elements they read in registers:
//
//   each thread reads R steps of its channels and composes their map,
//   the maps of a CTA's threads meet in shared memory, and the maps of the CTAs in each other's,
//   each thread starts from the state before its stretch and writes its steps,
//
// while the next R steps' loads are under way.  The orders are fixed, so the same inputs give the same bits.  The
// backward pass is the same walk from the last step to the first: with m_t = a_t (dh_t + m_(t+1)) the cotangent that
// step t sends to the state before it, the map of a step is x -> a x + a dh.
#include <cooperative_groups.h>
#include <algorithm>

#include "fem_layer.cuh"

namespace fem {
namespace cg = cooperative_groups;

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

// a = e^(-s) and w = 1 - a.  For s in [0, 1/8) w = s p(s), p the cubic with p(0) = 1 that is off least over the interval
// (by 8e-8 of w; coefficients by linear programming on the condition itself), and a is 1 - w, off by 2^-25 and little
// more: the error of a decay counts as often as its horizon has steps.  Elsewhere a is 2^(-s log2 e), off by 2 ulp and,
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

template <int V>
__device__ __forceinline__ Vec<V> load_state(const float *p, long long at) {
  Vec<V> x;
#pragma unroll
  for (int i = 0; i < V; ++i) x.set(i, p[at + i]);
  return x;
}

// The map x -> a x + b of a stretch of steps.
template <int V>
struct __align__(8 * V) Map {
  Vec<V> a, b;
};

// 16 or 4 bytes from global to shared memory, of which `bytes` are read and the rest is zero.
template <int SIZE>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, int bytes) {
  if (SIZE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

// A map into another CTA's shared memory, counted by its mbarrier.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, int rank) {
  uint32_t to;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(addr), "r"(rank));
  return to;
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, const Map<1> &m) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(to),
               "r"(__float_as_uint(m.a.x)), "r"(__float_as_uint(m.b.x)), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, const Map<2> &m) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(to),
               "r"(__float_as_uint(m.a.x.x)), "r"(__float_as_uint(m.a.x.y)), "r"(__float_as_uint(m.b.x.x)),
               "r"(__float_as_uint(m.b.x.y)), "r"(bar)
               : "memory");
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

constexpr int kMostCtas = 16;  // of a cluster
constexpr int kWarps = 4;

// What the kernel needs for its size; the layout of its shared memory.
template <typename T, int V, int L, bool MEAN, bool BWD>
struct Walk {
  static constexpr int W = kWarps, R = BWD ? 8 : 16, G = 32 / L, U = G * W, CH = L * V, TR = U * R;  // G threads behind each other in a warp
  static constexpr int IN = BWD ? (MEAN ? 4 : 3) : 2, OUT = BWD ? 2 : 1;  // arrays read and written
  static constexpr int WORD = V * sizeof(T), LINE = 32 * WORD, PART = R * LINE;  // of a warp: a step of its threads, its part of a tile
  static constexpr int STAGES = 2;
  static constexpr int kRing = W * STAGES * IN * PART, kMaps = 2 * W * L * sizeof(Map<V>);
  static constexpr int kCarry = 2 * L * sizeof(Vec<V>);
  static constexpr int bytes(int ctas) { return kRing + kMaps + (ctas > 1 ? ctas * 2 * L * static_cast<int>(sizeof(Map<V>)) + 16 : kCarry); }
};

// L lanes side by side take V channels each, U threads behind each other R steps each; GRAIN bytes a copy.
template <typename T, int V, int L, bool MEAN, bool BWD, int GRAIN>
__global__ void __launch_bounds__(32 * kWarps, 4) recur_walk_kernel(const RecurArgs a, int groups, int ctas) {
  using P = Walk<T, V, L, MEAN, BWD>;
  using F = Vec<V>;
  using Wd = Word<T, V>;
  constexpr int R = P::R, G = P::G, W = P::W, S = P::STAGES;
  extern __shared__ __align__(16) char smem[];
  Map<V> *s_map = reinterpret_cast<Map<V> *>(smem + P::kRing);  // [2][W][L]: the warps' maps
  F *s_carry = reinterpret_cast<F *>(s_map + 2 * W * L);  // alone, [2][L]: the state before a tile
  Map<V> *s_cta = s_map + 2 * W * L;                      // in a cluster, [2][ctas][L]: the CTAs' maps
  const uint32_t bars = smem_u32(s_cta + 2 * ctas * L);                    // [2]: they are there

  const int line = blockIdx.x / ctas, rank = blockIdx.x % ctas, q = line / groups;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, lc = lane % L, inner = lane / L, sub = warp * G + inner;
  const int c0 = (line % groups) * P::CH, c = c0 + lc * V;
  const bool on = c < a.C;
  long long lo, hi;
  int row;
  if (!sequence(a, q, lo, hi)) {  // the same for the whole cluster
    if (threadIdx.x == 0 && rank == 0) atomicOr(a.err, kErrPageRange);
    return;
  }
  if (!state_row(a, q, row) && (a.first || a.last) && threadIdx.x == 0 && rank == 0) atomicOr(a.err, kErrPageRange);
  const long long state_at = static_cast<long long>(row) * a.C + c;
  F carry = a.first && row >= 0 && on ? load_state<V>(a.first, state_at) : F::all(0.f);
  const long long n = hi - lo, tile = static_cast<long long>(ctas) * P::TR;
  const int tiles = static_cast<int>((n + tile - 1) / tile);

  if (ctas > 1 && tiles > 0) {
    if (threadIdx.x == 0) {
      mbar_init(bars, 1);
      mbar_init(bars + 8, 1);
      fence_mbar_init();
    }
    cg::this_cluster().sync();  // every CTA is there, its barriers ready, before another sends to it
  }

  // --- this lane's part of the copies: of every array PIECES pieces of GRAIN bytes, STEP lines between them
  constexpr int PIECES = P::PART / (32 * GRAIN), PER_LINE = P::LINE / GRAIN, STEP = 32 / PER_LINE;
  const int in_line = lane % PER_LINE * GRAIN, copy_sub = warp * G + in_line / (L * P::WORD);
  const int copy_k = copy_sub * R + lane / PER_LINE, copy_c = in_line % (L * P::WORD);  // first step, byte of the channels
  const int copy_bytes = max(0, min(GRAIN, (a.C - c0) * static_cast<int>(sizeof(T)) - copy_c));
  const uint32_t ring = smem_u32(smem) + warp * (S * P::IN * P::PART) + lane * GRAIN;
  char *ring_p = smem + warp * (S * P::IN * P::PART);
  // where the piece of tile 0 is in an array whose row lags `back` behind the step's
  const long long r0 = BWD ? hi - 1 - (static_cast<long long>(rank) * P::TR + copy_k) : lo + static_cast<long long>(rank) * P::TR + copy_k;
  auto first_piece = [&](const void *base, long long st, int back) {
    return static_cast<const char *>(base) + ((r0 - back) * st + c0) * static_cast<int>(sizeof(T)) + copy_c;
  };
  constexpr int WAY = BWD ? -static_cast<int>(sizeof(T)) : static_cast<int>(sizeof(T));
  const char *src[P::IN] = {first_piece(a.s, a.s_st, 0)};
  if (BWD) {
    src[1] = first_piece(a.dh, a.dh_st, 0);
    src[2 < P::IN ? 2 : 1] = first_piece(a.h, a.h_st, 1);  // what came before a step; before the first one h0 does
    if (MEAN) src[P::IN - 1] = first_piece(a.u, a.u_st, 0);
  } else {
    src[1] = first_piece(a.u, a.u_st, 0);
  }
  char *dst[2] = {const_cast<char *>(first_piece(a.out, a.out_st, 0)), const_cast<char *>(first_piece(a.du, a.du_st, 0))};
  auto stride = [&](int slot) { return slot == 0 ? a.s_st : !BWD || (MEAN && slot == P::IN - 1) ? a.u_st : slot == 1 ? a.dh_st : a.h_st; };
  // tiles that are whole for this CTA, the step before the first one among them
  const long long whole_n = n - (BWD ? 1 : 0) - static_cast<long long>(rank + 1) * P::TR;
  const int whole = GRAIN == 2 || c0 + P::CH > a.C || whole_n < 0 ? 0 : static_cast<int>(whole_n / tile) + 1;
  auto issue = [&](int tl, int stage) {
    if (tl < whole) {
#pragma unroll
      for (int s = 0; s < P::IN; ++s)
#pragma unroll
        for (int j = 0; j < PIECES; ++j)
          copy_async<GRAIN>(ring + (stage * P::IN + s) * P::PART + 32 * j * GRAIN, src[s] + WAY * STEP * j * stride(s), GRAIN);
    } else {
      const long long k = tl * tile + static_cast<long long>(rank) * P::TR + copy_k;
#pragma unroll
      for (int s = 0; s < P::IN; ++s) {
        const long long most = BWD && s == 2 ? n - 1 : n;
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
          const char *from = src[s] + WAY * STEP * j * stride(s);
          const int bytes = k + STEP * j < most ? copy_bytes : 0;
          if constexpr (GRAIN >= 4) {
            copy_async<GRAIN>(ring + (stage * P::IN + s) * P::PART + 32 * j * GRAIN, bytes ? from : static_cast<const char *>(a.s), bytes);
          } else {
            *reinterpret_cast<uint16_t *>(ring_p + (stage * P::IN + s) * P::PART + (lane + 32 * j) * GRAIN) =
                bytes ? *reinterpret_cast<const uint16_t *>(from) : uint16_t(0);
          }
        }
      }
    }
#pragma unroll
    for (int s = 0; s < P::IN; ++s) src[s] += WAY * tile * stride(s);
  };
  auto word = [&](int stage, int slot, int i) {
    return *reinterpret_cast<const Wd *>(ring_p + (stage * P::IN + slot) * P::PART + i * P::LINE + lane * P::WORD);
  };
  for (int tl = 0; tl < S - 1; ++tl) {
    if (tl < tiles) issue(tl, tl);
    copy_commit();
  }

  int stage = 0;
  for (int tl = 0; tl < tiles; ++tl) {
    const int buf = tl & 1;
    if (tl + S - 1 < tiles) issue(tl + S - 1, stage == 0 ? S - 1 : stage - 1);  // over the tile before, which this warp has read
    copy_commit();
    copy_wait<S - 1>();
    __syncwarp();
    // the map of the thread's steps: rates of zero behind the end change nothing
    F d[R], w[R];
    Wd v[R], g[BWD ? R : 1], h[BWD ? R : 1];  // u; dh and the states before
    Map<V> m = {F::all(1.f), F::all(0.f)};
#pragma unroll
    for (int i = 0; i < R; ++i) {
      decay<V>(word(stage, 0, i).get(), d[i], w[i]);
      if (BWD) {
        g[i] = word(stage, 1, i);
        h[i] = word(stage, 2, i);
        if (MEAN) v[i] = word(stage, P::IN - 1, i);
        m.b = d[i] * (g[i].get() + m.b);
      } else {
        v[i] = word(stage, 1, i);
        if (MEAN) w[i] = w[i] * v[i].get();
        m.b = fma(d[i], m.b, MEAN ? w[i] : v[i].get());
      }
      m.a = m.a * d[i];
    }
    // with those of the threads before it in the warp
#pragma unroll
    for (int o = 1; o < G; o *= 2) {
      const Map<V> before = shift_up(m, o * L);
      if (inner >= o) m = after(before, m);
    }
    if (inner == G - 1) s_map[(buf * W + warp) * L + lc] = m;
    __syncthreads();
    F x = carry;
    if (ctas > 1) {
      if (warp == W - 1 && inner == G - 1) {  // the CTA's map, to every CTA
        Map<V> all = s_map[buf * W * L + lc];
#pragma unroll
        for (int i = 1; i < W; ++i) all = after(all, s_map[(buf * W + i) * L + lc]);
        const uint32_t to = smem_u32(s_cta + (buf * ctas + rank) * L + lc);
#pragma unroll 4
        for (int r = 0; r < ctas; ++r) send(in_cta(to, r), in_cta(bars + 8 * buf, r), all);
      }
      if (threadIdx.x == 0) mbar_arrive_expect_tx(bars + 8 * buf, ctas * L * sizeof(Map<V>));
      if (!mbar_wait(bars + 8 * buf, (tl >> 1) & 1, a.err, kErrWaitTma)) {
        copy_wait<0>();
        cg::this_cluster().sync();  // no CTA leaves while another may send to it
        return;
      }
      const Map<V> *o = s_cta + buf * ctas * L + lc;
#pragma unroll 4
      for (int r = 0; r < rank; ++r, o += L) x = fma(o->a, x, o->b);
      carry = x;
#pragma unroll 4
      for (int r = rank; r < ctas; ++r, o += L) carry = fma(o->a, carry, o->b);
    } else if (tl > 0) {
      x = s_carry[(buf ^ 1) * L + lc];
    }
    {
      const Map<V> *o = s_map + buf * W * L + lc;
#pragma unroll 4
      for (int i = 0; i < warp; ++i, o += L) x = fma(o->a, x, o->b);
    }
    if (ctas == 1 && warp == W - 1 && inner == G - 1) {  // read behind the next tile's barrier
      carry = fma(m.a, x, m.b);
      s_carry[buf * L + lc] = carry;
    }
    if (G > 1) {
      const Map<V> before = shift_up(m, L);
      if (inner > 0) x = fma(before.a, x, before.b);
    }
    // the thread's steps, over the first inputs, which its warp has read, and from there in whole lines
    char *out_p = ring_p + stage * P::IN * P::PART;
    const long long k0 = tl * tile + static_cast<long long>(rank) * P::TR;
    auto put = [&](int slot, int i, F y) { *reinterpret_cast<Wd *>(out_p + slot * P::PART + i * P::LINE + lane * P::WORD) = Wd::of(y); };
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (BWD) {
        F before = h[i].get();
        if (a.h0 && on && k0 + sub * R + i == n - 1) before = load_state<V>(a.h0, static_cast<long long>(q) * a.C + c);
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
      for (int j = 0; j < PIECES; ++j) {
        const char *from = out_p + o * P::PART + (lane + 32 * j) * GRAIN;
        char *to = dst[o] + WAY * STEP * j * st;
        if (tl < whole || (k0 + copy_k + STEP * j < n && copy_bytes == GRAIN)) {
          if (GRAIN == 16) *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(from);
          else if (GRAIN == 4) *reinterpret_cast<uint32_t *>(to) = *reinterpret_cast<const uint32_t *>(from);
          else *reinterpret_cast<uint16_t *>(to) = *reinterpret_cast<const uint16_t *>(from);
        } else if (k0 + copy_k + STEP * j < n) {
          for (int e = 0; e < copy_bytes; e += sizeof(T)) *reinterpret_cast<T *>(to + e) = *reinterpret_cast<const T *>(from + e);
        }
      }
      dst[o] += WAY * tile * st;
    }
    stage = stage == S - 1 ? 0 : stage + 1;
    __syncwarp();
  }
  if (rank == 0 && warp == W - 1 && inner == G - 1 && on && a.last && row >= 0)
#pragma unroll
    for (int i = 0; i < V; ++i) a.last[state_at + i] = carry.get(i);
}

template <typename T, int V, int L, bool MEAN, bool BWD, int GRAIN>
cudaError_t launch_walk(const RecurArgs &a, int ctas, cudaStream_t stream) {
  using P = Walk<T, V, L, MEAN, BWD>;
  auto *kernel = recur_walk_kernel<T, V, L, MEAN, BWD, GRAIN>;
  const int groups = (a.C + P::CH - 1) / P::CH;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(a.S) * groups * ctas);
  cfg.blockDim = dim3(32 * P::W);
  cfg.dynamicSmemBytes = P::bytes(ctas);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = ctas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = ctas > 1 ? 1 : 0;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, P::bytes(kMostCtas));
  if (e == cudaSuccess && ctas > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  return cudaLaunchKernelEx(&cfg, kernel, a, groups, ctas);
}

// Sequences of few steps: a thread walks V channels of one, four steps' loads under way.
constexpr int kFewSteps = 16;

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
  F x = a.first && row >= 0 ? load_state<V>(a.first, state_at) : F::all(0.f);
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
        else if (a.h0) before = load_state<V>(a.h0, static_cast<long long>(q) * a.C + c);
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

template <typename T, int V, bool MEAN, bool BWD, int GRAIN>
cudaError_t launch_rule(const RecurArgs &a, int num_sms, cudaStream_t stream) {
  if (a.T <= kFewSteps) return launch_few<T, V, MEAN, BWD>(a, stream);
  auto lines = [&](int lanes) { return static_cast<long long>(a.S) * ((a.C + lanes * V - 1) / (lanes * V)); };
  int lanes = 32;
  while (lanes > 8 && lines(lanes) * kMostCtas < 2 * num_sms) lanes /= 2;
  const long long rows = 32 / lanes * kWarps * (BWD ? 8 : 16);  // of a CTA in a tile
  const long long want = (BWD ? 4 : 7) * num_sms / lines(lanes), most = (a.T + rows - 1) / rows;
  const int ctas = static_cast<int>(std::max(1ll, std::min({want, most, static_cast<long long>(kMostCtas)})));
  if (lanes == 32) return launch_walk<T, V, 32, MEAN, BWD, GRAIN>(a, ctas, stream);
  if (lanes == 16) return launch_walk<T, V, 16, MEAN, BWD, GRAIN>(a, ctas, stream);
  return launch_walk<T, V, 8, MEAN, BWD, GRAIN>(a, ctas, stream);
}

// Whether every row starts on a multiple of `bytes`.
bool starts_at(const RecurArgs &a, int bytes, int size) {
  bool ok = true;
  for (const void *p : {a.s, a.u, a.h, a.dh, static_cast<const void *>(a.out), static_cast<const void *>(a.du)})
    ok = ok && reinterpret_cast<uintptr_t>(p) % bytes == 0;
  for (long long st : {a.s_st, a.u_st, a.h_st, a.dh_st, a.out_st, a.du_st}) ok = ok && st * size % bytes == 0;
  return ok;
}

template <bool MEAN, bool BWD>
cudaError_t launch_mean(const RecurArgs &a, int type, int num_sms, cudaStream_t stream) {
  if (type == kTypeF32)
    return starts_at(a, 16, 4) ? launch_rule<float, 1, MEAN, BWD, 16>(a, num_sms, stream)
                               : launch_rule<float, 1, MEAN, BWD, 4>(a, num_sms, stream);
  if (a.C % 2 == 0 && starts_at(a, 16, 2)) return launch_rule<__nv_bfloat16, 2, MEAN, BWD, 16>(a, num_sms, stream);
  if (a.C % 2 == 0 && starts_at(a, 4, 2)) return launch_rule<__nv_bfloat16, 2, MEAN, BWD, 4>(a, num_sms, stream);
  return launch_rule<__nv_bfloat16, 1, MEAN, BWD, 2>(a, num_sms, stream);
}

template <bool BWD>
cudaError_t launch(const RecurArgs &a, int type, bool mean, int num_sms, cudaStream_t stream) {
  return mean ? launch_mean<true, BWD>(a, type, num_sms, stream) : launch_mean<false, BWD>(a, type, num_sms, stream);
}

}  // namespace

cudaError_t launch_recur_fwd(const RecurArgs &a, int type, bool mean, int num_sms, cudaStream_t stream) {
  return launch<false>(a, type, mean, num_sms, stream);
}
cudaError_t launch_recur_bwd(const RecurArgs &a, int type, bool mean, int num_sms, cudaStream_t stream) {
  return launch<true>(a, type, mean, num_sms, stream);
}

}  // namespace fem
