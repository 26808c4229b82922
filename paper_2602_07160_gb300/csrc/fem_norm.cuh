// What the forward and backward kernels of the norms share (include/fem.h, fem_norm): a row's elements in registers.
//
// TPR threads take a row, K pieces of eight elements each; a block goes through rows, as many at a time as it has threads
// for.  Where the row's length, alignment and strides allow (VEC) a piece is one or two 16-byte
// copies and neighbouring threads have neighbouring pieces; the next row's copies into shared memory are under way while
// a row is worked on, and as a thread reads back only what it copied itself, no barrier stands between.  Elsewhere
// neighbouring threads have neighbouring elements and read them when they need them: 32768 rows of 2048 of bf16, forward,
// take 112 us in pieces, 172 copied whole and read singly (a way for rows that start anywhere), 810 without copies.
#pragma once

#include <algorithm>
#include <type_traits>

#include "fem_layer.cuh"

namespace fem {

// A piece is made of runs of RUN elements that lie together: 8 where all is bf16, 4 with fp32 (16 bytes of it, so that a
// warp's accesses have no gaps), 1 where single elements are read.  Rows that lie together but start anywhere are STAGED
// (RUN_ 0): copied whole, in 16-byte pieces around them, and read as single elements.
template <int TPR_, int K_, int RUN_, int MOST_ = 256>
struct RowShape {
  static constexpr int TPR = TPR_, K = K_, RUN = RUN_ > 0 ? RUN_ : 1, ROWS = TPR_ < MOST_ ? MOST_ / TPR_ : 1, THREADS = TPR_ * ROWS;
  static constexpr bool VEC = RUN_ > 1, STAGED = RUN_ == 0, COPIED = VEC || STAGED;
  static constexpr int RUNS = VEC ? K_ * 8 / RUN : 1;  // of a thread, places to keep
  static constexpr int WARPS = TPR_ / 32;               // of a row
  static constexpr int WEIGHT = TPR_ * K * 32;          // bytes of a vector of weights

  // element j of piece i of thread `lane` of the row
  __device__ static __forceinline__ int at(int lane, int i, int j) { return (lane + (i * (8 / RUN) + j / RUN) * TPR) * RUN + j % RUN; }
};

// Sums of NV <= 4 values over a row's threads, the same bits in each.  In a warp the values are shared out as they are
// added (half the lanes go on with half of them), so that four cost little more than one; the warps' sums meet in shared
// memory, whose halves are used in turn, so that one barrier a call does, and rows of a block meet apart.
constexpr int kRowRed = 32 * 4;
template <typename S, int NV>
__device__ __forceinline__ void row_sums(float (&v)[NV], float *s_red, int &turn) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  float x;
  if constexpr (NV == 1) {
    x = v[0];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  } else {  // value 2 (lane / 16) + lane / 8 % 2 stays with a lane
    const bool hi = lane & 16, odd = lane & 8;
    float a, b = 0.f;
    if constexpr (NV == 2) {  // value lane / 16
      a = (hi ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[1], 16);
      x = a + __shfl_xor_sync(0xffffffffu, a, 8);
    } else {
      const float v3 = NV > 3 ? v[NV - 1] : 0.f;
      a = (hi ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, hi ? v[0] : v[2], 16);
      b = (hi ? v3 : v[1]) + __shfl_xor_sync(0xffffffffu, hi ? v[1] : v3, 16);
      x = (odd ? b : a) + __shfl_xor_sync(0xffffffffu, odd ? a : b, 8);
    }
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  }
  constexpr int EACH = NV == 1 ? 32 : NV == 2 ? 16 : 8;  // lanes that hold a value
  if constexpr (S::WARPS > 1) {
    float *red = s_red + turn * kRowRed;
    if (lane % EACH == 0 && lane / EACH < NV) red[(lane / EACH) * 32 + w] = x;
    bar_sync(1 + static_cast<int>(threadIdx.x) / S::TPR, S::TPR);
    const int w0 = w - w % S::WARPS;
    if constexpr (S::WARPS == 2 || S::WARPS == 4 || S::WARPS == 8) {  // lanes 8 k on add value k
      x = red[(lane >> 3) * 32 + w0 + (lane & (S::WARPS - 1))];
#pragma unroll
      for (int o = S::WARPS / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
#pragma unroll
      for (int k = 0; k < NV; ++k) v[k] = __shfl_sync(0xffffffffu, x, 8 * k);
    } else if constexpr ((S::WARPS & (S::WARPS - 1)) == 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k) v[k] = red[k * 32 + w0 + lane % S::WARPS];
#pragma unroll
      for (int o = S::WARPS / 2; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < NV; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    } else {
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        v[k] = red[k * 32 + w0];
#pragma unroll
        for (int o = 1; o < S::WARPS; ++o) v[k] += red[k * 32 + w0 + o];
      }
    }
    turn ^= 1;
  } else {
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = NV == 1 ? x : __shfl_sync(0xffffffffu, x, EACH * k);
  }
}

// Eight elements of a row in fp32, in pairs.
struct Piece {
  float2 v[4];
};
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
#define FEM_EACH_PAIR _Pragma("unroll") for (int j = 0; j < 4; ++j)

__device__ __forceinline__ void add_to(float2 &sum, const Piece &x) { FEM_EACH_PAIR sum = __fadd2_rn(sum, x.v[j]); }
__device__ __forceinline__ void add_product(float2 &sum, const Piece &x, const Piece &y) {
  FEM_EACH_PAIR sum = __ffma2_rn(x.v[j], y.v[j], sum);
}
__device__ __forceinline__ Piece times(const Piece &x, const Piece &y) {
  Piece z;
  FEM_EACH_PAIR z.v[j] = __fmul2_rn(x.v[j], y.v[j]);
  return z;
}
__device__ __forceinline__ Piece times(const Piece &x, float y) {
  Piece z;
  FEM_EACH_PAIR z.v[j] = __fmul2_rn(x.v[j], both(y));
  return z;
}
// Which of a thread's runs (VEC) or elements a row has: 1, and 0 behind its end.
template <typename S>
struct Mine {
  float f[S::VEC ? S::RUNS : 8 * S::K];
  __device__ __forceinline__ Mine(int lane, int D) {
#pragma unroll
    for (int k = 0; k < (S::VEC ? S::RUNS : 8 * S::K); ++k)
      f[k] = S::at(lane, S::VEC ? k * S::RUN / 8 : k / 8, S::VEC ? k * S::RUN % 8 : k % 8) < D ? 1.f : 0.f;
  }
  __device__ __forceinline__ bool run(int k) const { return f[k] != 0.f; }
  // x in the elements 2 j and 2 j + 1 of piece i that there are
  __device__ __forceinline__ float2 pair(float x, int i, int j) const {
    return S::VEC ? both(f[(i * 8 + 2 * j) / S::RUN] * x) : make_float2(f[(i * 8 + 2 * j) % (8 * S::K)] * x, f[(i * 8 + 2 * j + 1) % (8 * S::K)] * x);
  }
};
// x - mean where the row has elements; behind its end x is 0 and stays it.
template <typename S>
__device__ __forceinline__ void centre(Piece &x, float mean, const Mine<S> &mine, int i) {
  FEM_EACH_PAIR x.v[j] = __fadd2_rn(x.v[j], mine.pair(-mean, i, j));
}

__device__ __forceinline__ Piece unpack(const Eight<__nv_bfloat16> &x) {
  return {make_float2(bf16_lo(x.a.x), bf16_hi(x.a.x)), make_float2(bf16_lo(x.a.y), bf16_hi(x.a.y)),
          make_float2(bf16_lo(x.a.z), bf16_hi(x.a.z)), make_float2(bf16_lo(x.a.w), bf16_hi(x.a.w))};
}
__device__ __forceinline__ Piece unpack(const Eight<float> &x) {
  return {make_float2(x.a.x, x.a.y), make_float2(x.a.z, x.a.w), make_float2(x.b.x, x.b.y), make_float2(x.b.z, x.b.w)};
}
__device__ __forceinline__ void pack(Eight<__nv_bfloat16> &x, const Piece &f) {
  x.a = make_uint4(bf16_pack(f.v[0].x, f.v[0].y), bf16_pack(f.v[1].x, f.v[1].y), bf16_pack(f.v[2].x, f.v[2].y),
                   bf16_pack(f.v[3].x, f.v[3].y));
}
__device__ __forceinline__ void pack(Eight<float> &x, const Piece &f) {
  x.a = make_float4(f.v[0].x, f.v[0].y, f.v[1].x, f.v[1].y);
  x.b = make_float4(f.v[2].x, f.v[2].y, f.v[3].x, f.v[3].y);
}

__device__ __forceinline__ long long head_offset(const HeadsView &v, int d, int e) {
  const int h = e / d;
  return h * v.sh + (e - h * d);
}
// Row n = b T + t, followed from row to row.
struct RowAt {
  int b, t;
  __device__ __forceinline__ RowAt(int n, int T) : b(n / T), t(n - n / T * T) {}
  __device__ __forceinline__ void go(int rows, int T) {
    t += rows;
    if (t >= T) {
      const int q = t / T;
      b += q;
      t -= q * T;
    }
  }
};
// Element (b, t, 0, 0); where runs are copied strides are under 2^31.
template <typename S>
__device__ __forceinline__ long long heads_start(const HeadsView &v, int b, int t) {
  if (!S::VEC) return b * v.sb + t * v.st;
  const long long at = static_cast<long long>(t) * static_cast<int>(v.st);
  return b == 0 ? at : at + static_cast<long long>(b) * static_cast<int>(v.sb);
}

// One array's pieces of a row as a thread copies and reads them, a run beside its neighbours'.
template <typename S, typename T>
struct Copied {
  static constexpr int SIZE = S::RUN * sizeof(T);  // of a run: 16 bytes, 8 for bf16 beside fp32
  static constexpr int BYTES = S::K * 8 * sizeof(T) * S::THREADS;
  using Unit = std::conditional_t<SIZE == 16, uint4, uint2>;
  // `p` points at the row; run k is `off[k]` elements on, or where it is in a plain row if `off` is null.  A row that is
  // not there is one of zeros; what is behind a row's end is never written.
  __device__ static __forceinline__ void issue(uint32_t slot, const T *p, const int *off, int lane, const Mine<S> &mine, bool there) {
    static_assert(!S::VEC || SIZE == 16 || SIZE == 8, "a copy's size");
#pragma unroll
    for (int k = 0; k < (S::VEC ? S::RUNS : 0); ++k) {
      const T *src = p + (off ? off[k] : (lane + k * S::TPR) * S::RUN);
      const uint32_t to = slot + (k * S::THREADS + threadIdx.x) * SIZE;
      if (!there) zero(to);
      else if (mine.run(k)) {
        if (SIZE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(src) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(src) : "memory");
      }
    }
  }
  __device__ static __forceinline__ void zero(uint32_t to) {
    if (SIZE == 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0) : "memory");
    else asm volatile("st.shared.v2.b32 [%0], {%1, %1};" ::"r"(to), "r"(0) : "memory");
  }
  __device__ static __forceinline__ Piece read(const char *slot, int i) {
    constexpr int N = 8 / S::RUN;  // runs of a piece
    Unit u[N];
#pragma unroll
    for (int q = 0; q < N; ++q) u[q] = reinterpret_cast<const Unit *>(slot)[(i * N + q) * S::THREADS + threadIdx.x];
    return unpack(*reinterpret_cast<const Eight<T> *>(u));
  }
};

// Shared memory: `weights` bytes, where they fit beside a row, and copies of rows, of which the largest with all its arrays
// has `row` bytes: an SM's share of a block where `blocks` are to be on it.  As many rows as fit are under way, up to four.
constexpr int kMostSmem = 224 * 1024;
template <typename S>
constexpr bool keeps_weights(int row, int weights) { return S::STAGED ? S::THREADS < 1024 : S::VEC && row + weights <= kMostSmem; }
template <typename S>
constexpr int rows_smem(int row, int weights, int blocks) {
  const int share = kMostSmem / blocks - (blocks > 1 ? 2048 : 0), least = row + (keeps_weights<S>(row, weights) ? weights : 0);
  return !S::COPIED ? 0 : S::STAGED || share > least ? share : least;
}
// Zeros in the first `bytes` of shared memory behind `from`, 16 a thread, where rows leave some of it unwritten.
template <typename S>
__device__ __forceinline__ void clear_smem(char *from, int bytes, int D) {
  if (D == S::TPR * 8 * S::K) return;
  for (int i = threadIdx.x * 16; i < bytes; i += blockDim.x * 16) *reinterpret_cast<uint4 *>(from + i) = make_uint4(0, 0, 0, 0);
  __syncthreads();
}
__device__ __forceinline__ void rows_wait(int stages) {
  if (stages == 4) copy_wait<3>();
  else if (stages == 3) copy_wait<2>();
  else if (stages == 2) copy_wait<1>();
  else copy_wait<0>();
}

// Bytes of a staged row with what its pieces hold around it, and of an array in a stage.
template <typename T>
__host__ __device__ constexpr int staged_row(int D) { return (D * static_cast<int>(sizeof(T)) + 31) / 16 * 16; }
template <typename S, typename T>
__device__ __forceinline__ int stage_part(int D) {
  return S::VEC ? Copied<S, T>::BYTES : S::ROWS * staged_row<T>(D);
}
// Copies a row of D elements at p with the rest of its first 16 bytes, which are the same allocation's, and none of what
// follows its last.
template <typename S, typename T>
__device__ __forceinline__ void stage_issue(uint32_t slot, const T *p, int D, int lane) {
  const uintptr_t start = reinterpret_cast<uintptr_t>(p);
  const char *from = reinterpret_cast<const char *>(start & ~static_cast<uintptr_t>(15));
  const int bytes = static_cast<int>(start & 15) + D * static_cast<int>(sizeof(T));
  const uint32_t to = slot + threadIdx.x / S::TPR * staged_row<T>(D);
  for (int at = lane * 16; at < bytes; at += S::TPR * 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + at), "l"(from + at), "r"(min(16, bytes - at)) : "memory");
}
// Where the row at p is in shared memory.
template <typename S, typename T>
__device__ __forceinline__ const T *staged(const char *slot, const T *p, int D) {
  return reinterpret_cast<const T *>(slot + threadIdx.x / S::TPR * staged_row<T>(D) + (reinterpret_cast<uintptr_t>(p) & 15));
}

// Piece i of a row, element by element; what is past its end is 0.
template <typename S, typename T>
__device__ __forceinline__ Piece load_single(const T *row, const HeadsView *v, int d, int Dn, int lane, int i) {
  float f[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int e = S::at(lane, i, j);
    f[j] = e < Dn ? to_f32(row[v && v->sh != d ? head_offset(*v, d, e) : e]) : 0.f;
  }
  return {make_float2(f[0], f[1]), make_float2(f[2], f[3]), make_float2(f[4], f[5]), make_float2(f[6], f[7])};
}
// Piece i of the row at p, whichever way it comes; `slot` where its array's copies are.
template <typename S, typename T>
__device__ __forceinline__ Piece get_piece(const char *slot, const T *p, const HeadsView *v, int d, int D, int Dn, int lane, int i) {
  if constexpr (S::VEC) return Copied<S, T>::read(slot, i);
  else if constexpr (S::STAGED) return load_single<S, T>(staged<S, T>(slot, p, D), nullptr, 0, Dn, lane, i);
  else return load_single<S, T>(p, v, d, Dn, lane, i);
}
// Starts the copies of the row at p.
template <typename S, typename T>
__device__ __forceinline__ void issue_row(uint32_t slot, const T *p, const int *off, int D, int lane, const Mine<S> &mine, bool there) {
  if constexpr (S::VEC) Copied<S, T>::issue(slot, p, off, lane, mine, there);
  else if (there) stage_issue<S, T>(slot, p, D, lane);
}
template <typename S>
__device__ __forceinline__ void row_barrier() {
  if (S::TPR == 32) __syncwarp();
  else bar_sync(1 + static_cast<int>(threadIdx.x) / S::TPR, S::TPR);
}

// Writes piece i of a row; `off` as above (VEC), `v` the array of heads or null.
template <typename S, typename T>
__device__ __forceinline__ void store_piece(T *row, const HeadsView *v, const int *off, int d, int Dn, int lane,
                                            const Mine<S> &mine, int i, const Piece &f) {
  if constexpr (S::VEC) {
    constexpr int N = 8 / S::RUN;
    Eight<T> x;
    pack(x, f);
    const auto *u = reinterpret_cast<const typename Copied<S, T>::Unit *>(&x);
#pragma unroll
    for (int q = 0; q < N; ++q) {
      if (Dn && mine.run(i * N + q))
        *reinterpret_cast<typename Copied<S, T>::Unit *>(row + (off ? off[i * N + q] : S::at(lane, i, q * S::RUN))) = u[q];
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int e = S::at(lane, i, j);
      if (e < Dn) row[v && v->sh != d ? head_offset(*v, d, e) : e] = from_f32<T>(j % 2 ? f.v[j / 2].y : f.v[j / 2].x);
    }
  }
}

// A weight vector's elements of a piece, `none` where there is no vector; 0 past the row's end.
template <typename S>
__device__ __forceinline__ Piece load_weights(const float *w, float none, int D, int lane, int i, const Mine<S> &mine) {
  Piece f;
  if (!w) {
    FEM_EACH_PAIR f.v[j] = mine.pair(none, i, j);
  } else if constexpr (S::VEC) {
    const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
    const int e0 = S::at(lane, i, 0), e1 = S::at(lane, i, 4);
    const float4 p = e0 < D ? __ldg(reinterpret_cast<const float4 *>(w + e0)) : zero;
    const float4 q = e1 < D ? __ldg(reinterpret_cast<const float4 *>(w + e1)) : zero;
    f = {make_float2(p.x, p.y), make_float2(p.z, p.w), make_float2(q.x, q.y), make_float2(q.z, q.w)};
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = S::at(lane, i, j) < D ? __ldg(w + S::at(lane, i, j)) : 0.f;
      (j % 2 ? f.v[j / 2].y : f.v[j / 2].x) = x;
    }
  }
  return f;
}
// The same out of shared memory, in which all rows of a block share them: registers are short, and beside so much shared
// memory the L1 cache is too small for what is read row after row.
template <typename S>
__device__ __forceinline__ void keep_weights(char *slot, const Piece &f, int lane, int i) {
  float4 *p = reinterpret_cast<float4 *>(slot) + 2 * i * S::TPR + lane;
  p[0] = make_float4(f.v[0].x, f.v[0].y, f.v[1].x, f.v[1].y);
  p[S::TPR] = make_float4(f.v[2].x, f.v[2].y, f.v[3].x, f.v[3].y);
}
template <typename S>
__device__ __forceinline__ Piece kept_weights(const char *slot, int lane, int i) {
  const float4 *s = reinterpret_cast<const float4 *>(slot) + 2 * i * S::TPR + lane;
  const float4 p = s[0], q = s[S::TPR];
  return {make_float2(p.x, p.y), make_float2(p.z, p.w), make_float2(q.x, q.y), make_float2(q.z, q.w)};
}
__device__ __forceinline__ Piece weighted(const Piece &x, const Piece &w, const Piece &b) {
  Piece z;
  FEM_EACH_PAIR z.v[j] = __ffma2_rn(x.v[j], w.v[j], b.v[j]);
  return z;
}

// The sigmoid p of g and q = 1 - p = e p, e = e^(-g): no cancellation, and with e at most 2^127 no overflow (a NaN stays
// one).  Above 2^126, a gate below -87, p is flushed to 0 and with it p g and the slopes, whose limits these are: the type's
// lowest number times a p of 2^-126 would be -4.  The approximated exponential and reciprocal are off by 2 ulp and 1, the
// rounded exponent by |g| units of 2^-24, of what e is beside 1.
__device__ __forceinline__ void sigmoid(float g, float &p, float &q) {
  float t;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(t) : "f"(g * -kLog2e), "f"(127.f));
  const float e = ex2_approx(t);
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(p) : "f"(1.f + e));
  q = e * p;
}
// The gate's values and slopes; act as fem_gate_act.
__device__ __forceinline__ void gate_piece(const Piece &g, int act, Piece &value, Piece &slope) {
  value = g;
  FEM_EACH_PAIR slope.v[j] = both(1.f);
  if (act == 0) return;
  FEM_EACH_PAIR {
    float2 p, q;
    sigmoid(g.v[j].x, p.x, q.x);
    sigmoid(g.v[j].y, p.y, q.y);
    if (act == 1) {
      value.v[j] = p;
      slope.v[j] = __fmul2_rn(p, q);
    } else {
      value.v[j] = __fmul2_rn(g.v[j], p);
      slope.v[j] = __ffma2_rn(value.v[j], q, p);
    }
  }
}

// How rows are read: runs that the arrays allow to copy, rows copied whole, single elements.
enum Way { SINGLE, STAGED, PIECES };

// The shape for rows of D elements.  A thread has one piece, or two in rows up to 1024 elements with TWO, up to 2048 with
// LONG_TWO, where no threads are idle for it; WIDE of them in rows of more than 4096.  Where runs are copied a block is all
// that an SM has: ONE threads with one piece, or NARROW where a row's do not divide them, PAIR with two, FOUR in rows of
// 2048 to 4096 elements.
template <int RUN, bool TWO, bool LONG_TWO, int WIDE, int ONE, int NARROW, int PAIR, int FOUR, template <typename> class F, typename... Args>
cudaError_t with_shape(int D, Way way, Args &&...args) {
  constexpr int K = TWO ? 2 : 1, MOST = TWO ? PAIR : ONE, KL = LONG_TWO ? 2 : 1;
  if (way == SINGLE) {
    if (D <= 1024) return F<RowShape<128, 1, 1, 128>>::call(args...);
    if (D <= 4096) return F<RowShape<512, 1, 1>>::call(args...);
    return F<RowShape<1024, 2, 1>>::call(args...);
  }
  if (way == STAGED) {
    if (D <= 256) return F<RowShape<32, 1, 0>>::call(args...);
    if (D <= 1024) return F<RowShape<128, 1, 0>>::call(args...);
    if (D <= 2048) return F<RowShape<256, 1, 0>>::call(args...);
    if (D <= 5120) return F<RowShape<640, 1, 0>>::call(args...);
    return F<RowShape<1024, 1, 0>>::call(args...);
  }
  if (D <= 256) return F<RowShape<32, 1, RUN, ONE>>::call(args...);
  if (D <= 512) return F<RowShape<64 / K, K, RUN, MOST>>::call(args...);
  if (D <= 768) return F<RowShape<96, 1, RUN, NARROW>>::call(args...);
  if (D <= 1024) return F<RowShape<128 / K, K, RUN, MOST>>::call(args...);
  if (D <= 1536) return F<RowShape<192 / KL, KL, RUN, LONG_TWO ? PAIR : NARROW>>::call(args...);
  if (D <= 2048) return F<RowShape<256 / KL, KL, RUN, LONG_TWO ? PAIR : ONE>>::call(args...);
  if (D <= 4096) return F<RowShape<512, 1, RUN, FOUR>>::call(args...);
  if (D <= 8192) return F<RowShape<1024 / WIDE, WIDE, RUN>>::call(args...);
  return F<RowShape<1024, 2, RUN>>::call(args...);
}

// Rows that start anywhere, copied whole, take two to three times an aligned one's time (8192 rows of 4097 of bf16: forward
// 130 us, gradients 366, of 4096 aligned 56 and 124) and nine to ten times without (522, 1265).
//
// The way for a call whose rows of all arrays, staged, take `row` bytes: two of them have to fit beside the weights, in
// blocks of 256 threads of which `blocks` are on an SM.
inline Way way_of(const NormArgs &a, bool pieces, int row, int vectors, int blocks) {
  if (pieces) return PIECES;
  for (const HeadsView *v : {&a.y, &a.gate})
    if (v->p && a.H > 1 && v->sh != a.d) return SINGLE;
  if (a.D > 8192) return SINGLE;
  // least shared memory of a block that has a row of such a length, in the shapes above, and the rows it has at a time
  const int threads = a.D <= 2048 ? 256 : a.D <= 5120 ? 640 : 1024, rows = a.D <= 256 ? 8 : a.D <= 1024 ? 2 : 1;
  const int smem = threads == 256 ? kMostSmem / blocks - 2048 : kMostSmem, kept = threads < 1024 ? vectors * threads * 32 : 0;
  return 2 * rows * row + kept <= smem ? STAGED : SINGLE;
}

// Blocks for N rows in a shape of `rows` at a time, of which an SM holds `per_sm`: as many as there are SMs where each then
// has fewer rows at a time.  (100 rows of 2048: forward 3.1 us, gradients 8.8; in blocks of three rows 4.1 and
// 9.9.)
inline int blocks_of(int N, int rows, int per_sm, int num_sms) {
  const int few = (N + num_sms - 1) / num_sms;
  return few < rows ? (N + few - 1) / few : std::min((N + rows - 1) / rows, per_sm * num_sms);
}
inline int rows_of(int N, int rows, int blocks) { return std::min(rows, (N + blocks - 1) / blocks); }

// Whether every array allows 16-byte pieces of eight elements.
inline bool norm_pieces(const NormArgs &a, int y_size, int run) {
  auto whole = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
  bool ok = a.D % 8 == 0;
  for (const void *p : {a.x, static_cast<const void *>(a.r), static_cast<const void *>(a.z), a.dr, a.dz,
                        static_cast<const void *>(a.dx), static_cast<const void *>(a.w_post),
                        static_cast<const void *>(a.b_post), static_cast<const void *>(a.w_pre),
                        static_cast<const void *>(a.b_pre)})
    ok = ok && whole(p);
  for (const HeadsView *v : {&a.y, &a.gate, &a.dy, &a.dgate})
    if (v->p)
      ok = ok && a.d % 8 == 0 && reinterpret_cast<uintptr_t>(v->p) % (run * y_size) == 0 && v->sb % run == 0 && v->st % run == 0 && v->sh % run == 0 &&
           v->sb < (1ll << 31) && v->st < (1ll << 31) && v->sh < (1ll << 31) / a.H;
  return ok;
}

}  // namespace fem
