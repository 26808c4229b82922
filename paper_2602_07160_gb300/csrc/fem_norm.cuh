// What the forward and backward kernels of the norms share (include/fem.h, fem_norm): a row's elements in registers.
//
// TPR threads take a row, K pieces of eight elements each; a block of max(256, TPR) threads takes as many rows at a
// time.  Where the row's length, alignment and strides allow (VEC) a piece is 16 bytes of bf16 and neighbouring threads
// have neighbouring pieces; elsewhere neighbouring threads have neighbouring elements.
#pragma once

#include "fem_layer.cuh"

namespace fem {

template <int TPR_, int K_, bool VEC_>
struct RowShape {
  static constexpr int TPR = TPR_, K = K_, THREADS = TPR_ < 256 ? 256 : TPR_, ROWS = THREADS / TPR_;
  static constexpr bool VEC = VEC_;
  static constexpr int WARPS = TPR_ / 32;  // of a row

  // element j of piece i of thread `lane` of the row
  __device__ static __forceinline__ int at(int lane, int i, int j) {
    return VEC ? (lane + i * TPR) * 8 + j : lane + TPR * (i * 8 + j);
  }
};

// Sums of NV <= 4 values over a row's threads, the same bits in each.  The halves of s_red are used in turn, so that one
// barrier a call does.
constexpr int kRowRed = 32 * 4;
template <typename S, int NV>
__device__ __forceinline__ void row_sums(float (&v)[NV], float *s_red, int &turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
  if constexpr (S::WARPS > 1) {
    float *red = s_red + turn * kRowRed;
    const int w = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0)
#pragma unroll
      for (int k = 0; k < NV; ++k) red[k * 32 + w] = v[k];
    __syncthreads();
    const int from = w - w % S::WARPS + (threadIdx.x & 31) % S::WARPS;
#pragma unroll
    for (int k = 0; k < NV; ++k) v[k] = red[k * 32 + from];
#pragma unroll
    for (int o = S::WARPS / 2; o > 0; o >>= 1)
#pragma unroll
      for (int k = 0; k < NV; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    turn ^= 1;
  }
}

// Piece i of a contiguous row of D elements; what is past its end is 0.
template <typename S, typename T>
__device__ __forceinline__ void load_piece(const T *row, int D, int lane, int i, float (&f)[8]) {
  if constexpr (S::VEC) {
    Eight<T> x;
    if (S::at(lane, i, 0) < D) x.load(row + S::at(lane, i, 0));
    else x.zero();
    x.get(f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = S::at(lane, i, j) < D ? to_f32(row[S::at(lane, i, j)]) : 0.f;
  }
}
template <typename S, typename T>
__device__ __forceinline__ void store_piece(T *row, int D, int lane, int i, const float (&f)[8]) {
  if constexpr (S::VEC) {
    Eight<T> x;
    x.put(f);
    if (S::at(lane, i, 0) < D) x.store(row + S::at(lane, i, 0));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (S::at(lane, i, j) < D) row[S::at(lane, i, j)] = from_f32<T>(f[j]);
  }
}

// A weight vector's elements of a piece, `none` where there is no vector.
template <typename S>
__device__ __forceinline__ void load_weights(const float *w, int D, int lane, int i, float none, float (&f)[8]) {
  if (!w) {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = none;
  } else if constexpr (S::VEC) {
    const int e = S::at(lane, i, 0) < D ? S::at(lane, i, 0) : 0;  // past the end: any, nothing there counts
    const float4 p = __ldg(reinterpret_cast<const float4 *>(w + e));
    const float4 q = __ldg(reinterpret_cast<const float4 *>(w + e) + 1);
    f[0] = p.x, f[1] = p.y, f[2] = p.z, f[3] = p.w, f[4] = q.x, f[5] = q.y, f[6] = q.z, f[7] = q.w;
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = S::at(lane, i, j) < D ? __ldg(w + S::at(lane, i, j)) : 0.f;
  }
}

// Piece i of row (b, t) of an array of heads.
__device__ __forceinline__ long long head_offset(const HeadsView &v, int d, int e) {
  const int h = e / d;
  return h * v.sh + (e - h * d);
}
template <typename S, typename T>
__device__ __forceinline__ void load_heads(const HeadsView &v, long long row, int D, int d, int lane, int i, float (&f)[8]) {
  const T *p = static_cast<const T *>(v.p) + row;
  if constexpr (S::VEC) {
    Eight<T> x;
    if (S::at(lane, i, 0) < D) x.load(p + head_offset(v, d, S::at(lane, i, 0)));
    else x.zero();
    x.get(f);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = S::at(lane, i, j) < D ? to_f32(p[head_offset(v, d, S::at(lane, i, j))]) : 0.f;
  }
}
template <typename S, typename T>
__device__ __forceinline__ void store_heads(const HeadsView &v, long long row, int D, int d, int lane, int i, const float (&f)[8]) {
  T *p = static_cast<T *>(v.p) + row;
  if constexpr (S::VEC) {
    Eight<T> x;
    x.put(f);
    if (S::at(lane, i, 0) < D) x.store(p + head_offset(v, d, S::at(lane, i, 0)));
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (S::at(lane, i, j) < D) p[head_offset(v, d, S::at(lane, i, j))] = from_f32<T>(f[j]);
  }
}

// The gate's value and slope; act as fem_gate_act.
__device__ __forceinline__ float gate_value(float g, int act) {
  if (act == 0) return g;
  const float p = 1.f / (1.f + expf(-g));
  return act == 1 ? p : g * p;
}
__device__ __forceinline__ void gate_slope(float g, int act, float &value, float &slope) {
  value = g;
  slope = 1.f;
  if (act == 0) return;
  const float p = 1.f / (1.f + expf(-g)), q = 1.f / (1.f + expf(g));  // q = 1 - p without its cancellation
  value = act == 1 ? p : g * p;
  slope = act == 1 ? p * q : p * (1.f + g * q);
}

// Whether every array allows 16-byte pieces of eight elements.
inline bool norm_pieces(const NormArgs &a, int y_size) {
  auto whole = [](const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
  bool ok = a.D % 8 == 0;
  for (const void *p : {a.x, static_cast<const void *>(a.r), static_cast<const void *>(a.z), a.dr, a.dz,
                        static_cast<const void *>(a.dx), static_cast<const void *>(a.w_post),
                        static_cast<const void *>(a.b_post), static_cast<const void *>(a.w_pre),
                        static_cast<const void *>(a.b_pre)})
    ok = ok && whole(p);
  for (const HeadsView *v : {&a.y, &a.gate, &a.dy, &a.dgate})
    if (v->p)
      ok = ok && a.d % 8 == 0 && whole(v->p) && v->sb * y_size % 16 == 0 && v->st * y_size % 16 == 0 && v->sh * y_size % 16 == 0;
  return ok;
}

}  // namespace fem
