// The gated linear recurrence h_t = e^(-s_t) h_(t-1) + w(s_t) u_t, w = 1 or 1 - e^(-s_t), and its gradients
// (include/fem.h), a thread for each channel of each sequence.
#include "fem_layer.cuh"

namespace fem {

namespace {

// w = 1 - e^(-s) and a = e^(-s).  Near zero w is the Taylor polynomial (the term left out is under 2e-9 of it at 1/4)
// and a is 1 - w, off by at most 2^-25: a decay's error counts as often as its horizon has steps.
__device__ __forceinline__ void decay(float s, float &a, float &w) {
  const float t =
      s * (1.f - s * (0.5f - s * (1.f / 6.f - s * (1.f / 24.f - s * (1.f / 120.f - s * (1.f / 720.f - s * (1.f / 5040.f)))))));
  const float e = expf(-s);
  const bool near = fabsf(s) < 0.25f;
  w = near ? t : 1.f - e;
  a = near ? 1.f - t : e;
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

template <typename T, bool MEAN, bool BWD>
__global__ void __launch_bounds__(128) recur_serial_kernel(const RecurArgs a, int blocks_c) {
  const int q = blockIdx.x / blocks_c, c = (blockIdx.x % blocks_c) * 128 + threadIdx.x;
  if (c >= a.C) return;
  long long lo, hi;
  int row;
  if (!sequence(a, q, lo, hi)) {
    if (c == 0) atomicOr(a.err, kErrPageRange);
    return;
  }
  if (!state_row(a, q, row) && (a.first || a.last) && c == 0) atomicOr(a.err, kErrPageRange);
  const T *s = static_cast<const T *>(a.s) + c, *u = static_cast<const T *>(a.u) + c;
  float x = a.first && row >= 0 ? a.first[static_cast<long long>(row) * a.C + c] : 0.f;
  T *out = static_cast<T *>(a.out) + c;
  if (!BWD) {
    for (long long t = lo; t < hi; ++t) {
      float d, w;
      decay(to_f32(s[t * a.s_st]), d, w);
      const float v = to_f32(u[t * a.u_st]);
      x = fmaf(d, x, MEAN ? w * v : v);
      out[t * a.out_st] = from_f32<T>(x);
    }
  } else {
    const T *h = static_cast<const T *>(a.h) + c, *dh = static_cast<const T *>(a.dh) + c;
    T *du = static_cast<T *>(a.du) + c;
    const float h0 = a.h0 ? a.h0[static_cast<long long>(q) * a.C + c] : 0.f;
    for (long long t = hi - 1; t >= lo; --t) {
      float d, w;
      decay(to_f32(s[t * a.s_st]), d, w);
      const float total = to_f32(dh[t * a.dh_st]) + x, before = t > lo ? to_f32(h[(t - 1) * a.h_st]) : h0;
      x = d * total;
      out[t * a.out_st] = from_f32<T>(MEAN ? x * (to_f32(u[t * a.u_st]) - before) : -x * before);
      du[t * a.du_st] = from_f32<T>(MEAN ? w * total : total);
    }
  }
  if (a.last && row >= 0) a.last[static_cast<long long>(row) * a.C + c] = x;
}

template <bool BWD>
cudaError_t launch(const RecurArgs &a, int type, bool mean, cudaStream_t stream) {
  const int blocks_c = (a.C + 127) / 128;
  const unsigned grid = static_cast<unsigned>(a.S) * blocks_c;
  if (type == kTypeF32) {
    if (mean) recur_serial_kernel<float, true, BWD><<<grid, 128, 0, stream>>>(a, blocks_c);
    else recur_serial_kernel<float, false, BWD><<<grid, 128, 0, stream>>>(a, blocks_c);
  } else {
    if (mean) recur_serial_kernel<__nv_bfloat16, true, BWD><<<grid, 128, 0, stream>>>(a, blocks_c);
    else recur_serial_kernel<__nv_bfloat16, false, BWD><<<grid, 128, 0, stream>>>(a, blocks_c);
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_recur_fwd(const RecurArgs &a, int type, bool mean, int, cudaStream_t stream) {
  return launch<false>(a, type, mean, stream);
}
cudaError_t launch_recur_bwd(const RecurArgs &a, int type, bool mean, int, cudaStream_t stream) {
  return launch<true>(a, type, mean, stream);
}

}  // namespace fem
