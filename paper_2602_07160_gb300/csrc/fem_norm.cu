// A block's end and the next one's start: r = x + scale act(gate) (w_post P(y) + b_post), z = w_pre Q(r) + b_pre
// (include/fem.h, fem_norm_fwd).
//
// Bound by memory: x, y and the gate are read once, r and z written once.  A row stays in its threads' registers from
// the first load to the last store; the sums for a norm are a butterfly in each warp and one meeting of a row's warps,
// and the variance of a layer norm is taken about its mean, which costs a second one but no cancellation.
#include "fem_norm.cuh"

namespace fem {

namespace {

template <typename S, typename TX, typename TY>
__global__ void __launch_bounds__(S::THREADS) norm_fwd_kernel(const NormArgs a) {
  __shared__ float s_red[2 * kRowRed];
  int turn = 0;
  const int lane = threadIdx.x % S::TPR, D = a.D;
  const float inv_d = 1.f / static_cast<float>(D);
  for (long long row0 = static_cast<long long>(blockIdx.x) * S::ROWS; row0 < a.N; row0 += static_cast<long long>(gridDim.x) * S::ROWS) {
    const long long n = row0 + threadIdx.x / S::TPR;
    const bool on = n < a.N;
    const int Dn = on ? D : 0;  // a row past the end has no elements, and its threads meet the others
    float r[S::K][8];
#pragma unroll
    for (int i = 0; i < S::K; ++i) load_piece<S, TX>(static_cast<const TX *>(a.x) + n * D, Dn, lane, i, r[i]);
    if (a.y.p) {
      const int b = static_cast<int>(n / a.T), t = static_cast<int>(n - static_cast<long long>(b) * a.T);
      float y[S::K][8];
#pragma unroll
      for (int i = 0; i < S::K; ++i) load_heads<S, TY>(a.y, b * a.y.sb + t * a.y.st, Dn, a.d, lane, i, y[i]);
      if (a.post != 0) {
        float sum[1], mean = 0.f;
        if (a.post == 2) {
          sum[0] = 0.f;
#pragma unroll
          for (int i = 0; i < S::K; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[0] += y[i][j];
          row_sums<S>(sum, s_red, turn);
          mean = sum[0] * inv_d;
        }
        sum[0] = 0.f;
#pragma unroll
        for (int i = 0; i < S::K; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            y[i][j] = S::at(lane, i, j) < D ? y[i][j] - mean : 0.f;
            sum[0] = fmaf(y[i][j], y[i][j], sum[0]);
          }
        row_sums<S>(sum, s_red, turn);
        const float inv = rsqrtf(sum[0] * inv_d + a.eps);
#pragma unroll
        for (int i = 0; i < S::K; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) y[i][j] *= inv;
      }
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        float w[8], c[8], g[8];
        load_weights<S>(a.w_post, D, lane, i, 1.f, w);
        load_weights<S>(a.b_post, D, lane, i, 0.f, c);
        if (a.gate.p) load_heads<S, TY>(a.gate, b * a.gate.sb + t * a.gate.st, Dn, a.d, lane, i, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v = fmaf(y[i][j], w[j], c[j]);
          if (a.gate.p) v *= gate_value(g[j], a.act);
          r[i][j] = fmaf(a.scale, v, r[i][j]);
        }
        store_piece<S, TX>(static_cast<TX *>(a.r) + n * D, Dn, lane, i, r[i]);
      }
    }
    if (a.pre != 0) {
      float sum[1], mean = 0.f;
      if (a.pre == 2) {
        sum[0] = 0.f;
#pragma unroll
        for (int i = 0; i < S::K; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[0] += S::at(lane, i, j) < D ? r[i][j] : 0.f;
        row_sums<S>(sum, s_red, turn);
        mean = sum[0] * inv_d;
      }
      sum[0] = 0.f;
#pragma unroll
      for (int i = 0; i < S::K; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          r[i][j] = S::at(lane, i, j) < D ? r[i][j] - mean : 0.f;
          sum[0] = fmaf(r[i][j], r[i][j], sum[0]);
        }
      row_sums<S>(sum, s_red, turn);
      const float inv = rsqrtf(sum[0] * inv_d + a.eps);
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        float w[8], c[8], z[8];
        load_weights<S>(a.w_pre, D, lane, i, 1.f, w);
        load_weights<S>(a.b_pre, D, lane, i, 0.f, c);
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = fmaf(r[i][j] * inv, w[j], c[j]);
        store_piece<S, TY>(static_cast<TY *>(a.z) + n * D, Dn, lane, i, z);
      }
    }
  }
}

template <typename S, typename TX, typename TY>
cudaError_t launch_shape(const NormArgs &a, cudaStream_t stream) {
  const int groups = (a.N + S::ROWS - 1) / S::ROWS;
  norm_fwd_kernel<S, TX, TY><<<groups, S::THREADS, 0, stream>>>(a);
  return cudaGetLastError();
}

template <typename TX, typename TY>
cudaError_t launch_types(const NormArgs &a, cudaStream_t stream) {
  if (!norm_pieces(a, sizeof(TY))) {
    if (a.D <= 1024) return launch_shape<RowShape<128, 1, false>, TX, TY>(a, stream);
    if (a.D <= 4096) return launch_shape<RowShape<256, 2, false>, TX, TY>(a, stream);
    return launch_shape<RowShape<512, 4, false>, TX, TY>(a, stream);
  }
  if (a.D <= 256) return launch_shape<RowShape<32, 1, true>, TX, TY>(a, stream);
  if (a.D <= 512) return launch_shape<RowShape<32, 2, true>, TX, TY>(a, stream);
  if (a.D <= 1024) return launch_shape<RowShape<32, 4, true>, TX, TY>(a, stream);
  if (a.D <= 2048) return launch_shape<RowShape<128, 2, true>, TX, TY>(a, stream);
  if (a.D <= 4096) return launch_shape<RowShape<256, 2, true>, TX, TY>(a, stream);
  if (a.D <= 8192) return launch_shape<RowShape<512, 2, true>, TX, TY>(a, stream);
  return launch_shape<RowShape<1024, 2, true>, TX, TY>(a, stream);
}

}  // namespace

cudaError_t launch_norm_fwd(const NormArgs &a, int x_type, int y_type, int, cudaStream_t stream) {
  if (y_type == kTypeF32) return launch_types<float, float>(a, stream);
  if (x_type == kTypeF32) return launch_types<float, __nv_bfloat16>(a, stream);
  return launch_types<__nv_bfloat16, __nv_bfloat16>(a, stream);
}

}  // namespace fem
