// Gradients of a block's end and the next one's start (include/fem.h, fem_norm_bwd).  With u = Q(r)'s normalised row
// and rho its factor, v = P(y)'s and sigma its factor, means over the row:
//
//   f  = w_pre dz,  dx = dr + rho (f - [mean f] - u mean(f u))        ([]: layer norms)
//   e  = scale dx,  dgate = e (w_post v + b_post) act'(gate),  e' = e act(gate)
//   g  = w_post e', dy = sigma (g - [mean g] - v mean(g v))
//   dw_pre = sum dz u, db_pre = sum dz, dw_post = sum e' v, db_post = sum e'      over the rows
//
// Bound by memory: r, y, the gate, dr and dz are read once, dx, dy and dgate written once.  A row stays in its threads'
// registers; the sums of r, y and dz need one meeting of the row's warps (layer norms: two, the variance about the
// mean), those of g one more.  The weights' sums over rows stay in registers too while a block goes through its rows,
// and leave as one row of partial sums per block, which a second kernel adds in order.
#include "fem_launch.h"
#include "fem_norm.cuh"

namespace fem {

namespace {

template <typename S, typename TX, typename TY, bool BIAS>
__global__ void __launch_bounds__(S::THREADS) norm_bwd_kernel(const NormArgs a) {
  constexpr int SUMS = BIAS ? 4 : 2;
  __shared__ float s_red[2 * kRowRed];
  int turn = 0;
  const int lane = threadIdx.x % S::TPR, D = a.D;
  const float inv_d = 1.f / static_cast<float>(D);
  const bool branch = a.y.p != nullptr, centred = a.pre == 2 || (branch && a.post == 2);
  float acc[SUMS][S::K][8];  // dw_post, dw_pre, db_post, db_pre
#pragma unroll
  for (int k = 0; k < SUMS; ++k)
#pragma unroll
    for (int i = 0; i < S::K; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[k][i][j] = 0.f;

  for (long long row0 = static_cast<long long>(blockIdx.x) * S::ROWS; row0 < a.N; row0 += static_cast<long long>(gridDim.x) * S::ROWS) {
    const long long n = row0 + threadIdx.x / S::TPR;
    const int Dn = n < a.N ? D : 0;  // a row past the end has no elements, and its threads meet the others
    const int b = static_cast<int>(n / a.T), t = static_cast<int>(n - static_cast<long long>(b) * a.T);
    float r[S::K][8], y[S::K][8], dz[S::K][8], dx[S::K][8];
#pragma unroll
    for (int i = 0; i < S::K; ++i) {
      if (a.pre != 0) {
        load_piece<S, TX>(static_cast<const TX *>(a.x) + n * D, Dn, lane, i, r[i]);
        load_piece<S, TY>(static_cast<const TY *>(a.dz) + n * D, Dn, lane, i, dz[i]);
      }
      if (a.dr) load_piece<S, TX>(static_cast<const TX *>(a.dr) + n * D, Dn, lane, i, dx[i]);
      else
#pragma unroll
        for (int j = 0; j < 8; ++j) dx[i][j] = 0.f;
      if (branch) load_heads<S, TY>(a.y, b * a.y.sb + t * a.y.st, Dn, a.d, lane, i, y[i]);
    }
    // means for layer norms, then sums of squares and of f u, f being w_pre dz
    float mean_r = 0.f, mean_y = 0.f, mean_f = 0.f;
    if (centred) {
      float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        float w[8];
        load_weights<S>(a.w_pre, D, lane, i, 1.f, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (a.pre == 2 && S::at(lane, i, j) < D) {
            v[0] += r[i][j];
            v[2] = fmaf(w[j], dz[i][j], v[2]);
          }
          if (branch && a.post == 2) v[1] += y[i][j];
        }
      }
      row_sums<S>(v, s_red, turn);
      mean_r = v[0] * inv_d;
      mean_y = v[1] * inv_d;
      mean_f = v[2] * inv_d;
    }
    float v[3] = {0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S::K; ++i) {
      float w[8];
      load_weights<S>(a.w_pre, D, lane, i, 1.f, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = S::at(lane, i, j) < D;
        if (a.pre != 0) {
          r[i][j] = in ? r[i][j] - mean_r : 0.f;
          v[0] = fmaf(r[i][j], r[i][j], v[0]);
          if (in) v[1] = fmaf(w[j] * dz[i][j], r[i][j], v[1]);
        }
        if (branch && a.post != 0) {
          y[i][j] = in ? y[i][j] - mean_y : 0.f;
          v[2] = fmaf(y[i][j], y[i][j], v[2]);
        }
      }
    }
    if (a.pre != 0 || (branch && a.post != 0)) row_sums<S>(v, s_red, turn);
    const float rho = rsqrtf(fmaf(v[0], inv_d, a.eps)), fu = v[1] * inv_d * rho;
    const float sigma = a.post != 0 ? rsqrtf(fmaf(v[2], inv_d, a.eps)) : 1.f;
    // dx, dgate, and g = w_post e' with its sums
    float q[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < S::K; ++i) {
      if (a.pre != 0) {
        float w[8];
        load_weights<S>(a.w_pre, D, lane, i, 1.f, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float u = r[i][j] * rho;
          dx[i][j] += rho * (w[j] * dz[i][j] - mean_f - u * fu);
          acc[1][i][j] = fmaf(dz[i][j], u, acc[1][i][j]);
          if (BIAS) acc[SUMS - 1][i][j] += dz[i][j];
        }
      }
      store_piece<S, TX>(static_cast<TX *>(a.dx) + n * D, Dn, lane, i, dx[i]);
      if (!branch) continue;
      float w[8], c[8], g[8];
      load_weights<S>(a.w_post, D, lane, i, 1.f, w);
      load_weights<S>(a.b_post, D, lane, i, 0.f, c);
      if (a.gate.p) load_heads<S, TY>(a.gate, b * a.gate.sb + t * a.gate.st, Dn, a.d, lane, i, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = S::at(lane, i, j) < Dn ? a.scale * dx[i][j] : 0.f;
        float value = 1.f, slope = 0.f;
        if (a.gate.p) gate_slope(g[j], a.act, value, slope);
        y[i][j] *= sigma;
        g[j] = e * fmaf(y[i][j], w[j], c[j]) * slope;
        const float gated = e * value;
        acc[0][i][j] = fmaf(gated, y[i][j], acc[0][i][j]);
        if (BIAS) acc[SUMS - 2][i][j] += gated;
        dx[i][j] = w[j] * gated;
        if (S::at(lane, i, j) < Dn) {
          q[0] += dx[i][j];
          q[1] = fmaf(dx[i][j], y[i][j], q[1]);
        }
      }
      if (a.gate.p) store_heads<S, TY>(a.dgate, b * a.dgate.sb + t * a.dgate.st, Dn, a.d, lane, i, g);
    }
    if (!branch) continue;
    if (a.post != 0) {
      row_sums<S>(q, s_red, turn);
      const float mean_g = a.post == 2 ? q[0] * inv_d : 0.f, gv = q[1] * inv_d;
#pragma unroll
      for (int i = 0; i < S::K; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) dx[i][j] = sigma * (dx[i][j] - mean_g - y[i][j] * gv);
    }
#pragma unroll
    for (int i = 0; i < S::K; ++i) store_heads<S, TY>(a.dy, b * a.dy.sb + t * a.dy.st, Dn, a.d, lane, i, dx[i]);
  }

  // the block's sums: its rows' groups one after the other into row blockIdx.x of the partial sums
  float *part = a.part + static_cast<long long>(blockIdx.x) * SUMS * D;
  for (int g = 0; g < S::ROWS; ++g) {
    if (S::ROWS > 1) __syncthreads();
    if (static_cast<int>(threadIdx.x) / S::TPR != g) continue;
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
      for (int i = 0; i < S::K; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int e = S::at(lane, i, j);
          if (e < D) part[k * D + e] = g == 0 ? acc[k][i][j] : part[k * D + e] + acc[k][i][j];
        }
  }
}

// Adds the partial sums of `blocks` rows, 32 columns a block, its eight warps taking every eighth row.
__global__ void __launch_bounds__(256) norm_bwd_sum_kernel(const float *part, int blocks, int sums, int D, float *w_post,
                                                           float *b_post, float *w_pre, float *b_pre) {
  __shared__ float s_sum[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, k = blockIdx.y, e = blockIdx.x * 32 + lane;
  float *out = k == 0 ? w_post : k == 1 ? w_pre : k == 2 ? b_post : b_pre;
  if (!out) return;
  float v = 0.f;
  if (e < D)
    for (int i = w; i < blocks; i += 8) v += part[(static_cast<long long>(i) * sums + k) * D + e];
  s_sum[w][lane] = v;
  __syncthreads();
  if (w != 0 || e >= D) return;
#pragma unroll
  for (int i = 1; i < 8; ++i) v += s_sum[i][lane];
  out[e] = v;
}

template <typename S, typename TX, typename TY>
cudaError_t launch_shape(const NormArgs &a, int blocks, cudaStream_t stream) {
  const bool bias = a.dw[1] || a.dw[3];
  if (bias) norm_bwd_kernel<S, TX, TY, true><<<blocks, S::THREADS, 0, stream>>>(a);
  else norm_bwd_kernel<S, TX, TY, false><<<blocks, S::THREADS, 0, stream>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !(a.dw[0] || a.dw[1] || a.dw[2] || a.dw[3])) return e;
  const int sums = bias ? 4 : 2;
  norm_bwd_sum_kernel<<<dim3((a.D + 31) / 32, sums), 256, 0, stream>>>(a.part, blocks, sums, a.D, a.dw[0], a.dw[1], a.dw[2], a.dw[3]);
  return cudaGetLastError();
}

template <typename TX, typename TY>
cudaError_t launch_types(const NormArgs &a, int blocks, cudaStream_t stream) {
  if (!norm_pieces(a, sizeof(TY))) {
    if (a.D <= 1024) return launch_shape<RowShape<128, 1, false>, TX, TY>(a, blocks, stream);
    if (a.D <= 4096) return launch_shape<RowShape<512, 1, false>, TX, TY>(a, blocks, stream);
    return launch_shape<RowShape<1024, 2, false>, TX, TY>(a, blocks, stream);
  }
  if (a.D <= 256) return launch_shape<RowShape<32, 1, true>, TX, TY>(a, blocks, stream);
  if (a.D <= 512) return launch_shape<RowShape<64, 1, true>, TX, TY>(a, blocks, stream);
  if (a.D <= 1024) return launch_shape<RowShape<128, 1, true>, TX, TY>(a, blocks, stream);
  if (a.D <= 2048) return launch_shape<RowShape<256, 1, true>, TX, TY>(a, blocks, stream);
  if (a.D <= 4096) return launch_shape<RowShape<512, 1, true>, TX, TY>(a, blocks, stream);
  if (a.D <= 8192) return launch_shape<RowShape<1024, 1, true>, TX, TY>(a, blocks, stream);
  return launch_shape<RowShape<1024, 2, true>, TX, TY>(a, blocks, stream);
}

}  // namespace

int norm_bwd_blocks(int N, int D, int num_sms) {
  const int rows = D <= 256 ? 8 : D <= 512 ? 4 : D <= 1024 ? 2 : 1, per_sm = D <= 2048 ? 2 : 1;
  const int groups = (N + rows - 1) / rows, most = num_sms * per_sm;
  return groups < most ? groups : most;
}

cudaError_t launch_norm_bwd(const NormArgs &a, int x_type, int y_type, int num_sms, cudaStream_t stream) {
  const int blocks = norm_bwd_blocks(a.N, a.D, num_sms);
  if (y_type == kTypeF32) return launch_types<float, float>(a, blocks, stream);
  if (x_type == kTypeF32) return launch_types<float, __nv_bfloat16>(a, blocks, stream);
  return launch_types<__nv_bfloat16, __nv_bfloat16>(a, blocks, stream);
}

}  // namespace fem
