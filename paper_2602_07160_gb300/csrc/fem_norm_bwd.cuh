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
//
// Measured (32768 rows of 2048, rms, rms, a silu gate, bf16): 195 us with the sums' 5, 5.5 TB/s of the eight arrays, issue
// slots 59 % busy: what bounds it is the arithmetic of an element (some 70 instructions, a reciprocal and an exponential) as
// much as memory.
#pragma once

#include <algorithm>

#include "fem_launch.h"
#include "fem_norm.cuh"

namespace fem {

// Adds the partial sums of `blocks` rows in order: the dependent of the kernel that leaves them.
cudaError_t launch_norm_sums(const NormArgs &a, int blocks, int sums, cudaStream_t stream);
// How many blocks there will be (num_sms given), or the launch; float residual streams, and bf16 ones.
cudaError_t norm_bwd_f32(const NormArgs &a, int y_type, int num_sms, int *blocks, cudaStream_t stream);

namespace {

// Blocks on an SM that registers allow for: 168 a thread with two pieces, 128 with one.  (Spilled ones cost more than
// fewer warps do: beside so much shared memory the L1 cache is small.)
template <typename S>
constexpr int kBlocks = S::THREADS > 256 ? 1 : 512 / S::THREADS;
template <typename S, typename TX, typename TY>
constexpr int kRow = 2 * Copied<S, TX>::BYTES + 3 * Copied<S, TY>::BYTES;
template <typename S, bool BIAS>
constexpr int kWeights = (BIAS ? 3 : 2) * S::WEIGHT;
template <typename S, typename TX, typename TY, bool BIAS>
constexpr int kSmem = rows_smem<S>(kRow<S, TX, TY>, kWeights<S, BIAS>, kBlocks<S>);

template <typename S, typename TX, typename TY, bool BIAS>
__global__ void __launch_bounds__(S::THREADS, kBlocks<S>) norm_bwd_kernel(const NormArgs a) {
  constexpr int SUMS = BIAS ? 4 : 2;
  extern __shared__ __align__(16) char smem[];
  __shared__ float s_red[2 * kRowRed];
  int turn = 0;
  const int lane = threadIdx.x % S::TPR, D = a.D;
  const Mine<S> mine(lane, D);
  const float inv_d = 1.f / static_cast<float>(D);
  const bool branch = a.y.p != nullptr, gated = a.gate.p != nullptr, normed = a.pre != 0;
  Piece acc[SUMS][S::K];  // dw_post, dw_pre, db_post, db_pre
#pragma unroll
  for (int k = 0; k < SUMS; ++k)
#pragma unroll
    for (int i = 0; i < S::K; ++i) FEM_EACH_PAIR acc[k][i].v[j] = both(0.f);
  constexpr bool HOLD = keeps_weights<S>(kRow<S, TX, TY>, kWeights<S, BIAS>);
  constexpr int kept = HOLD ? kWeights<S, BIAS> : 0;  // weights, ahead of the stages
  auto weights = [&](int k, int i) {
    return load_weights<S>(k == 0 ? a.w_post : k == 1 ? a.w_pre : BIAS ? a.b_post : nullptr, k < 2 ? 1.f : 0.f, D, lane, i, mine);
  };
  auto weight = [&](int k, int i) {
    if (HOLD && (BIAS || k < 2)) return kept_weights<S>(smem + k * S::WEIGHT, lane, i);
    return weights(k, i);
  };
  if (HOLD) {
    if (threadIdx.x < S::TPR)
      for (int k = 0; k < (BIAS ? 3 : 2); ++k)
#pragma unroll
        for (int i = 0; i < S::K; ++i) keep_weights<S>(smem + k * S::WEIGHT, weights(k, i), lane, i);
    __syncthreads();
  }
  // r, dr, dz, y and the gate in a stage, those that there are
  const int part_x = stage_part<S, TX>(D), part_y = stage_part<S, TY>(D);
  const int at_dr = normed ? part_x : 0, at_dz = at_dr + (a.dr ? part_x : 0), at_y = at_dz + (normed ? part_y : 0);
  const int at_gate = at_y + (branch ? part_y : 0), stage_bytes = at_gate + (gated ? part_y : 0);
  const int stages = S::COPIED ? min(4, (kSmem<S, TX, TY, BIAS> - kept) / stage_bytes) : 1;  // staged: 2 at least
  // places of the pieces in the heads' arrays
  int off[4][S::RUNS];
  if (S::VEC && branch)
#pragma unroll
    for (int k = 0; k < S::RUNS; ++k) {
      const int e = min((lane + k * S::TPR) * S::RUN, D - S::RUN);
      off[0][k] = static_cast<int>(head_offset(a.y, a.d, e));
      off[1][k] = static_cast<int>(head_offset(a.gate, a.d, e));
      off[2][k] = static_cast<int>(head_offset(a.dy, a.d, e));
      off[3][k] = static_cast<int>(head_offset(a.dgate, a.d, e));
    }
  const int rows = blockDim.x / S::TPR, step = gridDim.x * rows;  // at a time: of the block, of the grid
  auto heads_row = [&](const HeadsView &v, int b, int t) { return static_cast<TY *>(v.p) + heads_start<S>(v, b, t); };
  int first = blockIdx.x * rows, n = first + threadIdx.x / S::TPR, stage = 0;  // the block's rows at a time, the thread's
  RowAt here(n, a.T), ahead = here;
  auto issue = [&](int n, int stage) {
    const bool there = n < a.N;
    const int b = there ? ahead.b : 0, t = there ? ahead.t : 0;
    const long long at = static_cast<long long>(there ? n : 0) * D;
    const uint32_t to = smem_u32(smem) + kept + stage * stage_bytes;
    if (normed) {
      issue_row<S>(to, static_cast<const TX *>(a.x) + at, nullptr, D, lane, mine, there);
      issue_row<S>(to + at_dz, static_cast<const TY *>(a.dz) + at, nullptr, D, lane, mine, there);
    }
    if (a.dr) issue_row<S>(to + at_dr, static_cast<const TX *>(a.dr) + at, nullptr, D, lane, mine, there);
    if (branch) issue_row<S>(to + at_y, static_cast<const TY *>(heads_row(a.y, b, t)), off[0], D, lane, mine, there);
    if (gated) issue_row<S>(to + at_gate, static_cast<const TY *>(heads_row(a.gate, b, t)), off[1], D, lane, mine, there);
    ahead.go(step, a.T);
  };
  if constexpr (S::COPIED) {
    if (S::VEC) clear_smem<S>(smem + kept, stages * stage_bytes, D);
    for (int k = 0; k < stages - 1; ++k) {
      if (k == 0 || first < a.N - k * step) issue(n + k * step, k);
      copy_commit();
    }
  }

  for (; first < a.N; first += step, n += step, here.go(step, a.T)) {
    const int Dn = n < a.N ? D : 0;  // a row past the end has no elements, and its threads meet the others
    const char *slot = smem + kept + stage * stage_bytes;
    if constexpr (S::COPIED) {
      if (S::STAGED) {  // the row's threads have all copied it, and have all done with the one before
        rows_wait(stages - 1);
        row_barrier<S>();
      }
      if (first < a.N - (stages - 1) * step) issue(n + (stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
      copy_commit();
      if (S::VEC) rows_wait(stages);
      stage = stage == stages - 1 ? 0 : stage + 1;
    }
    const long long at = static_cast<long long>(n) * D;
    const int b = here.b, t = here.t;
    // r and y stay in registers; dz, dr and the gate are read where they are used
    auto get_dz = [&](int i) { return get_piece<S>(slot + at_dz, static_cast<const TY *>(a.dz) + at, nullptr, 0, D, Dn, lane, i); };
    Piece r[S::K], y[S::K], dx[S::K];
#pragma unroll
    for (int i = 0; i < S::K; ++i) {
      if (normed) r[i] = get_piece<S>(slot, static_cast<const TX *>(a.x) + at, nullptr, 0, D, Dn, lane, i);
      if (branch) y[i] = get_piece<S>(slot + at_y, static_cast<const TY *>(heads_row(a.y, b, t)), &a.y, a.d, D, Dn, lane, i);
    }
    // means for layer norms, f being w_pre dz
    float mean_f = 0.f;
    if (a.pre == 2 || (branch && a.post == 2)) {
      float2 sr = both(0.f), sy = both(0.f), sf = both(0.f);
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        if (a.pre == 2) {
          add_to(sr, r[i]);
          add_to(sf, times(get_dz(i), weight(1, i)));
        }
        if (branch && a.post == 2) add_to(sy, y[i]);
      }
      float v[3] = {sr.x + sr.y, sy.x + sy.y, sf.x + sf.y};
      row_sums<S>(v, s_red, turn);
      mean_f = v[2] * inv_d;
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        if (a.pre == 2) centre<S>(r[i], v[0] * inv_d, mine, i);
        if (branch && a.post == 2) centre<S>(y[i], v[1] * inv_d, mine, i);
      }
    }
    // sums of squares, and of f r
    float rho = 1.f, fu = 0.f, sigma = 1.f;
    if (normed || (branch && a.post != 0)) {
      float2 sr = both(0.f), sy = both(0.f), sf = both(0.f);
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        if (normed) {
          add_product(sr, r[i], r[i]);
          add_product(sf, times(get_dz(i), weight(1, i)), r[i]);
        }
        if (branch && a.post != 0) add_product(sy, y[i], y[i]);
      }
      float v[3] = {sr.x + sr.y, sf.x + sf.y, sy.x + sy.y};
      row_sums<S>(v, s_red, turn);
      rho = rsqrtf(fmaf(v[0], inv_d, a.eps));
      fu = v[1] * inv_d * rho;
      if (a.post != 0) sigma = rsqrtf(fmaf(v[2], inv_d, a.eps));
    }
    // dx, dgate, and g = w_post e' with its sums
    float2 q0 = both(0.f), q1 = both(0.f);
#pragma unroll
    for (int i = 0; i < S::K; ++i) {
      if (a.dr) {
        dx[i] = get_piece<S>(slot + at_dr, static_cast<const TX *>(a.dr) + at, nullptr, 0, D, Dn, lane, i);
      } else {
        FEM_EACH_PAIR dx[i].v[j] = both(0.f);
      }
      if (normed) {
        const Piece dz = get_dz(i), f = times(dz, weight(1, i)), u = times(r[i], rho);
        FEM_EACH_PAIR {
          const float2 off_mean = __fadd2_rn(__ffma2_rn(u.v[j], both(-fu), f.v[j]), both(-mean_f));
          dx[i].v[j] = __ffma2_rn(off_mean, both(rho), dx[i].v[j]);
          acc[1][i].v[j] = __ffma2_rn(dz.v[j], u.v[j], acc[1][i].v[j]);
          if (BIAS) acc[SUMS - 1][i].v[j] = __fadd2_rn(acc[SUMS - 1][i].v[j], dz.v[j]);
        }
      }
      store_piece<S, TX>(static_cast<TX *>(a.dx) + at, nullptr, nullptr, 0, Dn, lane, mine, i, dx[i]);
      if (!branch) continue;
      Piece e = times(dx[i], a.scale);  // behind the row's end the weights are 0, and what e is does not count
      y[i] = times(y[i], sigma);
      Piece value, slope;
      if (gated) {
        gate_piece(get_piece<S>(slot + at_gate, static_cast<const TY *>(heads_row(a.gate, b, t)), &a.gate, a.d, D, Dn, lane, i), a.act,
                   value, slope);
        store_piece<S, TY>(heads_row(a.dgate, b, t), &a.dgate, off[3], a.d, Dn, lane, mine, i,
                           times(times(weighted(y[i], weight(0, i), weight(2, i)), slope), e));
        e = times(e, value);
      }
      FEM_EACH_PAIR {
        acc[0][i].v[j] = __ffma2_rn(e.v[j], y[i].v[j], acc[0][i].v[j]);
        if (BIAS) acc[SUMS - 2][i].v[j] = __fadd2_rn(acc[SUMS - 2][i].v[j], e.v[j]);
      }
      dx[i] = times(e, weight(0, i));
      add_to(q0, dx[i]);
      add_product(q1, dx[i], y[i]);
    }
    if (!branch) continue;
    if (a.post != 0) {
      float q[2] = {q0.x + q0.y, q1.x + q1.y};
      row_sums<S>(q, s_red, turn);
      const float mean_g = a.post == 2 ? q[0] * inv_d : 0.f, gv = q[1] * inv_d;
#pragma unroll
      for (int i = 0; i < S::K; ++i)
        FEM_EACH_PAIR dx[i].v[j] = __fmul2_rn(__fadd2_rn(__ffma2_rn(y[i].v[j], both(-gv), dx[i].v[j]), both(-mean_g)), both(sigma));
    }
#pragma unroll
    for (int i = 0; i < S::K; ++i) store_piece<S, TY>(heads_row(a.dy, b, t), &a.dy, off[2], a.d, Dn, lane, mine, i, dx[i]);
  }

  if (!a.part) return;  // no weights' gradients wanted
  grid_dep_launch_dependents();
  // the block's sums into row blockIdx.x of the partial sums: those of its rows meet in shared memory (where a row's copies
  // had 10 bytes an element and array or more, and now have 4 a sum), in order
  float *part = a.part + static_cast<long long>(blockIdx.x) * SUMS * D, *to = part;
  if constexpr (S::ROWS > 1) {
    to = reinterpret_cast<float *>(smem) + threadIdx.x / S::TPR * SUMS * D;
    __syncthreads();
  }
#pragma unroll
  for (int k = 0; k < SUMS; ++k)
#pragma unroll
    for (int i = 0; i < S::K; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int e = S::at(lane, i, j);
        if (e < D) to[k * D + e] = j % 2 ? acc[k][i].v[j / 2].y : acc[k][i].v[j / 2].x;
      }
  if constexpr (S::ROWS > 1) {
    static_assert(S::COPIED, "shared memory to meet in");
    __syncthreads();
    for (int e = threadIdx.x; e < SUMS * D; e += blockDim.x) {
      float x = 0.f;
      for (int g = 0; g < rows; ++g) x += reinterpret_cast<const float *>(smem)[g * SUMS * D + e];
      part[e] = x;
    }
  }
}

template <typename S, typename TX, typename TY, bool BIAS>
struct Tag;

// One of: how many blocks there will be (num_sms given), or the launch.
template <typename TX, typename TY, bool BIAS>
struct Launch {
  template <typename S>
  struct With {
    static cudaError_t call(const NormArgs &a, int num_sms, int *blocks, cudaStream_t stream) {
      auto *kernel = norm_bwd_kernel<S, TX, TY, BIAS>;
      constexpr int smem = kSmem<S, TX, TY, BIAS>;
      if (num_sms > 0) {
        int per_sm = 0;
        const cudaError_t e = resident_blocks<Tag<S, TX, TY, BIAS>>(kernel, S::THREADS, smem, &per_sm);
        *blocks = e == cudaSuccess ? blocks_of(a.N, S::ROWS, per_sm, num_sms) : 0;
        return e;
      }
      kernel<<<*blocks, S::TPR * rows_of(a.N, S::ROWS, *blocks), smem, stream>>>(a);
      const cudaError_t e = cudaGetLastError();
      if (e != cudaSuccess || !(a.dw[0] || a.dw[1] || a.dw[2] || a.dw[3])) return e;
      return launch_norm_sums(a, *blocks, BIAS ? 4 : 2, stream);
    }
  };
};

template <typename TX, typename TY>
cudaError_t types(const NormArgs &a, int num_sms, int *blocks, cudaStream_t stream) {
  constexpr int RUN = sizeof(TX) == 4 ? 4 : 8;
  // a row of all arrays that does not fit in shared memory is not copied
  const bool pieces = norm_pieces(a, sizeof(TY), RUN) && (a.D <= 8192 || (2 * sizeof(TX) + 3 * sizeof(TY)) * 16384 <= kMostSmem);
  const bool bias = a.dw[1] || a.dw[3] || a.b_post;
  const Way way = way_of(a, pieces, 2 * staged_row<TX>(a.D) + 3 * staged_row<TY>(a.D), bias ? 3 : 2, 2);
  // 32768 rows of 2048 of bf16: 199 us with two pieces, 224 with one; of fp32 two leave registers short.  32768 rows of 768
  // of fp32, layer norms: 141 us in blocks of 480 threads, 166 of 576, for which registers are 96
  constexpr bool TWO = RUN == 8;
  return bias ? with_shape<RUN, TWO, TWO, 2, 512, 480, 384, 512, Launch<TX, TY, true>::template With>(a.D, way, a, num_sms, blocks, stream)
              : with_shape<RUN, TWO, TWO, 2, 512, 480, 384, 512, Launch<TX, TY, false>::template With>(a.D, way, a, num_sms, blocks, stream);
}

}  // namespace
}  // namespace fem
