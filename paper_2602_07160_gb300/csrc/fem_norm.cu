// A block's end and the next one's start: r = x + scale act(gate) (w_post P(y) + b_post), z = w_pre Q(r) + b_pre
// (include/fem.h, fem_norm_fwd).
//
// Bound by memory: x, y and the gate are read once, r and z written once.  A row stays in its threads' registers from
// the first load to the last store; the sums for a norm are a butterfly in each warp and one meeting of a row's warps,
// and the variance of a layer norm is taken about its mean, which costs a second one but no cancellation.
//
// Measured (32768 rows of 2048): rms, rms, a silu gate, bf16 112 us, 6.0 TB/s of its five arrays; rms, layer, a gate and
// biases over an fp32 stream 159 us, 5.9 TB/s.
#include <algorithm>

#include "fem_norm.cuh"

namespace fem {

namespace {

// Blocks on an SM that registers allow for: 80 to 96 a thread, 64 with 1024 threads.
template <typename S>
constexpr int kBlocks = S::VEC || S::THREADS > 512 ? 1 : S::THREADS > 256 ? 2 : 768 / S::THREADS;
template <typename S, typename TX, typename TY>
constexpr int kRow = Copied<S, TX>::BYTES + 2 * Copied<S, TY>::BYTES;
template <typename S, bool BIAS>
constexpr int kWeights = (BIAS ? 4 : 2) * S::WEIGHT;
template <typename S, typename TX, typename TY, bool BIAS>
constexpr int kSmem = rows_smem<S>(kRow<S, TX, TY>, kWeights<S, BIAS>, kBlocks<S>);

template <typename S, typename TX, typename TY, bool BIAS>
__global__ void __launch_bounds__(S::THREADS, kBlocks<S>) norm_fwd_kernel(const NormArgs a) {
  extern __shared__ __align__(16) char smem[];
  __shared__ float s_red[2 * kRowRed];
  int turn = 0;
  const int lane = threadIdx.x % S::TPR, D = a.D;
  const Mine<S> mine(lane, D);
  const float inv_d = 1.f / static_cast<float>(D);
  const bool branch = a.y.p != nullptr, gated = a.gate.p != nullptr;
  // x, then y, then the gate in a stage
  constexpr bool HOLD = keeps_weights<S>(kRow<S, TX, TY>, kWeights<S, BIAS>);
  constexpr int kept = HOLD ? kWeights<S, BIAS> : 0;  // weights, ahead of the stages
  const int part_x = stage_part<S, TX>(D), part_y = stage_part<S, TY>(D);
  const int stage_bytes = part_x + (branch ? part_y : 0) + (gated ? part_y : 0);
  const int stages = S::COPIED ? min(4, (kSmem<S, TX, TY, BIAS> - kept) / stage_bytes) : 1;  // staged: 2 at least
  int y_off[S::RUNS], g_off[S::RUNS];
  if (S::VEC && branch)
#pragma unroll
    for (int k = 0; k < S::RUNS; ++k) {
      const int e = min((lane + k * S::TPR) * S::RUN, D - S::RUN);
      y_off[k] = static_cast<int>(head_offset(a.y, a.d, e));
      g_off[k] = static_cast<int>(head_offset(a.gate, a.d, e));
    }
  auto weights = [&](int k, int i) {
    const float *p = k == 0 ? a.w_post : k == 1 ? a.w_pre : k == 2 ? a.b_post : a.b_pre;
    if (k >= 2 && !BIAS) p = nullptr;
    return load_weights<S>(p, k < 2 ? 1.f : 0.f, D, lane, i, mine);
  };
  auto weight = [&](int k, int i) {
    if (HOLD && (BIAS || k < 2)) return kept_weights<S>(smem + k * S::WEIGHT, lane, i);
    return weights(k, i);
  };
  if (HOLD) {
    if (threadIdx.x < S::TPR)
      for (int k = 0; k < (BIAS ? 4 : 2); ++k)
#pragma unroll
        for (int i = 0; i < S::K; ++i) keep_weights<S>(smem + k * S::WEIGHT, weights(k, i), lane, i);
    __syncthreads();
  }
  const int rows = blockDim.x / S::TPR, step = gridDim.x * rows;  // at a time: of the block, of the grid
  auto heads_row = [&](const HeadsView &v, int b, int t) { return static_cast<const TY *>(v.p) + heads_start<S>(v, b, t); };
  int first = blockIdx.x * rows, n = first + threadIdx.x / S::TPR, stage = 0;  // the block's rows at a time, the thread's
  RowAt here(n, a.T), ahead = here;
  auto issue = [&](int n, int stage) {
    const bool there = n < a.N;
    const int m = there ? n : 0, b = there ? ahead.b : 0, t = there ? ahead.t : 0;
    const uint32_t to = smem_u32(smem) + kept + stage * stage_bytes;
    issue_row<S>(to, static_cast<const TX *>(a.x) + static_cast<long long>(m) * D, nullptr, D, lane, mine, there);
    if (branch) issue_row<S>(to + part_x, heads_row(a.y, b, t), y_off, D, lane, mine, there);
    if (gated) issue_row<S>(to + part_x + part_y, heads_row(a.gate, b, t), g_off, D, lane, mine, there);
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
    Piece r[S::K];
#pragma unroll
    for (int i = 0; i < S::K; ++i) r[i] = get_piece<S>(slot, static_cast<const TX *>(a.x) + at, nullptr, 0, D, Dn, lane, i);
    auto factor = [&](Piece (&x)[S::K], int kind) {  // 1 / the norm; a layer norm's mean is taken off x
      float sum[1];
      float2 s = both(0.f);
      if (kind == 2) {
#pragma unroll
        for (int i = 0; i < S::K; ++i) add_to(s, x[i]);
        sum[0] = s.x + s.y;
        row_sums<S>(sum, s_red, turn);
        s = both(0.f);
#pragma unroll
        for (int i = 0; i < S::K; ++i) centre<S>(x[i], sum[0] * inv_d, mine, i);
      }
#pragma unroll
      for (int i = 0; i < S::K; ++i) add_product(s, x[i], x[i]);
      sum[0] = s.x + s.y;
      row_sums<S>(sum, s_red, turn);
      return rsqrtf(fmaf(sum[0], inv_d, a.eps));
    };
    if (branch) {
      Piece y[S::K];
#pragma unroll
      for (int i = 0; i < S::K; ++i) y[i] = get_piece<S>(slot + part_x, heads_row(a.y, b, t), &a.y, a.d, D, Dn, lane, i);
      const float inv = a.post != 0 ? factor(y, a.post) : 1.f;
#pragma unroll
      for (int i = 0; i < S::K; ++i) {
        Piece v = weighted(times(y[i], inv), weight(0, i), weight(2, i));
        if (gated) {
          Piece value, slope;
          gate_piece(get_piece<S>(slot + part_x + part_y, heads_row(a.gate, b, t), &a.gate, a.d, D, Dn, lane, i), a.act, value, slope);
          v = times(v, value);
        }
        FEM_EACH_PAIR r[i].v[j] = __ffma2_rn(v.v[j], both(a.scale), r[i].v[j]);
        store_piece<S, TX>(static_cast<TX *>(a.r) + at, nullptr, nullptr, 0, Dn, lane, mine, i, r[i]);
      }
    }
    if (a.pre != 0) {
      const float inv = factor(r, a.pre);
#pragma unroll
      for (int i = 0; i < S::K; ++i)
        store_piece<S, TY>(static_cast<TY *>(a.z) + at, nullptr, nullptr, 0, Dn, lane, mine, i,
                           weighted(times(r[i], inv), weight(1, i), weight(3, i)));
    }
  }
}

template <typename S, typename TX, typename TY, bool BIAS>
struct Tag;

template <typename TX, typename TY, bool BIAS>
struct Launch {
  template <typename S>
  struct With {
    static cudaError_t call(const NormArgs &a, int num_sms, cudaStream_t stream) {
      auto *kernel = norm_fwd_kernel<S, TX, TY, BIAS>;
      int per_sm = 0;
      const cudaError_t e = resident_blocks<Tag<S, TX, TY, BIAS>>(kernel, S::THREADS, kSmem<S, TX, TY, BIAS>, &per_sm);
      if (e != cudaSuccess) return e;
      const int blocks = blocks_of(a.N, S::ROWS, per_sm, num_sms);
      kernel<<<blocks, S::TPR * rows_of(a.N, S::ROWS, blocks), kSmem<S, TX, TY, BIAS>, stream>>>(a);
      return cudaGetLastError();
    }
  };
};

template <typename TX, typename TY>
cudaError_t launch_types(const NormArgs &a, int num_sms, cudaStream_t stream) {
  constexpr int RUN = sizeof(TX) == 4 ? 4 : 8;
  const bool bias = a.b_post || a.b_pre;
  const Way way = way_of(a, norm_pieces(a, sizeof(TY), RUN), staged_row<TX>(a.D) + 2 * staged_row<TY>(a.D), bias ? 4 : 2, 3);
  // 32768 rows of 2048, biases: fp32 stream 162 us with two pieces, 173 with one; bf16 120 and 110.  65536 of 384: 92, 122
  constexpr bool LONG_TWO = RUN == 4;
  return bias ? with_shape<RUN, true, LONG_TWO, 1, 768, 768, 640, 1024, Launch<TX, TY, true>::template With>(a.D, way, a, num_sms, stream)
              : with_shape<RUN, true, LONG_TWO, 1, 768, 768, 640, 1024, Launch<TX, TY, false>::template With>(a.D, way, a, num_sms, stream);
}

}  // namespace

cudaError_t launch_norm_fwd(const NormArgs &a, int x_type, int y_type, int num_sms, cudaStream_t stream) {
  if (y_type == kTypeF32) return launch_types<float, float>(a, num_sms, stream);
  if (x_type == kTypeF32) return launch_types<float, __nv_bfloat16>(a, num_sms, stream);
  return launch_types<__nv_bfloat16, __nv_bfloat16>(a, num_sms, stream);
}

}  // namespace fem
