// Rotary positions of queries and keys, in one launch.
//
// A pair (a, b) of a head becomes A (a cos x - b sin x, b cos x + a sin x) with x = pos theta_i.  The rates come as
// fractions of a turn in 64-bit fixed point, so a position's angle is one integer product modulo a turn: exact for
// any position, where a product in fp32 has no correct digit left of the angle from 2^24 radians on.  The nearest
// quarter turn is taken off as an integer too, and what is left, at most an eighth, goes to sincospif.
//
// Bound by memory: every element is read once and written once, and a token's cosines and sines are formed once for
// all its heads, in shared memory.
#include "fem_layer.cuh"

namespace fem {

namespace {

// cos and sin of 2 pi turn / 2^64.
__device__ __forceinline__ float2 turn_cos_sin(unsigned long long turn) {
  const unsigned long long up = turn + (1ull << 61);                       // nearest quarter: round half up
  const long long rest = static_cast<long long>(turn - (up & (3ull << 62)));  // in [-2^61, 2^61)
  float sn, cs;
  sincospif(static_cast<float>(rest) * 0x1p-63f, &sn, &cs);  // 2 rest / 2^64 half turns
  const unsigned quarter = static_cast<unsigned>(up >> 62);
  if (quarter & 1) {
    const float t = cs;
    cs = -sn;
    sn = t;
  }
  return quarter & 2 ? make_float2(-cs, -sn) : make_float2(cs, sn);
}

// Eight elements of each side of eight pairs of halves, or eight neighbouring elements (four pairs), a thread; the
// piece of a head is a thread's own, so its cosines and sines stay in registers over the heads.
template <typename T, bool INTER, bool VEC>
__global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a, int tokens, int pieces, int head_lanes) {
  extern __shared__ float2 s_cs[];  // [tokens][rotary / 2]
  const int pairs = a.rotary / 2, first = blockIdx.x * tokens, rows = a.B * a.T;
  for (int i = threadIdx.x; i < tokens * pairs; i += blockDim.x) {
    const int tok = i / pairs, n = first + tok;
    if (n >= rows) break;
    const long long pos = a.pos ? __ldg(a.pos + n) : n % a.T;
    const unsigned long long turn = static_cast<unsigned long long>(pos) * __ldg(a.turns + (i - tok * pairs));
    float2 cs = turn_cos_sin(a.inverse ? 0ull - turn : turn);
    s_cs[i] = make_float2(cs.x * a.amplitude, cs.y * a.amplitude);
  }
  __syncthreads();
  const int piece = threadIdx.x % pieces, lane = threadIdx.x / pieces, tok = lane / head_lanes;
  const int n = first + tok, all = a.heads[0] + a.heads[1];
  if (tok >= tokens || n >= rows) return;
  const int b = n / a.T, t = n - b * a.T;
  const float2 *cs = s_cs + tok * pairs;
  for (int h = blockIdx.y * head_lanes + lane % head_lanes; h < all; h += gridDim.y * head_lanes) {
    const int which = h >= a.heads[0], hh = which ? h - a.heads[0] : h;
    const HeadsView &vi = a.in[which], &vo = a.out[which];
    const T *src = static_cast<const T *>(vi.p) + b * vi.sb + t * vi.st + hh * vi.sh;
    T *dst = static_cast<T *>(vo.p) + b * vo.sb + t * vo.st + hh * vo.sh;
    if constexpr (VEC) {
      // pieces: of the rotated part (pairs / 8 of halves, rotary / 8 of neighbours), then of the rest of the head
      const int turned = INTER ? a.rotary / 8 : pairs / 8;
      Eight<T> x, y;
      if (piece >= turned) {
        const int j = a.rotary + (piece - turned) * 8;
        x.load(src + j);
        x.store(dst + j);
        continue;
      }
      float f[8], g[8];
      if (INTER) {
        x.load(src + piece * 8);
        x.get(f);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float2 c = cs[piece * 4 + i / 2];
          const float p = f[i] * c.x - f[i + 1] * c.y;
          f[i + 1] = f[i + 1] * c.x + f[i] * c.y;
          f[i] = p;
        }
        x.put(f);
        x.store(dst + piece * 8);
      } else {
        x.load(src + piece * 8);
        y.load(src + pairs + piece * 8);
        x.get(f);
        y.get(g);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 c = cs[piece * 8 + i];
          const float p = f[i] * c.x - g[i] * c.y;
          g[i] = g[i] * c.x + f[i] * c.y;
          f[i] = p;
        }
        x.put(f);
        y.put(g);
        x.store(dst + piece * 8);
        y.store(dst + pairs + piece * 8);
      }
    } else {
      for (int i = piece; i < pairs; i += pieces) {
        const int ja = INTER ? 2 * i : i, jb = INTER ? 2 * i + 1 : pairs + i;
        const float x = to_f32(src[ja]), y = to_f32(src[jb]);
        const float2 c = cs[i];
        dst[ja] = from_f32<T>(x * c.x - y * c.y);
        dst[jb] = from_f32<T>(y * c.x + x * c.y);
      }
      for (int j = a.rotary + piece; j < a.d; j += pieces) dst[j] = src[j];
    }
  }
}

bool whole_pieces(const HeadsView &v, int size) {
  return (reinterpret_cast<uintptr_t>(v.p) & 15u) == 0 && v.sb * size % 16 == 0 && v.st * size % 16 == 0 &&
         v.sh * size % 16 == 0;
}

template <typename T, bool INTER>
cudaError_t launch_rope_t(const RopeArgs &a, cudaStream_t stream) {
  const int pairs = a.rotary / 2, all = a.heads[0] + a.heads[1], rows = a.B * a.T;
  bool vec = a.d % 8 == 0 && (INTER ? a.rotary : pairs) % 8 == 0;
  for (int i = 0; i < (a.heads[1] ? 2 : 1); ++i)
    vec = vec && whole_pieces(a.in[i], sizeof(T)) && whole_pieces(a.out[i], sizeof(T));
  const int pieces = vec ? (INTER ? a.d / 8 : pairs / 8 + (a.d - a.rotary) / 8) : 32;
  int lanes = 256 / pieces;  // at least 2: d is at most 1024
  const int head_lanes = all < lanes ? all : lanes, tokens = lanes / head_lanes;
  const dim3 grid((rows + tokens - 1) / tokens, 1);
  const size_t smem = static_cast<size_t>(tokens) * pairs * sizeof(float2);
  if (vec) rope_kernel<T, INTER, true><<<grid, 256, smem, stream>>>(a, tokens, pieces, head_lanes);
  else rope_kernel<T, INTER, false><<<grid, 256, smem, stream>>>(a, tokens, pieces, head_lanes);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeArgs &a, int type, bool interleaved, cudaStream_t stream) {
  if (type == kTypeF32) return interleaved ? launch_rope_t<float, true>(a, stream) : launch_rope_t<float, false>(a, stream);
  return interleaved ? launch_rope_t<__nv_bfloat16, true>(a, stream) : launch_rope_t<__nv_bfloat16, false>(a, stream);
}

}  // namespace fem
