// Rotary positions of queries and keys, in one launch.
//
// A pair (a, b) of a head becomes A (a cos x - b sin x, b cos x + a sin x) with x = pos theta_i.  The rates come as
// fractions of a turn in 64-bit fixed point, so a position's angle is one integer product modulo a turn: exact for
// any position, where a product in fp32 has no correct digit left of the angle from 2^24 radians on.  The nearest
// quarter turn is taken off as an integer too, and what is left, at most an eighth, to polynomials.
//
// Bound by memory: every element is read once and written once, and a token's cosines and sines are formed once for
// all its heads, in shared memory.
//
// Measured: 16383 tokens of 32 + 8 heads of 128, bf16, 60 us, 5.6 TB/s; 8192 of 16 + 16 heads of 64, half of each, fp32
// pairs of neighbours 25 us, 5.3 TB/s.
#include <algorithm>

#include "fem_layer.cuh"

namespace fem {

namespace {

// cos and sin of 2 pi turn / 2^64: of the rest r behind the nearest quarter, |r| <= pi/4, by their Taylor polynomials (the
// first terms left out are under 2e-9 and 3e-8), each off by at most 2 units of 2^-24 of 1.
__device__ __forceinline__ float2 turn_cos_sin(unsigned long long turn) {
  const unsigned long long up = turn + (1ull << 61);                       // nearest quarter: round half up
  const long long rest = static_cast<long long>(turn - (up & (3ull << 62)));  // in [-2^61, 2^61)
  const float r = static_cast<float>(rest) * (0x1p-63f * 3.14159265358979f), q = r * r;
  float sn = fmaf(q, 1.f / 362880.f, -1.f / 5040.f), cs = fmaf(q, 1.f / 40320.f, -1.f / 720.f);
  sn = fmaf(q, sn, 1.f / 120.f);
  cs = fmaf(q, cs, 1.f / 24.f);
  sn = fmaf(q, sn, -1.f / 6.f);
  cs = fmaf(q, cs, -0.5f);
  sn = fmaf(r * q, sn, r);
  cs = fmaf(q, cs, 1.f);
  const unsigned quarter = static_cast<unsigned>(up >> 62);
  if (quarter & 1) {
    const float t = cs;
    cs = -sn;
    sn = t;
  }
  return quarter & 2 ? make_float2(-cs, -sn) : make_float2(cs, sn);
}

// 16 bytes of a head: PER elements.
template <typename T>
struct Chunk {
  static constexpr int PER = 16 / sizeof(T);
  uint4 w;
  __device__ __forceinline__ void load(const T *p) { w = __ldcs(reinterpret_cast<const uint4 *>(p)); }
  __device__ __forceinline__ void store(T *p) const { *reinterpret_cast<uint4 *>(p) = w; }
  __device__ __forceinline__ void get(float (&f)[PER]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (PER == 4) f[i] = __uint_as_float(u[i]);
      else f[2 * i % PER] = bf16_lo(u[i]), f[(2 * i + 1) % PER] = bf16_hi(u[i]);
    }
  }
  __device__ __forceinline__ void put(const float (&f)[PER]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = PER == 4 ? __float_as_uint(f[i]) : bf16_pack(f[2 * i % PER], f[(2 * i + 1) % PER]);
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
};

constexpr int kHeads = 4;  // of a thread under way

// How a head is shared out.  WHOLE: a thread has 16 bytes of each half, twice 16 bytes of neighbours, or twice 16 bytes to
// copy, whose cosines and sines stay in registers from head to head (twice: 16383 tokens of 32 + 8 heads of 128 in
// neighbours 57 us, once 67; of 16 + 4 heads of 256, half turned, 57 and 79).  SHIFTED: where the halves do not end on 16 bytes a thread has
// any 16 bytes of the head and finds their other halves in shared memory.  SINGLE: every pieces-th pair.  (16383 tokens of
// 32 + 8 heads of 128, bf16: WHOLE 56 us, SHIFTED 132, SINGLE 465; 8192 of heads of 80, 74 turned: SHIFTED 32, SINGLE 85.)
enum Way { SINGLE, WHOLE, SHIFTED };

template <typename T, bool INTER, Way WAY>
__global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a, int tokens, int pieces, int hl) {
  extern __shared__ __align__(16) float2 s_cs[];  // [tokens][rotary / 2], SHIFTED behind [kHeads][256] pieces
  constexpr bool VEC = WAY == WHOLE;
  constexpr int PER = Chunk<T>::PER;
  const int pairs = a.rotary / 2, first = blockIdx.x * tokens, rows = a.B * a.T, all = a.heads[0] + a.heads[1];
  const int piece = threadIdx.x % pieces, lane = threadIdx.x / pieces, tok = lane / hl, n = first + tok;
  const int turned = INTER ? a.rotary / PER : pairs / PER;  // pieces of the rotated part
  const bool on = tok < tokens && n < rows;
  const int b = on ? n / a.T : 0, t = on ? n - b * a.T : 0, h0 = blockIdx.y * hl + lane % hl, step = gridDim.y * hl;
  auto place = [&](const HeadsView *v, int h) {
    const int which = h >= a.heads[0];
    return static_cast<T *>(v[which].p) + b * v[which].sb + t * v[which].st + (which ? h - a.heads[0] : h) * v[which].sh;
  };
  // VEC: a thread's first 16 bytes, the second ones `gap` behind them if there are `two`
  const bool copies = VEC && !INTER && piece >= turned;
  const int at = WAY == SINGLE ? 0 : copies ? a.rotary + (piece - turned) * PER : piece * PER;
  const int gap = INTER ? pieces * PER : copies ? (pieces - turned) * PER : pairs;
  const bool two = VEC && (INTER || copies ? at + gap < a.d : true);
  Chunk<T> x[kHeads], y[kHeads];
  auto load = [&](int from) {
#pragma unroll
    for (int u = 0; u < kHeads; ++u) {
      const int h = from + u * step;
      if (!on || h >= all) break;
      const T *src = place(a.in, h) + at;
      x[u].load(src);
      if (two) y[u].load(src + gap);
    }
  };
  if (WAY != SINGLE) load(h0);  // under way while the angles are formed

  float2 *s_turn = s_cs + (WAY == SHIFTED ? kHeads * 256 * 2 : 0);
  {  // a thread forms one pair's angles, for every `each`-th token
    const int each = max(1, 256 / pairs);
    if (threadIdx.x < each * pairs || pairs > 256)
      for (int p = pairs > 256 ? threadIdx.x : threadIdx.x % pairs; p < pairs; p += pairs > 256 ? 256 : pairs) {
        const unsigned long long rate = __ldg(a.turns + p);
#pragma unroll 4
        for (int k = pairs > 256 ? 0 : threadIdx.x / pairs; k < tokens; k += each) {
          const int m = min(first + k, rows - 1);
          const long long pos = a.pos ? __ldg(a.pos + m) : m % a.T;
          const unsigned long long turn = static_cast<unsigned long long>(pos) * rate;
          const float2 cs = turn_cos_sin(a.inverse ? 0ull - turn : turn);
          s_turn[k * pairs + p] = make_float2(cs.x * a.amplitude, cs.y * a.amplitude);
        }
      }
  }
  __syncthreads();
  const float2 *cs = s_turn + (on ? tok : 0) * pairs;
  if constexpr (WAY == SHIFTED) {
    // every thread goes round as often as the one with the most heads: the others wait for it
    const int rounds = (all + kHeads * step - 1) / (kHeads * step);
    uint4 *buf = reinterpret_cast<uint4 *>(s_cs);
    float2 w[PER];  // what an element and its other half are taken by
    int other[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = min(at + i, a.rotary - 1);
      const bool second = INTER ? e & 1 : e >= pairs;
      w[i] = cs[INTER ? e / 2 : second ? e - pairs : e];
      if (!second) w[i].y = -w[i].y;
      other[i] = INTER ? e ^ 1 : second ? e - pairs : e + pairs;
    }
    for (int it = 0; it < rounds; ++it) {
      const int from = h0 + it * kHeads * step;
      if (it > 0) load(from);
#pragma unroll
      for (int u = 0; u < kHeads; ++u)
        if (on && from + u * step < all) buf[u * 256 + threadIdx.x] = x[u].w;
      __syncthreads();
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        const int h = from + u * step;
        if (!on || h >= all) break;
        const T *head = reinterpret_cast<const T *>(buf + u * 256 + threadIdx.x - piece);
        float f[PER];
        x[u].get(f);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const float turned = f[i] * w[i].x + to_f32(head[other[i]]) * w[i].y;
          f[i] = at + i < a.rotary ? turned : f[i];
        }
        x[u].put(f);
        x[u].store(place(a.out, h) + at);
      }
      __syncthreads();
    }
    return;
  }
  if (!on) return;
  if constexpr (VEC) {
    float2 c[PER];  // neighbours: the first pairs' and the second ones'
    const bool turns = piece < turned, turns_too = INTER && piece + pieces < turned;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const bool second = INTER && i >= PER / 2;
      if (second ? turns_too : turns) c[i] = cs[INTER ? (piece + (second ? pieces : 0)) * (PER / 2) + i % (PER / 2) : piece * PER + i];
    }
    auto turn_neighbours = [&](Chunk<T> &v, int from) {
      float f[PER];
      v.get(f);
#pragma unroll
      for (int i = 0; i < PER; i += 2) {
        const float2 w = c[(from + i / 2) % PER];
        const float p = f[i] * w.x - f[i + 1] * w.y;
        f[i + 1] = f[i + 1] * w.x + f[i] * w.y;
        f[i] = p;
      }
      v.put(f);
    };
    for (int from = h0; from < all; from += kHeads * step) {
      if (from != h0) load(from);
#pragma unroll
      for (int u = 0; u < kHeads; ++u) {
        const int h = from + u * step;
        if (h >= all) break;
        T *dst = place(a.out, h) + at;
        if constexpr (INTER) {
          if (turns) turn_neighbours(x[u], 0);
          if (turns_too) turn_neighbours(y[u], PER / 2);
        } else if (turns) {
          float f[PER], g[PER];
          x[u].get(f);
          y[u].get(g);
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const float p = f[i] * c[i].x - g[i] * c[i].y;
            g[i] = g[i] * c[i].x + f[i] * c[i].y;
            f[i] = p;
          }
          x[u].put(f);
          y[u].put(g);
        }
        if (two) y[u].store(dst + gap);
        x[u].store(dst);
      }
    }
  } else {
    for (int i = piece; i < pairs; i += pieces) {
      const int ja = INTER ? 2 * i : i, jb = INTER ? 2 * i + 1 : pairs + i;
      const float2 w = cs[i];
      for (int from = h0; from < all; from += kHeads * step) {
        float f[kHeads], g[kHeads];
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          if (from + u * step >= all) break;
          const T *src = place(a.in, from + u * step);
          f[u] = to_f32(src[ja]);
          g[u] = to_f32(src[jb]);
        }
#pragma unroll
        for (int u = 0; u < kHeads; ++u) {
          if (from + u * step >= all) break;
          T *dst = place(a.out, from + u * step);
          dst[ja] = from_f32<T>(f[u] * w.x - g[u] * w.y);
          dst[jb] = from_f32<T>(g[u] * w.x + f[u] * w.y);
        }
      }
    }
    for (int j = a.rotary + piece; j < a.d; j += pieces)
      for (int h = h0; h < all; h += step) place(a.out, h)[j] = place(a.in, h)[j];
  }
}

bool whole_pieces(const HeadsView &v, int size) {
  return (reinterpret_cast<uintptr_t>(v.p) & 15u) == 0 && v.sb * size % 16 == 0 && v.st * size % 16 == 0 &&
         v.sh * size % 16 == 0;
}

template <typename T, bool INTER>
cudaError_t launch_rope_t(const RopeArgs &a, int num_sms, cudaStream_t stream) {
  constexpr int PER = Chunk<T>::PER;
  const int pairs = a.rotary / 2, all = a.heads[0] + a.heads[1], rows = a.B * a.T;
  bool vec = a.d % PER == 0 && a.d / PER <= 128;
  for (int i = 0; i < (a.heads[1] ? 2 : 1); ++i)
    vec = vec && whole_pieces(a.in[i], sizeof(T)) && whole_pieces(a.out[i], sizeof(T));
  const Way way = !vec ? SINGLE : (INTER ? a.rotary : pairs) % PER == 0 ? WHOLE : SHIFTED;
  const int pieces = way == SINGLE ? std::min(std::max(pairs, (a.d - a.rotary) / 2), 128) : way == SHIFTED ? a.d / PER : INTER ? (a.d / PER + 1) / 2 : pairs / PER + ((a.d - a.rotary) / PER + 1) / 2;
  const int lanes = 256 / pieces;  // at least 2
  // As few heads to a thread as the GPU has room for, up to eight; then tokens to a block, so that the fewest lanes idle.
  const long long room = 4ll * num_sms * lanes;
  const int most = static_cast<int>(std::min(8ll, (static_cast<long long>(rows) * all + room - 1) / room));
  int hl = std::min(all, lanes);
  if (most > 1) {
    double least = 1e9;
    for (int w = 1; w <= std::min(all, lanes); ++w) {
      const int each = (all + w - 1) / w, used = w * (lanes / w);
      const double cost = static_cast<double>(each) * w / all * lanes / used;
      if (each <= most && cost < least - 1e-9) {
        least = cost;
        hl = w;
      }
    }
  }
  const int tokens = std::max(1, std::min(lanes / hl, rows));
  const dim3 grid((rows + tokens - 1) / tokens, most > 1 && (all + hl - 1) / hl <= most ? 1 : std::min(65535, (all + hl - 1) / hl));
  const size_t smem = static_cast<size_t>(tokens) * pairs * sizeof(float2) + (way == SHIFTED ? kHeads * 256 * 16 : 0);
  if (way == WHOLE) rope_kernel<T, INTER, WHOLE><<<grid, 256, smem, stream>>>(a, tokens, pieces, hl);
  else if (way == SHIFTED) rope_kernel<T, INTER, SHIFTED><<<grid, 256, smem, stream>>>(a, tokens, pieces, hl);
  else rope_kernel<T, INTER, SINGLE><<<grid, 256, smem, stream>>>(a, tokens, pieces, hl);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_rope(const RopeArgs &a, int type, bool interleaved, int num_sms, cudaStream_t stream) {
  if (type == kTypeF32) return interleaved ? launch_rope_t<float, true>(a, num_sms, stream) : launch_rope_t<float, false>(a, num_sms, stream);
  return interleaved ? launch_rope_t<__nv_bfloat16, true>(a, num_sms, stream) : launch_rope_t<__nv_bfloat16, false>(a, num_sms, stream);
}

}  // namespace fem
