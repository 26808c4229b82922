// The paged read of few new tokens per sequence: decode steps and drafted tokens.
//
// Bound by memory: the cached keys and values are read once and each is used by
// the few rows of its head's group.  A CTA of four warps takes a stretch of the
// line of work (fem_paged_split.cuh) in tiles of 64 keys, 16 per warp; each warp
// runs its own ring of TMA copies, with no barrier between warps inside an item.
// The scores are K Q^T with the keys as the rows of the matrix instruction and
// the (8 or 16) query rows as its columns, so that no row of the wide side is
// wasted; the second product is E^T P^T with the channels as rows.  Both
// operands come straight from shared memory in the lane layout the instruction
// wants: the contraction index of the first (channels of q and k) and the row
// and contraction indices of the second (channels; keys) are renumbered so that
// a lane's share is 16 contiguous bytes of a key's row, and key_of and chunk_of
// keep the eight lanes of each quarter warp on distinct banks of the swizzled
// tile.  The value bank is formed in registers on the way, once per value for
// all rows.  mma.sync suffices here: at 8 rows the products take a fraction of
// the time the bytes do (tensor pipe 9 to 10 % busy).
// One token over 131071 keys, 8 heads of 128 for 32 query heads, bf16: 101 us with
// the join, 5.3 TB/s of the 6.8 that a copy reaches.  48 tokens over 2048 to 8192
// keys each in e4m3: 131 us, 3.8 TB/s: the bytes are half and the bank the same, and
// the eleven warps of an SM that its registers leave issue in 55 % of the cycles.
#include <type_traits>

#include "fem_launch.h"
#include "fem_paged.cuh"
#include "fem_paged_split.cuh"

namespace fem {

namespace {

constexpr int kTokWarps = 4;
constexpr int kTokThreads = 32 * kTokWarps;
constexpr int kTokKeys = 16;                          // keys per warp and stage

template <int FORMAT, int D, int NT>
struct TokLayout {
  static constexpr int kElem = FORMAT == kCacheBf16 ? 2 : 1;
  static constexpr int kRow = D * kElem;                       // bytes of a cached row
  static constexpr int kBox = kRow < 128 ? kRow : 128;         // bytes of a row in one TMA box
  static constexpr int kBoxes = kRow / kBox;
  static constexpr int kStage = 2 * kTokKeys * kRow;           // K and V of 16 keys
  // CTAs per SM, and the ring: at d = 128 in bf16 a key takes 512 bytes, and two CTAs with three stages
  // keep more in flight than three with two (131071 keys: 106 us against 118 when it was chosen); the others
  // gain from the twelve warps (48 sequences over e4m3: 158 us against 185)
  static constexpr int kCtas = kStage >= 8192 ? 2 : 3;
  static constexpr int kStages = (kCtas == 2 ? 24576 : 16384) / kStage < 6 ? (kCtas == 2 ? 24576 : 16384) / kStage : 6;
  static constexpr int kRows = 8 * NT;
  static constexpr int kRedStride = D + 1;  // so that the lanes of a store to the join meet on two banks at most
  static_assert(kRows * kRedStride * 4 <= kStages * kStage, "a warp's ring holds its rows");
  // shared memory: rings (in the join, the warps' rows), then scale bytes, barriers, coefficients
  static constexpr int kScale = kTokWarps * kStages * kStage;
  static constexpr int kBar = kScale + kTokWarps * kStages * 32;
  static constexpr int kCoef4 = (kBar + kTokWarps * kStages * 8 + 15) & ~15;
  static constexpr int kShift = kCoef4 + D * 16;
  static constexpr int kStat = kShift + D * 4;  // [warps][rows] {m, L}
  static constexpr int kEmax = kStat + kTokWarps * kRows * 8;  // per channel: largest |E| as held (its bits) where wide, or 0
  static constexpr int kRowBad = kEmax + D * 4;  // per row: some channel needs the exact path
  static constexpr int kBytes = kRowBad + kRows * 4;
  static constexpr int kAlloc = kBytes + 1024;
};

// Key (of 16) at row or contraction index x of the matrix instruction.
template <bool ROW128>
__device__ __forceinline__ int key_of(int x) {
  return ROW128 ? (x & 8) + ((x & 7) >> 1) + 4 * (x & 1) : x;
}

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr));
  return v;
}

// Byte offset of 16-byte chunk `chunk` of row `row` in a stage's K or V tile.
template <int BOX>
__device__ __forceinline__ uint32_t tok_offset(int row, int chunk) {
  if (BOX == 128) return (chunk >> 3) * (kTokKeys * 128) + sw128_offset(row, chunk & 7);
  return row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4);  // the 64-byte swizzle of 64-byte rows
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __int_as_float(static_cast<int>(w << 16)); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __int_as_float(static_cast<int>(w & 0xffff0000u)); }

// Four e4m3 codes as two words of f16 pairs, exactly.
__device__ __forceinline__ uint2 e4m3x4_to_f16(uint32_t x) {
  uint2 r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
      : "=r"(r.x), "=r"(r.y)
      : "r"(x));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_float2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2 *>(&x)); }

template <int FORMAT, int D, int NT, bool BETA>
__global__ void __launch_bounds__(kTokThreads, (TokLayout<FORMAT, D, NT>::kCtas))
    paged_token_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                       const PagedReadArgs a, const PagedSplit sp, const SplitShape shape) {
  using Lay = TokLayout<FORMAT, D, NT>;
  constexpr bool R128 = Lay::kBox == 128;
  constexpr int kRows = Lay::kRows, NS = Lay::kStages, MT = D / 16;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ SplitScan<kTokThreads> scan;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
  const int g = lane >> 2, i4 = lane & 3;
  const uint32_t sbase = smem_u32(smem);
  const uint32_t ring = sbase + warp * NS * Lay::kStage;
  const uint32_t scales = sbase + Lay::kScale + warp * NS * 32;
  const uint32_t bars = sbase + Lay::kBar + warp * NS * 8;
  float *s_coef = reinterpret_cast<float *>(smem + Lay::kCoef4);
  float *s_shift = reinterpret_cast<float *>(smem + Lay::kShift);
  float2 *s_stat = reinterpret_cast<float2 *>(smem + Lay::kStat);
  int *s_emax = reinterpret_cast<int *>(smem + Lay::kEmax);
  int *s_bad = reinterpret_cast<int *>(smem + Lay::kRowBad);

  grid_dep_launch_dependents();
  if (lane == 0) {
    for (int st = 0; st < NS; ++st) mbar_init(bars + 8 * st, 1);
    fence_mbar_init();
  }
  const int cta = blockIdx.x;
  SplitWalk walk;
  __shared__ SplitRecord record;
  if (tid == 0) record = SplitRecord{};
  if (!split_begin(a, shape, cta, gridDim.x, scan, walk)) {
    if (tid == 0) sp.records[cta] = SplitRecord{};
    return;
  }
  SplitSeg sg;
  unsigned phases = 0;  // parity of each stage's barrier
  bool alive = true;

  while (walk.next(a, shape, sg)) {
    const int row0 = sg.r * kRows, total = sg.si.n * a.group, n_rows = min(kRows, total - row0);
    // loads that wait for nothing go first
    const float beta_c = BETA && tid < D ? __ldg(a.beta + static_cast<long long>(sg.h) * D + tid) : 0.f;
    // ---- Q^T as the second operand: column g of row tile t, the lane's channels in the order K's 16-byte pieces bring them
    uint32_t qf[NT][MT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int r = row0 + 8 * t + g;
      const bool on = r < total;
      const int tok = on ? r / a.group : 0, hq = sg.h * a.group + (on ? r % a.group : 0);
      const __nv_bfloat16 *qp = static_cast<const __nv_bfloat16 *>(a.q) +
                                (static_cast<long long>(sg.si.q0) + tok) * a.q_sn + hq * a.q_sh;
#pragma unroll
      for (int kk = 0; kk < MT; ++kk) {
        // bf16: piece kk/2 of 8 channels at 32 (kk/2) + 8 i, half kk%2; e4m3: piece kk/4 of 16 at 64 (kk/4) + 16 i, quarter kk%4
        const int at = FORMAT == kCacheBf16 ? 32 * (kk >> 1) + 8 * i4 + 4 * (kk & 1) : 64 * (kk >> 2) + 16 * i4 + 4 * (kk & 3);
        const uint2 w = on ? *reinterpret_cast<const uint2 *>(qp + at) : make_uint2(0, 0);
        qf[t][kk][0] = w.x;
        qf[t][kk][1] = w.y;
      }
    }
    // e4m3: codes are f16 numbers exactly, and the scores' product runs in f16.  A query row goes in times
    // the power of two that brings its largest element to [2^7, 2^8); what f16 then loses of its smaller
    // elements is under 2^-32 of that largest.  row_scale undoes it (columns 2 i, 2 i + 1).
    float row_scale[NT][2];
    if (FORMAT == kCacheE4m3) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        uint32_t top = 0;  // magnitudes of bf16 order as their bits
#pragma unroll
        for (int kk = 0; kk < MT; ++kk)
#pragma unroll
          for (int u = 0; u < 2; ++u) top = max(top, max(qf[t][kk][u] & 0x7fffu, (qf[t][kk][u] >> 16) & 0x7fffu));
#pragma unroll
        for (int o = 1; o < 4; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        // exponent field of the scale: 127 + 7 - (x - 127) for a largest element of exponent field x (infinities
        // and NaN stay what they are; a row of subnormals, far under any score, keeps a representable scale)
        const int x = min(max(static_cast<int>(top >> 7), 8), 254);
        const float sc = __int_as_float((261 - x) << 23);
#pragma unroll
        for (int kk = 0; kk < MT; ++kk)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const __half2 h = __floats2half2_rn(bf16_lo(qf[t][kk][u]) * sc, bf16_hi(qf[t][kk][u]) * sc);
            qf[t][kk][u] = *reinterpret_cast<const uint32_t *>(&h);
          }
        const float undo = __int_as_float((x - 7) << 23);  // 2^(x - 134)
        row_scale[t][0] = __shfl_sync(0xffffffffu, undo, 8 * i4);
        row_scale[t][1] = __shfl_sync(0xffffffffu, undo, 8 * i4 + 4);
      }
    }
    // ---- this warp's stages: key groups kt * 4 + warp, kt0 <= kt < kt1, that hold a key
    const int n_st = [&] {
      const int groups = (sg.si.ctx + kTokKeys - 1) / kTokKeys;  // of the sequence
      const int last = min(sg.kt1, (groups - warp + kTokWarps - 1) / kTokWarps);
      return max(last - sg.kt0, 0);
    }();
    int page_base = -1, page_reg = -1;  // lane l: the table's entry page_base + l
    unsigned valid = 0;                 // stages whose page is there
    auto issue = [&](int j) {
      const int st = j % NS;
      const int key0 = ((sg.kt0 + j) * kTokWarps + warp) * kTokKeys;
      const int pi = key0 >> a.c.page_shift;
      if (page_base < 0 || pi >= page_base + 32) {
        page_base = pi;
        const int mine = pi + lane;
        page_reg = mine < a.max_pages ? __ldg(a.table + static_cast<long long>(sg.s) * a.max_pages + mine) : -1;
      }
      const int page = __shfl_sync(0xffffffffu, page_reg, pi - page_base);
      if (static_cast<unsigned>(page) < static_cast<unsigned>(a.c.num_pages)) {
        valid |= 1u << st;
        if (lane == 0) {
          const uint32_t dst = ring + st * Lay::kStage, bar = bars + 8 * st;
          mbar_arrive_expect_tx(bar, Lay::kStage + (FORMAT == kCacheE4m3 ? 32 : 0));
          const int y = key0 & ((1 << a.c.page_shift) - 1), z = page * a.c.H + sg.h;
#pragma unroll
          for (int b = 0; b < Lay::kBoxes; ++b) {
            tma_load_3d(dst + b * kTokKeys * Lay::kBox, &tmap_k, bar, b * (Lay::kBox / Lay::kElem), y, z);
            tma_load_3d(dst + Lay::kStage / 2 + b * kTokKeys * Lay::kBox, &tmap_v, bar, b * (Lay::kBox / Lay::kElem), y,
                        z);
          }
          if (FORMAT == kCacheE4m3) {
            const long long row = paged_row(a.c, page, sg.h, key0);
            bulk_load(scales + st * 32, a.c.ke + row, 16, bar);
            bulk_load(scales + st * 32 + 16, a.c.ve + row, 16, bar);
          }
        }
      } else {
        valid &= ~(1u << st);
        if (lane == 0) atomicOr(a.err, kErrPageRange);
      }
    };
    for (int j = 0; alive && j < min(n_st, NS); ++j) issue(j);

    // ---- the bank's coefficients, from the sequence's first keys (thread per channel)
    if (tid < D) s_emax[tid] = 0;
    if (tid < kRows) s_bad[tid] = 0;
    if (BETA) {
      if (tid < D) {
        float vmax = -INFINITY, vabs = 0.f;
        const int page = sg.si.ctx > 0 ? paged_page(a, sg.s, 0) : -1;
        if (page >= 0) {
          const long long row = paged_row(a.c, page, sg.h, 0);
          const int cnt = min(kSampleKeys, sg.si.ctx);
          float v[kSampleKeys];
#pragma unroll
          for (int kk = 0; kk < kSampleKeys; ++kk) {
            const long long r = row + min(kk, cnt - 1);
            if (FORMAT == kCacheBf16) v[kk] = __bfloat162float(static_cast<const __nv_bfloat16 *>(a.c.v)[r * D + tid]);
            else v[kk] = e4m3x2_to_float2(static_cast<const uint8_t *>(a.c.v)[r * D + tid]).x * paged_scale(a.c.ve[r]);
          }
#pragma unroll
          for (int kk = 0; kk < kSampleKeys; ++kk) {
            vmax = fmaxf(vmax, v[kk]);
            vabs = fmaxf(vabs, fabsf(v[kk]));
          }
        }
        if (vabs == 0.f) {
#pragma unroll 1
          for (int i = sample_last(sg.si.ctx); i < sg.si.ctx; ++i) {
            const int p = sample_page(a, sg.s, i);
            if (p >= 0) {
              const long long r = paged_row(a.c, p, sg.h, i);
              const float x = FORMAT == kCacheBf16
                                  ? __bfloat162float(static_cast<const __nv_bfloat16 *>(a.c.v)[r * D + tid])
                                  : e4m3x2_to_float2(static_cast<const uint8_t *>(a.c.v)[r * D + tid]).x * paged_scale(a.c.ve[r]);
              vmax = fmaxf(vmax, x);
              vabs = fmaxf(vabs, fabsf(x));
            }
          }
        }
        const BankCoef c = bank_coef(beta_c, vmax, vabs);
        // element e of a lane's piece of 8 channels, lanes side by side
        const int at = Lay::kElem == 2 || !R128 ? (tid & ~63) + (tid & 7) * 8 + ((tid >> 3) & 7)
                                                : (tid & 15) * 8 + (tid >> 4);
        // coefficients of a pair of channels side by side: {b, b', s, s'}, {ic, ic', d, d'}
        float *cp = s_coef + (at & ~8) * 4 + ((at >> 3) & 1);
        cp[0] = c.b;
        cp[2] = c.s;
        cp[32] = c.ic;
        cp[34] = c.d;
        s_shift[tid] = bank_kind(c);
      }
    } else if (tid < D) {
      s_shift[tid] = INFINITY;
    }

    // keys seen by the lane's columns (rows 2 i, 2 i + 1 of each row tile)
    int lim[NT][2], lim_min = 0x7fffffff;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int r = row0 + 8 * t + 2 * i4 + u;
        lim[t][u] = r < total ? min(paged_limit(sg.si, r / a.group, a.causal), sg.si.ctx) : 0;
        if (r < total) lim_min = min(lim_min, lim[t][u]);
      }
    lim_min = __reduce_min_sync(0xffffffffu, lim_min);
    float m[NT][2], L[NT][2], acc[NT][MT][4];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      m[t][0] = m[t][1] = -INFINITY;
      L[t][0] = L[t][1] = 0.f;
#pragma unroll
      for (int u = 0; u < MT; ++u) acc[t][u][0] = acc[t][u][1] = acc[t][u][2] = acc[t][u][3] = 0.f;
    }
    const float qk_scale = a.scale * kLog2e;
    // the coefficients are there
    const bool any_dv = __syncthreads_or(BETA && tid < D && s_shift[tid] == INFINITY) != 0;  // tiny channels, beta = 0 among them
    const bool tiny = any_dv && __syncthreads_or(beta_c > 0.f && s_shift[min(tid, D - 1)] == INFINITY) != 0;

    for (int j = 0; j < n_st; ++j) {
      const int st = j % NS, key0 = ((sg.kt0 + j) * kTokWarps + warp) * kTokKeys;
      if ((valid >> st) & 1u) {
        // after a wait that gave up nothing is issued, and what is in flight is still waited for, with the limit
        if (!__all_sync(0xffffffffu, mbar_wait(bars + 8 * st, (phases >> st) & 1u, a.err, kErrWaitTma))) alive = false;
        phases ^= 1u << st;
        if (alive) {
          const uint32_t kt = ring + st * Lay::kStage, vt = kt + Lay::kStage / 2;
          // ---- S^T = K Q^T
          float sc[NT][4], s2[NT][4];  // two sums, so that every other product need not wait for the one before
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[t][i] = s2[t][i] = 0.f;
          const int r0 = key_of<R128>(g), r1 = key_of<R128>(g + 8);
          uint32_t ksc0 = 0, ksc1 = 0;
          if (FORMAT == kCacheBf16) {
#pragma unroll
            for (int p = 0; p < MT / 2; ++p) {
              const uint4 x = lds128(kt + tok_offset<Lay::kBox>(r0, 4 * p + i4));
              const uint4 y = lds128(kt + tok_offset<Lay::kBox>(r1, 4 * p + i4));
#pragma unroll
              for (int t = 0; t < NT; ++t) {
                mma_bf16(sc[t], x.x, y.x, x.y, y.y, qf[t][2 * p][0], qf[t][2 * p][1]);
                mma_bf16(s2[t], x.z, y.z, x.w, y.w, qf[t][2 * p + 1][0], qf[t][2 * p + 1][1]);
              }
            }
          } else {
            // codes go in as their values; the keys' and rows' scales multiply the scores
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ksc0) : "r"(scales + st * 32 + r0));
            asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ksc1) : "r"(scales + st * 32 + r1));
#pragma unroll
            for (int p = 0; p < MT / 4; ++p) {
              const uint4 x = lds128(kt + tok_offset<Lay::kBox>(r0, 4 * p + i4));
              const uint4 y = lds128(kt + tok_offset<Lay::kBox>(r1, 4 * p + i4));
              const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const uint2 xa = e4m3x4_to_f16(xs[u]), ya = e4m3x4_to_f16(ys[u]);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_f16(u & 1 ? s2[t] : sc[t], xa.x, ya.x, xa.y, ya.y, qf[t][4 * p + u][0], qf[t][4 * p + u][1]);
              }
            }
          }
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) sc[t][i] += s2[t][i];
          const float f0 = FORMAT == kCacheE4m3 ? qk_scale * paged_scale(ksc0) : qk_scale;
          const float f1 = FORMAT == kCacheE4m3 ? qk_scale * paged_scale(ksc1) : qk_scale;
          const bool tail = key0 + kTokKeys > lim_min;
          bool raise = false;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float c0 = FORMAT == kCacheE4m3 ? row_scale[t][0] : 1.f, c1 = FORMAT == kCacheE4m3 ? row_scale[t][1] : 1.f;
            sc[t][0] *= f0 * c0;
            sc[t][1] *= f0 * c1;
            sc[t][2] *= f1 * c0;
            sc[t][3] *= f1 * c1;
            if (tail) {
              if (key0 + r0 >= lim[t][0]) sc[t][0] = -INFINITY;
              if (key0 + r0 >= lim[t][1]) sc[t][1] = -INFINITY;
              if (key0 + r1 >= lim[t][0]) sc[t][2] = -INFINITY;
              if (key0 + r1 >= lim[t][1]) sc[t][3] = -INFINITY;
            }
            raise = raise || fmaxf(sc[t][0], sc[t][2]) > m[t][0] + kRowMaxLag || fmaxf(sc[t][1], sc[t][3]) > m[t][1] + kRowMaxLag;
          }
          if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                float mx = fmaxf(sc[t][u], sc[t][u + 2]);
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                if (mx > m[t][u] + kRowMaxLag) {
                  const float root = weight_root(m[t][u] - mx);  // (the first time there is nothing to move)
                  m[t][u] = mx;
                  L[t][u] = L[t][u] * root * root;
#pragma unroll
                  for (int c = 0; c < MT; ++c) {
                    acc[t][c][u] = acc[t][c][u] * root * root;
                    acc[t][c][u + 2] = acc[t][c][u + 2] * root * root;
                  }
                }
              }
          }
          // ---- P^T as the second operand of the second product
          uint32_t pf[NT][2];
          bool deep = false;
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const float m0 = m[t][0] == -INFINITY ? 0.f : m[t][0], m1 = m[t][1] == -INFINITY ? 0.f : m[t][1];
            const float x0 = sc[t][0] - m0, x1 = sc[t][1] - m1, x2 = sc[t][2] - m0, x3 = sc[t][3] - m1;
            if (BETA) {
              const float low = fminf(fminf(x0, x1), fminf(x2, x3));
              if (low < kDeepP) {  // seldom, and then mostly keys that are not seen
                deep = deep || (x0 < kDeepP && x0 > -INFINITY) || (x1 < kDeepP && x1 > -INFINITY) ||
                       (x2 < kDeepP && x2 > -INFINITY) || (x3 < kDeepP && x3 > -INFINITY);
              }
            }
            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1), p2 = ex2_approx(x2), p3 = ex2_approx(x3);
            L[t][0] += p0 + p2;
            L[t][1] += p1 + p3;
            pf[t][0] = transpose8x8(pack_bf16(p0, p1));
            pf[t][1] = transpose8x8(pack_bf16(p2, p3));
          }
          // ---- O^T += E^T P^T: the lane's keys are contraction indices 2 i, 2 i + 1, 2 i + 8, 2 i + 9
          int vr[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) vr[u] = key_of<R128>(2 * i4 + (u & 1) + 8 * (u >> 1));
          if (tail) {
            // a key past the sequence has no weight, but whatever its row holds must not be infinite either:
            // the stage's first key, which is there, stands in for it
#pragma unroll
            for (int u = 0; u < 4; ++u) vr[u] = key0 + vr[u] >= sg.si.ctx ? 0 : vr[u];
          }
          float vscale[4];
          if (FORMAT == kCacheE4m3) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              uint32_t b;
              asm volatile("ld.shared.u8 %0, [%1];" : "=r"(b) : "r"(scales + st * 32 + 16 + vr[u]));
              vscale[u] = paged_scale(b);
            }
          }
          constexpr int kPieces = FORMAT == kCacheBf16 ? Lay::kBoxes : 1;  // of a lane, per key
          constexpr int kPer = MT * 2 / kPieces;                           // channels of a piece (8 or 16)
          // Without a tiny channel the bank has no term d v: 136 us to 132 for 48 sequences over e4m3.  Over bf16, bound
          // by memory, one copy of the code is 2 % faster than two.
          auto mix = [&](auto tiny_head) {
            constexpr bool kTiny = decltype(tiny_head)::value;
#pragma unroll
            for (int pc = 0; pc < kPieces; ++pc) {
              uint32_t w[4][4];
              uint2 vh[4];
              if (R128) {
                const int chunk = 8 * pc + (g >> 1) + 4 * (g & 1);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const uint4 x = lds128(vt + tok_offset<Lay::kBox>(vr[u], chunk));
                  w[u][0] = x.x;
                  w[u][1] = x.y;
                  w[u][2] = x.z;
                  w[u][3] = x.w;
                }
              } else {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                  const uint2 x = lds64(vt + tok_offset<Lay::kBox>(vr[u], g >> 1) + 8 * (g & 1));
                  w[u][0] = x.x;
                  w[u][1] = x.y;
                }
              }
              const int lane_g = R128 ? (g >> 1) + 4 * (g & 1) : g;  // the piece's place among the coefficients
#pragma unroll
              for (int q = 0; q < kPer / 2; ++q) {  // pairs of channels: one row block of the product each
                uint32_t a0, a1, a2, a3;
                float lo[4], hi[4];
                if (FORMAT == kCacheE4m3 && !(q & 1)) {
#pragma unroll
                  for (int u = 0; u < 4; ++u) vh[u] = e4m3x4_to_f16(w[u][q >> 1]);
                }
                if (FORMAT == kCacheBf16) {
#pragma unroll
                  for (int u = 0; u < 4; ++u) {
                    lo[u] = bf16_lo(w[u][q]);
                    hi[u] = bf16_hi(w[u][q]);
                  }
                } else {
#pragma unroll
                  for (int u = 0; u < 4; ++u) {
                    const float2 f = __fmul2_rn(f16x2_to_float2(q & 1 ? vh[u].y : vh[u].x), make_float2(vscale[u], vscale[u]));
                    lo[u] = f.x;
                    hi[u] = f.y;
                  }
                }
                if (BETA) {
                  const float4 *cp = reinterpret_cast<const float4 *>(s_coef) + pc * 64 + 2 * q * 8 + lane_g;
                  const float4 bs = cp[0], id = cp[8];
                  const float2 b2 = make_float2(bs.x, bs.y), s2 = make_float2(bs.z, bs.w);
                  const float2 ic2 = make_float2(id.x, id.y), d2 = make_float2(id.z, id.w);
#pragma unroll
                  for (int u = 0; u < 4; ++u) {
                    const float2 e = bank_pair(b2, s2, ic2, d2, make_float2(lo[u], hi[u]), kTiny);
                    lo[u] = e.x;
                    hi[u] = e.y;
                  }
                }
                a0 = pack_bf16(lo[0], lo[1]);
                a1 = pack_bf16(hi[0], hi[1]);
                a2 = pack_bf16(lo[2], lo[3]);
                a3 = pack_bf16(hi[2], hi[3]);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma_bf16(acc[t][pc * (kPer / 2) + q], a0, a1, a2, a3, pf[t][0], pf[t][1]);
              }
            }
          };
          if (BETA && (FORMAT == kCacheBf16 || any_dv)) mix(std::true_type{});
          else mix(std::false_type{});
          // The largest |E| matters where weights come near the end of the range, or where a tiny channel
          // could leave its own: it is then found by forming the bank once more, out of the loop above, which
          // stays one stretch of code (a head with a tiny channel takes 2 to 2.5 times as long).  (Channel ch of the
          // tile, lane by lane; the keys one after the other.)
          if (BETA && (tiny || __any_sync(0xffffffffu, deep))) {
#pragma unroll 1
            for (int ch = lane; ch < D; ch += 32) {
              const int at = Lay::kElem == 2 || !R128 ? (ch & ~63) + (ch & 7) * 8 + ((ch >> 3) & 7) : (ch & 15) * 8 + (ch >> 4);
              const float *cp = s_coef + (at & ~8) * 4 + ((at >> 3) & 1);
              const BankCoef c = {cp[0], cp[2], cp[32], cp[34]};
              float emax = 0.f;
#pragma unroll 4
              for (int kx = 0; kx < kTokKeys; ++kx) {
                const int kk = min(kx, sg.si.ctx - 1 - key0);
                const uint8_t *p = smem + (vt - sbase) + tok_offset<Lay::kBox>(kk, ch * Lay::kElem >> 4) + (ch * Lay::kElem & 15);
                const float v = FORMAT == kCacheBf16
                                    ? __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(p))
                                    : e4m3x2_to_float2(*p).x * paged_scale(smem[scales - sbase + st * 32 + 16 + kk]);
                emax = fmaxf(emax, fabsf(fmaf(c.d, v, ex2_approx(fmaf(c.b, v, c.s)) + c.ic)));
              }
              if (emax >= 2.f) atomicMax(s_emax + ch, __float_as_int(emax));
            }
          }
        }
        __syncwarp();
      }
      if (alive && j + NS < n_st) issue(j + NS);
      else if (!alive) valid &= ~(1u << st);
    }

    // ---- join the warps: each leaves its rows' {m, L} and accumulators (over its own ring, which is idle)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) L[t][u] += __shfl_xor_sync(0xffffffffu, L[t][u], o);
        if (g == 0) s_stat[warp * kRows + 8 * t + 2 * i4 + u] = make_float2(m[t][u], L[t][u]);
      }
    {
      float *own = reinterpret_cast<float *>(smem + warp * NS * Lay::kStage);
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < MT; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // channel of the product's row g (e < 2) or g + 8 (e >= 2)
            const int ch = FORMAT == kCacheBf16
                               ? 64 * (c >> 2) + 8 * ((g >> 1) + 4 * (g & 1)) + 2 * (c & 3) + (e >> 1)
                               : R128 ? 16 * ((g >> 1) + 4 * (g & 1)) + 2 * c + (e >> 1) : 8 * g + 2 * c + (e >> 1);
            own[(8 * t + 2 * i4 + (e & 1)) * Lay::kRedStride + ch] = acc[t][c][e];
          }
    }
    __syncthreads();
    // ---- the segment's rows: their output, or a piece of it
    const bool whole = sg.kt0 == 0 && sg.kt1 == sg.kt_all;
    const int slot = cta * 2 + (sg.kt0 == 0 ? 1 : 0);
    float *piece = sp.pieces + static_cast<size_t>(slot) * piece_floats(kRows, D);
    const int wide = tid < D ? wide_class(s_emax[tid] >> 23) : 0;
    const OutCoef oc = out_coef(beta_c, tid < D ? s_shift[tid] : INFINITY, wide);
    for (int r = 0; r < n_rows; ++r) {
      float M = -INFINITY, Lr = 0.f, av = 0.f;
#pragma unroll
      for (int q = 0; q < kTokWarps; ++q) M = fmaxf(M, s_stat[q * kRows + r].x);
#pragma unroll
      for (int q = 0; q < kTokWarps; ++q) {
        const float2 st = s_stat[q * kRows + r];
        // a row of NaN scores has no maximum
        const float root = st.x != -INFINITY ? weight_root(st.x - M) : st.y != st.y ? 1.f : 0.f;
        Lr = fmaf(root, root * st.y, Lr);
        const float x = tid < D ? reinterpret_cast<const float *>(smem + q * NS * Lay::kStage)[r * Lay::kRedStride + tid] : 0.f;
        if (root != 0.f) av = fmaf(root, root * x, av);
      }
      const int rr = row0 + r, tok = rr / a.group, hq = sg.h * a.group + rr % a.group;
      const long long orow = (static_cast<long long>(sg.si.q0) + tok) * a.Hq + hq;
      if (whole) {
        if (tid < D) {
          bool ok = true;
          float o = 0.f;
          if (!(M == -INFINITY && Lr == 0.f)) {
            o = paged_out(oc, av * ((BETA ? kBankUnit : 1.f) / Lr), &ok);
          }
          if (!ok) {
            s_bad[r] = 1;
            o = __int_as_float(0x7fffffff);  // the mark, as bf16
          }
          static_cast<__nv_bfloat16 *>(a.out)[orow * D + tid] = __float2bfloat16_rn(o);
        }
        if (tid == 0 && a.lse != nullptr)
          a.lse[orow] = M == -INFINITY && Lr == 0.f ? -INFINITY : (M + log2f(Lr)) * kLn2;
      } else {
        if (tid < D) piece[piece_at(r, tid >> 2, D) + (tid & 3)] = av;
        if (tid == 0) {
          piece[kRows * D + 2 * r] = M;
          piece[kRows * D + 2 * r + 1] = Lr;
        }
      }
    }
    if (!whole) {
      if (tid < D) {
        piece[piece_kinds(kRows, D) + tid] = s_shift[tid];
        piece[piece_classes(kRows, D) + tid] = static_cast<float>(wide);
      }
      const bool any = __any_sync(0xffffffffu, wide != 0);
      if (lane == 0) piece[piece_wide(kRows, D) + warp] = any ? 1.f : 0.f;
    }
    fence_proxy_async_smem();  // the rings go back to the copies
    __syncthreads();
    if (whole && tid < n_rows) {
      const int rr = row0 + tid, tok = rr / a.group, hq = sg.h * a.group + rr % a.group;
      sp.exact[(static_cast<long long>(sg.si.q0) + tok) * a.Hq + hq] = s_bad[tid] != 0;
      if (s_bad[tid]) record.any_exact = 1;
    }
    if (!whole && sg.kt0 == 0 && tid == 0) {
      record.n = split_owner(walk.W, walk.G, sg.x_end - 1) - cta + 1;
      record.s = sg.s;
      record.h = sg.h;
      record.row0 = row0;
      record.rows = n_rows;
    }
  }
  __syncthreads();
  if (tid == 0) sp.records[cta] = record;
}

}  // namespace

template <int FORMAT, int D, int NT>
static cudaError_t launch_token_n(const CUtensorMap &tk, const CUtensorMap &tv, const PagedReadArgs &a,
                                  const PagedSplit &sp, const SplitShape &shape, int grid, cudaStream_t stream) {
  const size_t smem = TokLayout<FORMAT, D, NT>::kAlloc;
  auto go = [&](auto kernel) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    kernel<<<grid, kTokThreads, smem, stream>>>(tk, tv, a, sp, shape);
    return cudaGetLastError();
  };
  return a.beta ? go(paged_token_kernel<FORMAT, D, NT, true>) : go(paged_token_kernel<FORMAT, D, NT, false>);
}

int paged_token_ctas(int format, int d) { return format == kCacheBf16 && d == 128 ? 2 : 3; }
static_assert(TokLayout<kCacheBf16, 128, 1>::kCtas == 2 && TokLayout<kCacheBf16, 64, 1>::kCtas == 3 &&
                  TokLayout<kCacheE4m3, 128, 1>::kCtas == 3 && TokLayout<kCacheE4m3, 64, 1>::kCtas == 3,
              "paged_token_ctas");

cudaError_t launch_paged_token(const CUtensorMap &tk, const CUtensorMap &tv, const PagedReadArgs &a,
                               const PagedSplit &sp, const SplitShape &shape, int grid, cudaStream_t stream) {
#define FEM_TOK(F, DD)                                                                            \
  if (a.c.format == F && a.c.d == DD)                                                             \
    return shape.row_tile == 8 ? launch_token_n<F, DD, 1>(tk, tv, a, sp, shape, grid, stream)     \
                               : launch_token_n<F, DD, 2>(tk, tv, a, sp, shape, grid, stream);
  FEM_TOK(kCacheBf16, 64)
  FEM_TOK(kCacheBf16, 128)
  FEM_TOK(kCacheE4m3, 64)
  FEM_TOK(kCacheE4m3, 128)
#undef FEM_TOK
  return cudaErrorInvalidValue;
}

}  // namespace fem
