// The paged read of many new tokens per sequence: chunks of prompts and whole prompts.
//
// Bound by the tensor cores and by the exponentials that feed them.  A CTA takes
// a stretch of the line of work (fem_paged_split.cuh) in tiles of up to 256 query
// rows (whole tokens, the head's group interleaved) by 128 keys.  The 256 rows
// are two tiles of 128 that share every key tile, so the value bank is formed
// once for both and each tile's softmax runs under the other's products:
//
//   warps 0-3    bank: the key tile's values (TMA, 128-byte swizzle) become E(v) in
//                place; e4m3 keys and values are widened to bf16 from a staging
//                tile.  Rows past the sequence, or of pages that are not there,
//                become zeros
//   warps 4-7    softmax of row tile 0 (thread = row): S from TMEM, P = 2^(s - m)
//                as bf16 over the first 64 columns of S, the row sum, the lazily
//                raised maximum (and, when it moves, the accumulator's rescale);
//                the rows' queries into shared memory at an item's start, their
//                output or piece at its end
//   warps 8-11   the same for row tile 1
//   warp 12      TMA of K and V, one box per page (or part of a page) of the tile
//   warp 13      issues the products: S0 = Q0 K^T, S1 = Q1 K^T, then for
//                each tile, once its P is written, O += P E and the next S.  The
//                tensor pipe takes them in the order issued, so S of the next key
//                tile may overwrite a P whose product was issued before it, and
//                the commit of S also says that the product before it is done: the
//                softmax may then rescale O
//
// TMEM: S0 [0,128), S1 [128,256), O0 [256, 256 + D), O1 after it.
// Shared memory: Q (two tiles), K and E (two stages each), and for e4m3 a staging
// tile for K and one for V; [128 x D] tiles of bf16 in 64-column blocks of 128
// rows x 128 bytes, chunk c of row r at chunk c ^ (r & 7).
#include "fem_launch.h"
#include "fem_paged.cuh"
#include "fem_paged_split.cuh"

namespace fem {

namespace {

constexpr int kChunkThreads = 512;
constexpr int kChunkKeys = 128;
constexpr int kInvRing = 8;   // key tiles whose missing pages are remembered

template <int FORMAT, int D>
struct ChunkLayout {
  static constexpr uint32_t kTile = 128 * D * 2;
  static constexpr uint32_t kRaw = FORMAT == kCacheE4m3 ? 128 * D : 0;  // a staging tile of codes
  // bank stages: a third lets the copies of V and the bank's warps run ahead of the products (e4m3 at
  // d = 128 has no room for it beside the staging tiles, which hold a tile more themselves)
  static constexpr int kES = FORMAT == kCacheE4m3 ? 2 : 3;
  // Segments whose channels' kinds are remembered.  When the bank's warps begin a segment, the product kES
  // tiles back is done; so at most the segments of the kES tiles from that one on, their own, and one
  // before them, which a row tile out of use since may still be writing out, are alive.
  static constexpr int kSegRing = kES + 2;
  static constexpr uint32_t kQ = 0;
  static constexpr uint32_t kK = 2 * kTile;
  static constexpr uint32_t kE = kK + 2 * kTile;
  static constexpr uint32_t kRawK = kE + kES * kTile;
  static constexpr uint32_t kRawV = kRawK + kRaw;
  static constexpr uint32_t kCtl = kRawV + kRaw;
  static constexpr uint32_t kShift = kCtl;                                // [kSegRing][D]
  static constexpr uint32_t kRecord = kShift + kSegRing * D * 4;
  static constexpr uint32_t kInv = kRecord + sizeof(SplitRecord);         // [kInvRing]
  static constexpr uint32_t kWide = kInv + kInvRing * 4;                  // [kSegRing]: number (from 1) of the segment whose |E| went wide
  static constexpr uint32_t kScaleK = (kWide + kSegRing * 4 + 15) & ~15u;  // e4m3: scale bytes of the staged keys, then values
  static constexpr uint32_t kScaleV = kScaleK + (FORMAT == kCacheE4m3 ? 128 : 0);
  static constexpr uint32_t kBars = (kScaleV + (FORMAT == kCacheE4m3 ? 128 : 0) + 7) & ~7u;
  static constexpr uint32_t kNumBars = 25;
  static constexpr uint32_t kTmem = kBars + kNumBars * 8;
  static constexpr uint32_t kAbort = kTmem + 4;
  static constexpr uint32_t kScan = (kAbort + 4 + 7) & ~7u;
  static constexpr uint32_t kBytes = kScan + sizeof(SplitScan<kChunkThreads>);
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

enum : int {
  kCbQ = 0,        // + row tile: its queries are in shared memory (128 arrivals)
  kCbKFull = 2,    // + stage: K as bf16 (TMA, or 128 arrivals of the bank warps)
  kCbKEmpty = 4,   // + stage: both S of the tile are done
  kCbVFull = 6,    // + bank stage: V as TMA brought it (bf16)
  kCbEFull = 9,    // + bank stage: the bank (128 arrivals)
  kCbEEmpty = 12,  // + bank stage: both P E of the tile are done
  kCbRawKFull = 15,
  kCbRawVFull = 16,
  kCbRawKEmpty = 17,  // 128 arrivals
  kCbRawVEmpty = 18,
  kCbS = 19,       // + row tile: S is in TMEM
  kCbP = 21,       // + row tile: P is in TMEM (128 arrivals)
  kCbO = 23,       // every product of the segment is done
  kCbDone = 24,    // every product this CTA issued is done
};

__device__ __forceinline__ bool chunk_wait(uint32_t bar, uint32_t parity, unsigned *err, unsigned code,
                                           volatile int *abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = global_timer_ns();
  while (true) {
    if (mbar_try_wait_sleep(bar, parity, 200000u)) return true;
    if (*abort_flag) return false;
    if (global_timer_ns() - t0 > kWaitLimitNs) {
      atomicOr(err, code);
      *abort_flag = 1;
      return false;
    }
  }
}

// True in one thread of the warp, always the same one.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ float bf16_lo(uint32_t w) { return __int_as_float(static_cast<int>(w << 16)); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __int_as_float(static_cast<int>(w & 0xffff0000u)); }

// Rows of a segment's two row tiles.
struct ChunkRows {
  int tok0, rows, tiles;  // first token, rows, row tiles in use (1 or 2)
};
__device__ __forceinline__ ChunkRows chunk_rows(const SplitSeg &g, int group, const SplitShape &sh) {
  ChunkRows r;
  r.tok0 = g.r * sh.tok;
  r.rows = min(sh.tok, g.si.n - r.tok0) * group;
  r.tiles = r.rows > 128 ? 2 : 1;
  return r;
}

template <int FORMAT, int D, bool BETA>
__global__ void __launch_bounds__(kChunkThreads, 1)
    paged_chunk_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                       const PagedReadArgs a, const PagedSplit sp, const SplitShape shape, int box_shift) {
  using Lay = ChunkLayout<FORMAT, D>;
  constexpr bool kCodes = FORMAT == kCacheE4m3;
  constexpr unsigned kES = Lay::kES, kSegRing = Lay::kSegRing;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  const uint32_t bars = sbase + Lay::kBars;
#define FEM_CB(i) (bars + 8u * static_cast<uint32_t>(i))
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + Lay::kAbort);
  SplitScan<kChunkThreads> &scan = *reinterpret_cast<SplitScan<kChunkThreads> *>(smem + Lay::kScan);
  float *s_shift = reinterpret_cast<float *>(smem + Lay::kShift);
  volatile unsigned *s_inv = reinterpret_cast<volatile unsigned *>(smem + Lay::kInv);
  volatile int *s_wide = reinterpret_cast<volatile int *>(smem + Lay::kWide);
  const int box_rows = 1 << box_shift;
  const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

  grid_dep_launch_dependents();
  const int cta = blockIdx.x;
  SplitWalk walk;
  SplitRecord &record = *reinterpret_cast<SplitRecord *>(smem + Lay::kRecord);
  if (tid == 0) record = SplitRecord{};
  if (!split_begin(a, shape, cta, gridDim.x, scan, walk)) {
    if (tid == 0) sp.records[cta] = SplitRecord{};
    return;
  }
  if (warp == 12) {
    tmem_alloc(sbase + Lay::kTmem, 512);
    tmem_relinquish();
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(FEM_CB(kCbQ + i), 128);
      mbar_init(FEM_CB(kCbKFull + i), kCodes ? 128 : 1);
      mbar_init(FEM_CB(kCbKEmpty + i), 1);
      mbar_init(FEM_CB(kCbS + i), 1);
      mbar_init(FEM_CB(kCbP + i), 128);
    }
    for (unsigned i = 0; i < kES; ++i) {
      mbar_init(FEM_CB(kCbVFull + i), 1);
      mbar_init(FEM_CB(kCbEFull + i), 128);
      mbar_init(FEM_CB(kCbEEmpty + i), 1);
    }
    mbar_init(FEM_CB(kCbRawKFull), 1);
    mbar_init(FEM_CB(kCbRawVFull), 1);
    mbar_init(FEM_CB(kCbRawKEmpty), 128);
    mbar_init(FEM_CB(kCbRawVEmpty), 128);
    mbar_init(FEM_CB(kCbO), 1);
    mbar_init(FEM_CB(kCbDone), 1);
    fence_mbar_init();
    *abort_flag = 0;
    for (unsigned i = 0; i < kSegRing; ++i) s_wide[i] = 0;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + Lay::kTmem);
  SplitSeg sg;

  // The block's registers are 512 x 128; the softmax warps take 168 each, the bank's 104, the others 72:
  // 256 x 168 + 128 x 104 + 128 x 72 = 512 x 128.
  if (warp >= 12) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
  if (warp == 12) {
    // ------------------------------------------------------------ TMA of K and V
    const int boxes = kChunkKeys / box_rows;
    constexpr int kCols = kCodes ? (D < 128 ? D : 128) : 64;  // elements of a box's row
    constexpr int kBlocks = D / kCols;
    const uint32_t box_bytes = static_cast<uint32_t>(box_rows) * kCols * (kCodes ? 1 : 2);
    unsigned n = 0;  // key tiles so far
    bool ok = true;
    while (ok && walk.next(a, shape, sg)) {
      for (int kt = sg.kt0; ok && kt < sg.kt1; ++kt, ++n) {
        const unsigned st = n & 1, use = n >> 1, es = n % kES, euse = n / kES;
        // lane b: box b of the tile
        const int key = kt * kChunkKeys + lane * box_rows;
        const bool wanted = lane < boxes && key < sg.si.ctx;
        const int page = wanted ? paged_page(a, sg.s, key) : -1;
        const unsigned there = __ballot_sync(0xffffffffu, page >= 0), want = __ballot_sync(0xffffffffu, wanted);
        if (lane == 0) s_inv[n % kInvRing] = want & ~there;
        __syncwarp();
        const uint32_t bytes = __popc(there) * (box_bytes * kBlocks + (kCodes ? box_rows : 0));
        const long long row = page >= 0 ? paged_row(a.c, page, sg.h, key) : 0;
        const int y = key & ((1 << a.c.page_shift) - 1), z = page * a.c.H + sg.h;
        auto load = [&](const CUtensorMap *map, uint32_t dst, uint32_t bar, uint32_t sc, const uint8_t *exps) {
          if (lane == 0) mbar_arrive_expect_tx(bar, bytes);
          __syncwarp();
          if (page >= 0) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
              tma_load_3d(dst + b * (128 * kCols * (kCodes ? 1 : 2)) + lane * box_bytes, map, bar, b * kCols, y, z);
            if (kCodes) bulk_load(sc + lane * box_rows, exps + row, box_rows, bar);
          }
        };
        if (kCodes) {
          if (n > 0) ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbRawKEmpty), (n - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (ok) load(&tmap_k, sbase + Lay::kRawK, FEM_CB(kCbRawKFull), sbase + Lay::kScaleK, a.c.ke);
          if (ok && n > 0) ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbRawVEmpty), (n - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (ok) load(&tmap_v, sbase + Lay::kRawV, FEM_CB(kCbRawVFull), sbase + Lay::kScaleV, a.c.ve);
        } else {
          if (use > 0) ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbKEmpty + st), (use - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (ok) load(&tmap_k, sbase + Lay::kK + st * Lay::kTile, FEM_CB(kCbKFull + st), 0, nullptr);
          if (ok && euse > 0) ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbEEmpty + es), (euse - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (ok) load(&tmap_v, sbase + Lay::kE + es * Lay::kTile, FEM_CB(kCbVFull + es), 0, nullptr);
        }
      }
    }
    if (!ok && lane == 0) {
      // another role gave up: the copies in flight land before the block ends (the last few tiles')
      for (unsigned t = n + 1 > kES ? n + 1 - kES : 0; t <= n; ++t) {
        if (kCodes) {
          mbar_wait_for(FEM_CB(kCbRawKFull), t & 1, a.err, kErrWaitTma, 100000000ull);
          mbar_wait_for(FEM_CB(kCbRawVFull), t & 1, a.err, kErrWaitTma, 100000000ull);
        } else {
          mbar_wait_for(FEM_CB(kCbKFull + (t & 1)), (t >> 1) & 1, a.err, kErrWaitTma, 100000000ull);
          mbar_wait_for(FEM_CB(kCbVFull + t % kES), (t / kES) & 1, a.err, kErrWaitTma, 100000000ull);
        }
      }
    }
  } else if (warp == 13) {
    // ------------------------------------------------------------ products
    // The whole warp walks the loop and one elected thread issues: the loop then stays uniform, and the
    // operands' descriptors are sums of per-tile bases and constants in uniform registers.  With one
    // thread in the loop alone its address arithmetic, between the other warps' instructions, took 6000
    // cycles a key tile, and the tensor pipe was idle for three quarters of them.
    constexpr uint32_t idesc_s = idesc_f16(128, 128, true, false);
    constexpr uint32_t idesc_o = idesc_f16(128, D, true, true);
    const uint64_t desc_q = smem_desc_sw128(sbase + Lay::kQ, 16, 1024), desc_k = smem_desc_sw128(sbase + Lay::kK, 16, 1024);
    const uint64_t desc_e = smem_desc_sw128(sbase + Lay::kE, 16384, 1024);
    const bool leader = elect_one();
    unsigned n = 0, np0 = 0, np1 = 0, seg = 0;  // key tiles, P of each row tile, segments so far
    bool ok = true;
    auto wait = [&](int bar, unsigned parity, unsigned code) {
      return __all_sync(0xffffffffu, chunk_wait(FEM_CB(bar), parity & 1, a.err, code, abort_flag)) != 0;
    };
    while (ok && walk.next(a, shape, sg)) {
      const int tiles = chunk_rows(sg, a.group, shape).tiles, nk = sg.kt1 - sg.kt0;
      // both row tiles' warps arrive whether their tile is in use or not: the phases stay together
      ok = wait(kCbQ, seg, kErrWaitMma) && wait(kCbQ + 1, seg, kErrWaitMma);
      for (int k = 0; ok && k <= nk; ++k) {
        const unsigned i = n + k, e = i - 1;  // this key tile, and the one whose bank is used
        if (k < nk) {
          if (!(ok = wait(kCbKFull + (i & 1), i >> 1, kErrWaitTma))) break;
        }
        if (k > 0) {
          if (!(ok = wait(kCbEFull + e % kES, e / kES, kErrWaitMma))) break;
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (t >= tiles) break;
          if (k > 0) {
            // O_t += P_t E of key tile e
            if (!(ok = wait(kCbP + t, t ? np1 : np0, kErrWaitMma))) break;
            if (t) ++np1; else ++np0;
            tc_fence_after_sync();
            const uint64_t de = desc_e + (e % kES) * (Lay::kTile >> 4);
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < 8; ++kk)
                mma_f16_ts(tmem + 256 + t * D, tmem + t * 128 + kk * 8, de + ((kk * 2048) >> 4), idesc_o,
                           (k > 1 || kk > 0) ? 1u : 0u);
              if (t == tiles - 1) mma_commit(FEM_CB(kCbEEmpty + e % kES));
            }
          }
          if (k < nk) {
            tc_fence_after_sync();
            const uint64_t dq = desc_q + t * (Lay::kTile >> 4), dk = desc_k + (i & 1) * (Lay::kTile >> 4);
            if (leader) {
#pragma unroll
              for (int kk = 0; kk < D / 16; ++kk) {
                const uint32_t off = ((kk >> 2) * 16384 + (kk & 3) * 32) >> 4;
                mma_f16_ss(tmem + t * 128, dq + off, dk + off, idesc_s, kk > 0 ? 1u : 0u);
              }
              mma_commit(FEM_CB(kCbS + t));
              if (t == tiles - 1) mma_commit(FEM_CB(kCbKEmpty + (i & 1)));
            }
          }
        }
      }
      if (ok && leader) mma_commit(FEM_CB(kCbO));
      n += nk;
      ++seg;
    }
    if (leader) {
      mma_commit(FEM_CB(kCbDone));
      // nothing may be in flight when TMEM is freed
      mbar_wait(FEM_CB(kCbDone), 0, a.err, kErrWaitMma);
    }
  } else if (warp < 4) {
    // ------------------------------------------------------------ the bank
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    const int rl = tid & 7, cc = tid >> 3;  // rows rl, rl + 8, ...; 16-byte chunk cc (of bf16)
    constexpr int kChunks = D / 8;          // per row: 16 at D = 128, 8 at D = 64 (then two row groups)
    const int col = cc % kChunks, r_first = rl + 8 * (cc / kChunks);
    constexpr int kRowStep = 8 * (16 / kChunks), kRowsEach = 128 / kRowStep;
    constexpr int kBatch = 4;
    // the thread's 8 codes of a row in a staging tile
    auto raw_offset = [&](int r) {
      return D == 128 ? sw128_offset(r, col >> 1) + 8 * (col & 1) : r * 64 + (((col >> 1) ^ ((r >> 1) & 3)) << 4) + 8 * (col & 1);
    };
    float2 cb[4], cs[4], ci[4], cd[4];  // the thread's channels, in pairs
    int last_s = -1, last_h = -1;
    unsigned n = 0, seg = 0;
    bool ok = true;
    while (ok && walk.next(a, shape, sg)) {
      // coefficients of the thread's 8 channels, from the sequence's first values
      if (BETA && (sg.s != last_s || sg.h != last_h)) {
        last_s = sg.s;
        last_h = sg.h;
        float vmax[8], vabs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          vmax[e] = -INFINITY;
          vabs[e] = 0.f;
        }
        const int page = sg.si.ctx > 0 ? paged_page(a, sg.s, 0) : -1;
        if (page >= 0) {
          const long long row = paged_row(a.c, page, sg.h, 0);
          const int cnt = min(kSampleKeys, sg.si.ctx);
#pragma unroll 4
          for (int kk = 0; kk < cnt; ++kk) {
            float v[8];
            if (kCodes) {
              const uint2 w = *reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(a.c.v) + (row + kk) * D + col * 8);
              const float sc = paged_scale(a.c.ve[row + kk]);
              const uint32_t x[4] = {w.x & 0xffffu, w.x >> 16, w.y & 0xffffu, w.y >> 16};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float2 f = e4m3x2_to_float2(x[e]);
                v[2 * e] = f.x * sc;
                v[2 * e + 1] = f.y * sc;
              }
            } else {
              const uint4 w = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.c.v) + (row + kk) * D + col * 8);
              const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                v[2 * e] = bf16_lo(x[e]);
                v[2 * e + 1] = bf16_hi(x[e]);
              }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              vmax[e] = fmaxf(vmax[e], v[e]);
              vabs[e] = fmaxf(vabs[e], fabsf(v[e]));
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          const float *bp = a.beta + static_cast<long long>(sg.h) * D + col * 8 + e;
          const BankCoef x = bank_coef(__ldg(bp), vmax[e], vabs[e]), y = bank_coef(__ldg(bp + 1), vmax[e + 1], vabs[e + 1]);
          cb[e / 2] = make_float2(x.b, y.b);
          cs[e / 2] = make_float2(x.s, y.s);
          ci[e / 2] = make_float2(x.ic, y.ic);
          cd[e / 2] = make_float2(x.d, y.d);
        }
      }
      float emax = 0.f;
      bool wrote = false;  // this segment's shifts, once its first stage is free
      for (int kt = sg.kt0; ok && kt < sg.kt1; ++kt, ++n) {
        const unsigned st = n & 1, use = n >> 1, es = n % kES, euse = n / kES;
        const int k0 = kt * kChunkKeys;
        uint8_t *tE = smem + Lay::kE + es * Lay::kTile;
        if (kCodes) {
          // K: codes to bf16
          ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbRawKFull), n & 1, a.err, kErrWaitTma, abort_flag));
          if (ok && use > 0) ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbKEmpty + st), (use - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (!ok) break;
        } else {
          ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbVFull + es), euse & 1, a.err, kErrWaitTma, abort_flag));
          if (!ok) break;
        }
        const unsigned inv = s_inv[n % kInvRing];
        const bool ragged = inv != 0 || k0 + kChunkKeys > sg.si.ctx;
        auto gone = [&](int r) { return k0 + r >= sg.si.ctx || ((inv >> (r >> box_shift)) & 1u); };
        if (kCodes) {
          uint8_t *tK = smem + Lay::kK + st * Lay::kTile;
          const uint8_t *raw = smem + Lay::kRawK;
#pragma unroll 1
          for (int i0 = 0; i0 < kRowsEach; i0 += kBatch) {
            uint2 w[kBatch];
            float sc[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const int r = r_first + kRowStep * (i0 + u);
              w[u] = *reinterpret_cast<const uint2 *>(raw + raw_offset(r));
              sc[u] = paged_scale(smem[Lay::kScaleK + r]);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const int r = r_first + kRowStep * (i0 + u);
              const float2 s2 = make_float2(sc[u], sc[u]);
              const float2 f0 = __fmul2_rn(e4m3x2_to_float2(w[u].x & 0xffffu), s2), f1 = __fmul2_rn(e4m3x2_to_float2(w[u].x >> 16), s2);
              const float2 f2 = __fmul2_rn(e4m3x2_to_float2(w[u].y & 0xffffu), s2), f3 = __fmul2_rn(e4m3x2_to_float2(w[u].y >> 16), s2);
              uint4 y = make_uint4(pack_bf16(f0.x, f0.y), pack_bf16(f1.x, f1.y), pack_bf16(f2.x, f2.y), pack_bf16(f3.x, f3.y));
              if (ragged && gone(r)) y = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4 *>(tK + (col >> 3) * 16384 + sw128_offset(r, col & 7)) = y;
            }
          }
          fence_proxy_async_smem();
          mbar_arrive(FEM_CB(kCbKFull + st));
          mbar_arrive(FEM_CB(kCbRawKEmpty));
          ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbRawVFull), n & 1, a.err, kErrWaitTma, abort_flag));
          if (ok && euse > 0) ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbEEmpty + es), (euse - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (!ok) break;
        }
        if (!wrote) {
          // the stage is free: see kSegRing
          wrote = true;
          if (rl == 0 && cc < kChunks) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              s_shift[(seg % kSegRing) * D + col * 8 + e] =
                  BETA ? bank_kind(e & 1 ? BankCoef{cb[e / 2].y, cs[e / 2].y, ci[e / 2].y, cd[e / 2].y}
                                         : BankCoef{cb[e / 2].x, cs[e / 2].x, ci[e / 2].x, cd[e / 2].x})
                       : INFINITY;
          }
        }
        if (BETA || kCodes || ragged) {
          // rows in batches: their loads leave together (a store to the tile would hold the next row's back)
#pragma unroll 1
          for (int i0 = 0; i0 < kRowsEach; i0 += kBatch) {
            uint4 w[kBatch];
            float sc[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const int r = r_first + kRowStep * (i0 + u);
              if (kCodes) {
                const uint2 x = *reinterpret_cast<const uint2 *>(smem + Lay::kRawV + raw_offset(r));
                w[u] = make_uint4(x.x & 0xffffu, x.x >> 16, x.y & 0xffffu, x.y >> 16);
                sc[u] = paged_scale(smem[Lay::kScaleV + r]);
              } else {
                w[u] = *reinterpret_cast<const uint4 *>(tE + (col >> 3) * 16384 + sw128_offset(r, col & 7));
              }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const int r = r_first + kRowStep * (i0 + u);
              const uint32_t x[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
              uint32_t y[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float2 v = kCodes ? __fmul2_rn(e4m3x2_to_float2(x[e]), make_float2(sc[u], sc[u]))
                                  : make_float2(bf16_lo(x[e]), bf16_hi(x[e]));
                if (BETA) {
                  v = bank_pair(cb[e], cs[e], ci[e], cd[e], v);
                  emax = fmaxf(fmaxf(emax, fabsf(v.x)), fabsf(v.y));
                }
                y[e] = pack_bf16(v.x, v.y);
              }
              if (ragged && gone(r)) y[0] = y[1] = y[2] = y[3] = 0;
              *reinterpret_cast<uint4 *>(tE + (col >> 3) * 16384 + sw128_offset(r, col & 7)) = make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
          if (BETA && emax > kWideE) s_wide[seg % kSegRing] = static_cast<int>(seg + 1);
        }
        fence_proxy_async_smem();
        mbar_arrive(FEM_CB(kCbEFull + es));
        if (kCodes) mbar_arrive(FEM_CB(kCbRawVEmpty));
      }
      ++seg;
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------ softmax, queries and output of a row tile
    asm volatile("setmaxnreg.inc.sync.aligned.u32 168;");
    const int t = (warp >> 2) - 1, r = tid & 127;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + t * 128 + lane_off, tO = tmem + 256 + t * D + lane_off;
    const float qk_scale = a.scale * kLog2e;
    unsigned n = 0, ns = 0, seg = 0;
    // The thread's row of a segment: whether there is one, its place in the output, the keys it sees.
    struct Row {
      bool on;
      int lim;
      long long qrow, orow;
      int hq;
    };
    auto row_of = [&](const SplitSeg &g, const ChunkRows &cr) {
      const int ir = t * 128 + r;
      Row w;
      w.on = ir < cr.rows;
      const int tok = cr.tok0 + (w.on ? ir / a.group : 0);
      w.hq = g.h * a.group + (w.on ? ir % a.group : 0);
      w.qrow = static_cast<long long>(g.si.q0) + tok;
      w.orow = w.qrow * a.Hq + w.hq;
      w.lim = w.on ? min(paged_limit(g.si, tok, a.causal), g.si.ctx) : 0;
      return w;
    };
    // The row's query into shared memory, and the arrival that lets the segment's products start.
    auto load_q = [&](const Row &w, bool used) {
      if (used) {
        uint8_t *tQ = smem + Lay::kQ + t * Lay::kTile;
        const uint4 *qp = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.q) + w.qrow * a.q_sn + w.hq * a.q_sh);
        uint4 x[D / 8];
#pragma unroll
        for (int c = 0; c < D / 8; ++c) x[c] = w.on ? __ldg(qp + c) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < D / 8; ++c) *reinterpret_cast<uint4 *>(tQ + (c >> 3) * 16384 + sw128_offset(r, c & 7)) = x[c];
        fence_proxy_async_smem();
      }
      mbar_arrive(FEM_CB(kCbQ + t));
    };
    bool ok = walk.next(a, shape, sg);
    ChunkRows cr;
    Row w;
    if (ok) {
      cr = chunk_rows(sg, a.group, shape);
      w = row_of(sg, cr);
      load_q(w, t < cr.tiles);
    }
    while (ok) {
      const int nk = sg.kt1 - sg.kt0, ir = t * 128 + r;
      const int lim = w.lim;
      float m = -INFINITY, L = 0.f;
      if (t < cr.tiles) {
        for (int k = 0; k < nk; ++k, ++ns) {
          ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbS + t), ns & 1, a.err, kErrWaitMma, abort_flag));
          if (!ok) break;
          tc_fence_after_sync();
          uint32_t sr[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(tS + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&sr[c * 32]));
          tmem_ld_wait();
          float *s = reinterpret_cast<float *>(sr);
          const int k0 = (sg.kt0 + k) * kChunkKeys;
          const unsigned inv = s_inv[(n + k) % kInvRing];
          if (__any_sync(0xffffffffu, k0 + kChunkKeys > lim) || inv) {
#pragma unroll
            for (int j = 0; j < 128; ++j) s[j] = k0 + j < lim ? s[j] : -INFINITY;
            if (inv) {
#pragma unroll
              for (int j = 0; j < 128; ++j) s[j] = (inv >> (j >> box_shift)) & 1u ? -INFINITY : s[j];
            }
          }
          float mx[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) mx[u] = fmax3(s[u], s[u + 8], s[u + 16]);
#pragma unroll
          for (int j = 24; j < 120; j += 16)
#pragma unroll
            for (int u = 0; u < 8; ++u) mx[u] = fmax3(mx[u], s[j + u], s[j + 8 + u]);
#pragma unroll
          for (int u = 0; u < 8; ++u) mx[u] = fmaxf(mx[u], s[120 + u]);
          const float tmax = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7])) * qk_scale;
          float alpha = 1.f;
          if (tmax > m + kRowMaxLag) {
            alpha = ex2_approx(m - tmax);  // 0 the first time
            m = tmax;
            L *= alpha;
          }
          if (k > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
            // O holds the products of the key tiles before (see the issue order)
#pragma unroll 1
            for (int c = 0; c < D / 32; ++c) {
              uint32_t v[32];
              tmem_ld32(tO + c * 32, v);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * alpha);
              tmem_st32(tO + c * 32, v);
            }
            tmem_st_wait();
          }
          const float mz = m == -INFINITY ? 0.f : m;
          const float2 scale2 = make_float2(qk_scale, qk_scale), negm2 = make_float2(-mz, -mz);
          float2 ls[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) ls[u] = make_float2(0.f, 0.f);
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 x = __ffma2_rn(make_float2(s[c * 32 + 2 * i], s[c * 32 + 2 * i + 1]), scale2, negm2);
              const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
              ls[i & 3] = __fadd2_rn(ls[i & 3], e);
              p[i] = pack_bf16(e.x, e.y);
            }
            tmem_st16(tS + c * 16, p);
          }
          L += (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y) + (ls[2].x + ls[2].y) + (ls[3].x + ls[3].y);
          tmem_st_wait();
          tc_fence_before_sync();
          mbar_arrive(FEM_CB(kCbP + t));
        }
        if (!ok) break;
      }
      // The next segment's queries, before this one's output: its S then wait for nothing.  The last S
      // of this row tile is done.  A row tile out of use has seen none, and first waits for the segment's
      // end, so that its arrivals stay within one segment of the products.
      SplitSeg sg2;
      ChunkRows cr2;
      Row w2;
      const bool more = walk.next(a, shape, sg2);
      if (more) {
        cr2 = chunk_rows(sg2, a.group, shape);
        w2 = row_of(sg2, cr2);
        if (t < cr.tiles) load_q(w2, t < cr2.tiles);
      }
      ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbO), seg & 1, a.err, kErrWaitMma, abort_flag));
      if (!ok) break;
      tc_fence_after_sync();
      if (more && t >= cr.tiles) load_q(w2, t < cr2.tiles);
      if (t < cr.tiles) {
        // ---- the row's output, or its piece
        const bool whole = sg.kt0 == 0 && sg.kt1 == sg.kt_all;
        const bool wide = BETA && s_wide[seg % kSegRing] == static_cast<int>(seg + 1);
        const float *shift = s_shift + (seg % kSegRing) * D;
        float *piece = sp.pieces + static_cast<size_t>(cta * 2 + (sg.kt0 == 0 ? 1 : 0)) * piece_floats(256, D);
        const bool empty = m == -INFINITY && L == 0.f;
        const float inv_l = empty ? 0.f : 1.f / L;
        bool good = true;
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
          uint32_t v[32];
          tmem_ld32(tO + c * 32, v);
          tmem_ld_wait();
          if (whole) {
            // lane l has channel 32 c + l's coefficients; every row needs all of them
            const OutCoef oc = out_coef(BETA ? __ldg(a.beta + static_cast<long long>(sg.h) * D + c * 32 + lane) : 0.f,
                                        shift[c * 32 + lane], wide);
            uint32_t o[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              float x[2];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const float av = __uint_as_float(v[2 * i + u]) * inv_l;
                if (BETA) {
                  OutCoef k;
                  k.g = __shfl_sync(0xffffffffu, oc.g, 2 * i + u);
                  k.z = __shfl_sync(0xffffffffu, oc.z, 2 * i + u);
                  k.y = __shfl_sync(0xffffffffu, oc.y, 2 * i + u);
                  k.w = __shfl_sync(0xffffffffu, oc.w, 2 * i + u);
                  k.lo = __shfl_sync(0xffffffffu, oc.lo, 2 * i + u);
                  bool fine;
                  x[u] = paged_out(k, av, &fine);
                  good = good && fine;
                } else {
                  x[u] = av;
                  good = good && fabsf(av) < kMostA;
                }
              }
              o[i] = empty ? 0u : pack_bf16(x[0], x[1]);
            }
            if (!w.on) continue;
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + w.orow * D + c * 32);
#pragma unroll
            for (int i = 0; i < 4; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
          } else if (w.on) {
            float4 *dst = reinterpret_cast<float4 *>(piece + static_cast<size_t>(ir) * D + c * 32);
#pragma unroll
            for (int i = 0; i < 8; ++i)
              dst[i] = make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]),
                                   __uint_as_float(v[4 * i + 3]));
          }
        }
        if (w.on) {
          if (whole) {
            if (a.lse != nullptr) a.lse[w.orow] = empty ? -INFINITY : (m + log2f(L)) * kLn2;
          } else {
            piece[256 * D + 2 * ir] = m;
            piece[256 * D + 2 * ir + 1] = L;
          }
          if (whole) {
            const bool exact = !good && !empty;
            sp.exact[w.orow] = exact;
            if (exact) record.any_exact = 1;
          }
        }
        if (!whole && t == 0) {
          if (r < D) piece[256 * D + 512 + r] = shift[r];
          if (r == 0) {
            piece[256 * D + 512 + D] = wide ? 1.f : 0.f;
            if (sg.kt0 == 0) {
              record.n = split_owner(walk.W, walk.G, sg.x_end - 1) - cta + 1;
              record.s = sg.s;
              record.h = sg.h;
              record.row0 = cr.tok0 * a.group;
              record.rows = cr.rows;
            }
          }
        }
        tc_fence_before_sync();  // the next segment's P E overwrite O, after this thread's next P arrives
      }
      n += nk;
      ++seg;
      if (!more) break;
      sg = sg2;
      cr = cr2;
      w = w2;
    }
  }

  tc_fence_before_sync();
  __syncthreads();
  if (tid == 0) sp.records[cta] = record;
  if (warp == 12) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
#undef FEM_CB
}

}  // namespace

template <int FORMAT, int D>
static cudaError_t launch_chunk_d(const CUtensorMap &tk, const CUtensorMap &tv, const PagedReadArgs &a,
                                  const PagedSplit &sp, const SplitShape &shape, int grid, int box_shift,
                                  cudaStream_t stream) {
  const size_t smem = ChunkLayout<FORMAT, D>::kBytes;
  auto go = [&](auto kernel) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
    if (e != cudaSuccess) return e;
    kernel<<<grid, kChunkThreads, smem, stream>>>(tk, tv, a, sp, shape, box_shift);
    return cudaGetLastError();
  };
  return a.beta ? go(paged_chunk_kernel<FORMAT, D, true>) : go(paged_chunk_kernel<FORMAT, D, false>);
}

cudaError_t launch_paged_chunk(const CUtensorMap &tk, const CUtensorMap &tv, const PagedReadArgs &a,
                               const PagedSplit &sp, const SplitShape &shape, int grid, int box_rows,
                               cudaStream_t stream) {
  int box_shift = 4;
  while ((1 << box_shift) < box_rows) ++box_shift;
  if ((1 << box_shift) != box_rows || box_rows > kChunkKeys) return cudaErrorInvalidValue;
  if (shape.row_tile != 256 || (1 << shape.key_shift) != kChunkKeys || shape.tok < 1) return cudaErrorInvalidValue;
  if (a.c.format == kCacheBf16)
    return a.c.d == 64 ? launch_chunk_d<kCacheBf16, 64>(tk, tv, a, sp, shape, grid, box_shift, stream)
                       : launch_chunk_d<kCacheBf16, 128>(tk, tv, a, sp, shape, grid, box_shift, stream);
  return a.c.d == 64 ? launch_chunk_d<kCacheE4m3, 64>(tk, tv, a, sp, shape, grid, box_shift, stream)
                     : launch_chunk_d<kCacheE4m3, 128>(tk, tv, a, sp, shape, grid, box_shift, stream);
}

}  // namespace fem
