// The paged read of many new tokens per sequence: chunks of prompts and whole prompts.
//
// Bound by the tensor cores and by the exponentials that feed them.  A CTA takes
// a stretch of the line of work (fem_paged_split.cuh) in tiles of up to 256 query
// rows (whole tokens, the head's group interleaved) by 128 keys.  The 256 rows
// are two tiles of 128 that share every key tile, so the value bank is formed
// once for both and each tile's softmax runs under the other's products:
//
//   warps 0-7    bank: the key tile's values (TMA, 128-byte swizzle) become E(v) in
//                place; e4m3 keys and values are widened to bf16 from a staging
//                tile.  Rows past the sequence, or of pages that are not there,
//                become zeros
//   warps 8-15   softmax of row tile 0, two threads per row (64 keys each): S from
//                TMEM, P = 2^(s - m) as bf16 over the first 32 of their 64 columns of S,
//                the row's sum; the rows' queries into shared memory at an item's start,
//                their output or piece at its end.  A tile's chain S, softmax, P E, S is
//                what the pace hangs on.  The maximum m need only keep P in range, and
//                bf16's is fp32's: it is found once, in a segment's first tile, and raised
//                when a tile's weights sum to over 2^40, at the tile after (then O is
//                rescaled), so that the two threads never wait for each other in between
//   warps 16-23  the same for row tile 1
//   warp 24      TMA of K and V, one box per page (or part of a page) of the tile
//   warp 25      issues the products: S0 = Q0 K^T, S1 = Q1 K^T, then for
//                each tile, once its P is written, O += P E and the next S.  The
//                tensor pipe takes them in the order issued, so S of the next key
//                tile may overwrite a P whose product was issued before it, and
//                the commit of S also says that the product before it is done: the
//                softmax may then rescale O
//
// A causal prompt of 8192, 16 heads of 128, bf16: 281 us with the join, 979 TFLOP/s
// (tensor pipe 48 % busy, issue slots 60 %; without the value bank 207 us before the
// join); the bank's OR of what it forms, which finds the wide channels, takes 10 us.
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

constexpr int kChunkThreads = 896;
constexpr int kChunkKeys = 128;
constexpr int kBankThreads = 256;
constexpr float kAskSum = 1.0995116e12f;  // 2^40
constexpr float kLeastSum = 0.25f;
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
  static constexpr uint32_t kShift = kCtl;                       // channels' kinds, 16 bits, [kSegRing][D]
  // classes of the channels' |E|, four of 4 bits in 16: [kSegRing], one for each group of the bank's threads
  // that has the channel, [D / 4]
  static constexpr int kParts = 128 / D;
  static constexpr uint32_t kClass = kShift + kSegRing * D * 2;
  static constexpr uint32_t kRow = (kClass + kSegRing * kParts * (D / 4) * 2 + 15) & ~15u;  // what the threads of a row exchange: 4 bytes per row
  static constexpr uint32_t kAsk = kRow + 2 * 128 * 4;         // per pair of warps and half: see the softmax
  static constexpr uint32_t kRecord = kAsk + 16 * 4;
  static constexpr uint32_t kInv = kRecord + sizeof(SplitRecord);         // [kInvRing]
  static constexpr uint32_t kScaleK = (kInv + kInvRing * 4 + 15) & ~15u;  // e4m3: scale bytes of the staged keys, then values
  static constexpr uint32_t kScaleV = kScaleK + (FORMAT == kCacheE4m3 ? 128 : 0);
  static constexpr uint32_t kBars = (kScaleV + (FORMAT == kCacheE4m3 ? 128 : 0) + 7) & ~7u;
  static constexpr uint32_t kNumBars = 33;
  static constexpr uint32_t kTmem = kBars + kNumBars * 8;
  static constexpr uint32_t kAbort = kTmem + 4;
  static constexpr uint32_t kScan = kRow;  // before the roles begin
  static_assert(sizeof(SplitScan<kChunkThreads>) <= 1024, "the scan lies over kRow");
  static constexpr uint32_t kBytes = kAbort + 4;
  static_assert(kBytes <= 227 * 1024, "shared memory");
};

enum : int {
  kCbQ = 0,        // + row tile: its queries are in shared memory (256 arrivals)
  kCbKFull = 2,    // + stage: K as bf16 (TMA, or an arrival of each bank thread)
  kCbKEmpty = 4,   // + stage: both S of the tile are done
  kCbVFull = 6,    // + bank stage: V as TMA brought it (bf16)
  kCbEFull = 9,    // + bank stage: the bank (an arrival of each of its threads)
  kCbEEmpty = 12,  // + bank stage: both P E of the tile are done
  kCbRawKFull = 15,
  kCbRawVFull = 16,
  kCbRawKEmpty = 17,  // an arrival of each bank thread
  kCbRawVEmpty = 18,
  kCbS = 19,       // + row tile: S is in TMEM
  kCbP = 21,       // + row tile: P is in TMEM (256 arrivals)
  kCbO = 23,       // every product of the segment is done
  kCbDone = 24,    // every product this CTA issued is done
  kCbPair = 25,    // + pair of softmax warps (64 arrivals)
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

// tcgen05.mma and its commit by the one thread with leader != 0, in code that the whole warp runs: the
// operands are then formed once per warp, in uniform registers.
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t leader, uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar), "r"(leader)
      : "memory");
}

// True in one thread of the warp, always the same one.
__device__ __forceinline__ uint32_t elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}

// 8 columns of the warp's lanes of TMEM (see tmem_ld32).
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
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
  short *s_shift = reinterpret_cast<short *>(smem + Lay::kShift);
  volatile unsigned *s_inv = reinterpret_cast<volatile unsigned *>(smem + Lay::kInv);
  unsigned short *s_class = reinterpret_cast<unsigned short *>(smem + Lay::kClass);
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
  if (warp == 24) {
    tmem_alloc(sbase + Lay::kTmem, 512);
    tmem_relinquish();
  }
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(FEM_CB(kCbQ + i), 256);
      mbar_init(FEM_CB(kCbKFull + i), kCodes ? kBankThreads : 1);
      mbar_init(FEM_CB(kCbKEmpty + i), 1);
      mbar_init(FEM_CB(kCbS + i), 1);
      mbar_init(FEM_CB(kCbP + i), 256);
    }
    for (unsigned i = 0; i < kES; ++i) {
      mbar_init(FEM_CB(kCbVFull + i), 1);
      mbar_init(FEM_CB(kCbEFull + i), kBankThreads);
      mbar_init(FEM_CB(kCbEEmpty + i), 1);
    }
    for (int i = 0; i < 8; ++i) mbar_init(FEM_CB(kCbPair + i), 64);
    mbar_init(FEM_CB(kCbRawKFull), 1);
    mbar_init(FEM_CB(kCbRawVFull), 1);
    mbar_init(FEM_CB(kCbRawKEmpty), kBankThreads);
    mbar_init(FEM_CB(kCbRawVEmpty), kBankThreads);
    mbar_init(FEM_CB(kCbO), 1);
    mbar_init(FEM_CB(kCbDone), 1);
    fence_mbar_init();
    *abort_flag = 0;
    for (int i = 0; i < 16; ++i) reinterpret_cast<unsigned *>(smem + Lay::kAsk)[i] = ~0u;  // no tile
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t *>(smem + Lay::kTmem);
  SplitSeg sg;

  // The block's registers are 896 x 72; the softmax warps take 88 each, the bank's 56, the others 40:
  // 512 x 88 + 256 x 56 + 128 x 40 = 896 x 72.
  if (warp >= 24) asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
  if (warp == 24) {
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
  } else if (warp == 25) {
    // ------------------------------------------------------------ products
    // The whole warp walks the loop and one elected thread issues: the loop then stays uniform, and the
    // operands' descriptors are sums of per-tile bases and constants in uniform registers.  With one
    // thread in the loop alone its address arithmetic, between the other warps' instructions, took 6000
    // cycles a key tile, and the tensor pipe was idle for three quarters of them.
    constexpr uint32_t idesc_s = idesc_f16(128, 128, true, false);
    constexpr uint32_t idesc_o = idesc_f16(128, D, true, true);
    const uint64_t desc_q = smem_desc_sw128(sbase + Lay::kQ, 16, 1024), desc_k = smem_desc_sw128(sbase + Lay::kK, 16, 1024);
    const uint64_t desc_e = smem_desc_sw128(sbase + Lay::kE, 16384, 1024);
    const uint32_t leader = elect_one();
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
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              mma_ts(leader, tmem + 256 + t * D, tmem + t * 128 + (kk >> 2) * 64 + (kk & 3) * 8, de + ((kk * 2048) >> 4), idesc_o,
                     (k > 1 || kk > 0) ? 1u : 0u);
            if (t == tiles - 1) commit(leader, FEM_CB(kCbEEmpty + e % kES));
          }
          if (k < nk) {
            tc_fence_after_sync();
            const uint64_t dq = desc_q + t * (Lay::kTile >> 4), dk = desc_k + (i & 1) * (Lay::kTile >> 4);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk) {
              const uint32_t off = ((kk >> 2) * 16384 + (kk & 3) * 32) >> 4;
              mma_ss(leader, tmem + t * 128, dq + off, dk + off, idesc_s, kk > 0 ? 1u : 0u);
            }
            commit(leader, FEM_CB(kCbS + t));
            if (t == tiles - 1) commit(leader, FEM_CB(kCbKEmpty + (i & 1)));
          }
        }
      }
      if (ok) commit(leader, FEM_CB(kCbO));
      n += nk;
      ++seg;
    }
    if (leader) {
      mma_commit(FEM_CB(kCbDone));
      // nothing may be in flight when TMEM is freed
      mbar_wait(FEM_CB(kCbDone), 0, a.err, kErrWaitMma);
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------ the bank
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    // A thread has 4 channels (8 bytes of bf16) of every kRowStep-th row: the lanes of a half warp the two
    // halves of one 16-byte chunk in 8 rows, which the swizzle keeps on distinct banks.
    const int rl = tid & 7, col = (tid >> 3) % (D / 4);
    constexpr int kRowStep = kBankThreads / (D / 4), kRowsEach = 128 / kRowStep;
    const int r_first = rl + 8 * ((tid >> 3) / (D / 4));
    constexpr int kBatch = kCodes ? 4 : 8;  // rows whose loads are under way together (fewer where each takes more registers)
    // The thread's 4 codes of its first row in a staging tile, and its 4 elements in a tile of bf16; its rows
    // are a multiple of 8 apart, so they share the swizzle's pattern and lie at a fixed distance.
    static_assert(kRowStep % 8 == 0, "rows share the swizzle's pattern");
    const uint32_t raw_first =
        (D == 128 ? sw128_offset(r_first, col >> 2) : r_first * 64 + (((col >> 2) ^ ((r_first >> 1) & 3)) << 4)) + 4 * (col & 3);
    const uint32_t first = (col >> 4) * 16384 + sw128_offset(r_first, (col >> 1) & 7) + 8 * (col & 1);
    constexpr uint32_t kRawStep = kRowStep * (D == 128 ? 128 : 64), kStep = kRowStep * 128;
    float2 cb[2], cs[2], ci[2], cd[2];  // the thread's channels, in pairs
    int last_s = -1, last_h = -1;
    unsigned n = 0, seg = 0;
    bool ok = true;
    while (ok && walk.next(a, shape, sg)) {
      // coefficients of the thread's channels, from the sequence's first values
      if (BETA && (sg.s != last_s || sg.h != last_h)) {
        last_s = sg.s;
        last_h = sg.h;
        float vmax[4], vabs[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          vmax[e] = -INFINITY;
          vabs[e] = 0.f;
        }
        auto values = [&](long long row, float2 (&v)[2]) {
          if (kCodes) {
            const uint32_t x = *reinterpret_cast<const uint32_t *>(static_cast<const uint8_t *>(a.c.v) + row * D + col * 4);
            const float sc = paged_scale(a.c.ve[row]);
            v[0] = __fmul2_rn(e4m3x2_to_float2(x & 0xffffu), make_float2(sc, sc));
            v[1] = __fmul2_rn(e4m3x2_to_float2(x >> 16), make_float2(sc, sc));
          } else {
            const uint2 x = *reinterpret_cast<const uint2 *>(static_cast<const __nv_bfloat16 *>(a.c.v) + row * D + col * 4);
            v[0] = make_float2(bf16_lo(x.x), bf16_hi(x.x));
            v[1] = make_float2(bf16_lo(x.y), bf16_hi(x.y));
          }
        };
        const int page = sg.si.ctx > 0 ? paged_page(a, sg.s, 0) : -1;
        if (page >= 0) {
          const long long row = paged_row(a.c, page, sg.h, 0);
          const int cnt = min(kSampleKeys, sg.si.ctx);
#pragma unroll 4
          for (int kk = 0; kk < cnt; ++kk) {
            float2 v[2];
            values(row + kk, v);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              vmax[2 * e] = fmaxf(vmax[2 * e], v[e].x);
              vmax[2 * e + 1] = fmaxf(vmax[2 * e + 1], v[e].y);
              vabs[2 * e] = fmaxf(vabs[2 * e], fabsf(v[e].x));
              vabs[2 * e + 1] = fmaxf(vabs[2 * e + 1], fabsf(v[e].y));
            }
          }
        }
        unsigned zero = 0;  // the channels that have met nothing but zeros
#pragma unroll
        for (int e = 0; e < 4; ++e) zero |= vabs[e] == 0.f ? 1u << e : 0u;
        if (zero) {
#pragma unroll 2
          for (int i = sample_last(sg.si.ctx); i < sg.si.ctx; ++i) {
            const int p = sample_page(a, sg.s, i);
            if (p >= 0) {
              float2 v[2];
              values(paged_row(a.c, p, sg.h, i), v);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float x = e & 1 ? v[e / 2].y : v[e / 2].x;
                if ((zero >> e) & 1u) {
                  vmax[e] = fmaxf(vmax[e], x);
                  vabs[e] = fmaxf(vabs[e], fabsf(x));
                }
              }
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          const float *bp = a.beta + static_cast<long long>(sg.h) * D + col * 4 + e;
          const BankCoef x = bank_coef(__ldg(bp), vmax[e], vabs[e]), y = bank_coef(__ldg(bp + 1), vmax[e + 1], vabs[e + 1]);
          cb[e / 2] = make_float2(x.b, y.b);
          cs[e / 2] = make_float2(x.s, y.s);
          ci[e / 2] = make_float2(x.ic, y.ic);
          cd[e / 2] = make_float2(x.d, y.d);
        }
      }
      uint32_t most = 0;   // of each of the thread's channels, a byte: the exponent field of its largest |E| in tiles with a wide one
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
            uint32_t w[kBatch];
            float sc[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              w[u] = *reinterpret_cast<const uint32_t *>(raw + raw_first + kRawStep * (i0 + u));
              sc[u] = paged_scale(smem[Lay::kScaleK + r_first + kRowStep * (i0 + u)]);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const int r = r_first + kRowStep * (i0 + u);
              const float2 s2 = make_float2(sc[u], sc[u]);
              const float2 f0 = __fmul2_rn(e4m3x2_to_float2(w[u] & 0xffffu), s2), f1 = __fmul2_rn(e4m3x2_to_float2(w[u] >> 16), s2);
              uint2 y = make_uint2(pack_bf16(f0.x, f0.y), pack_bf16(f1.x, f1.y));
              if (ragged && gone(r)) y = make_uint2(0, 0);
              *reinterpret_cast<uint2 *>(tK + first + kStep * (i0 + u)) = y;
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
          if (tid < 8 * (D / 4) && rl == 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s_shift[(seg % kSegRing) * D + col * 4 + e] =
                  kind_pack(BETA ? bank_kind(e & 1 ? BankCoef{cb[e / 2].y, cs[e / 2].y, ci[e / 2].y, cd[e / 2].y}
                                                   : BankCoef{cb[e / 2].x, cs[e / 2].x, ci[e / 2].x, cd[e / 2].x})
                                 : INFINITY);
          }
        }
        if (BETA || kCodes || ragged) {
          uint32_t all[2] = {0, 0};  // the bits of the tile's E
          // rows in batches: their loads leave together (a store to the tile would hold the next row's back)
#pragma unroll 1
          for (int i0 = 0; i0 < kRowsEach; i0 += kBatch) {
            uint2 w[kBatch];
            float sc[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              if (kCodes) {
                const uint32_t x = *reinterpret_cast<const uint32_t *>(smem + Lay::kRawV + raw_first + kRawStep * (i0 + u));
                w[u] = make_uint2(x & 0xffffu, x >> 16);
                sc[u] = paged_scale(smem[Lay::kScaleV + r_first + kRowStep * (i0 + u)]);
              } else {
                w[u] = *reinterpret_cast<const uint2 *>(tE + first + kStep * (i0 + u));
              }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
              const uint32_t x[2] = {w[u].x, w[u].y};
              const bool none = ragged && gone(r_first + kRowStep * (i0 + u));  // whatever is there, it has no part in the largest |E| either
              uint32_t y[2];
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                float2 v = kCodes ? __fmul2_rn(e4m3x2_to_float2(x[e]), make_float2(sc[u], sc[u]))
                                  : make_float2(bf16_lo(x[e]), bf16_hi(x[e]));
                if (BETA) v = bank_pair(cb[e], cs[e], ci[e], cd[e], v);
                if (none) v = make_float2(0.f, 0.f);
                y[e] = pack_bf16(v.x, v.y);
                if (BETA) all[e] |= y[e];
              }
              *reinterpret_cast<uint2 *>(tE + first + kStep * (i0 + u)) = make_uint2(y[0], y[1]);
            }
          }
          // 2 or more sets the exponent's highest bit
          if (BETA && ((all[0] | all[1]) & 0x40004000u)) {
#pragma unroll 1
            for (int u = 0; u < kRowsEach; ++u) {
              const uint2 y = *reinterpret_cast<const uint2 *>(tE + first + kStep * u);
              most = __vmaxu4(most, __byte_perm((y.x >> 7) & 0xff00ffu, (y.y >> 7) & 0xff00ffu, 0x6420));
            }
          }
        }
        if (BETA && kt == sg.kt1 - 1) {
          // the channels' classes over the segment: eight lanes (rl) have them, one writes
          uint32_t c = 0;
          if (__any_sync(0xffffffffu, most != 0)) {
#pragma unroll 1
            for (int o = 1; o < 8; o <<= 1) most = __vmaxu4(most, __shfl_xor_sync(0xffffffffu, most, o));
#pragma unroll 1
            for (int e = 0; e < 16; e += 4) c |= static_cast<uint32_t>(wide_class((most >> (2 * e)) & 0xff)) << e;
          }
          if (rl == 0) s_class[(seg % kSegRing * Lay::kParts + (tid >> 3) / (D / 4)) * (D / 4) + col] = static_cast<unsigned short>(c);
        }
        fence_proxy_async_smem();
        mbar_arrive(FEM_CB(kCbEFull + es));
        if (kCodes) mbar_arrive(FEM_CB(kCbRawVEmpty));
      }
      ++seg;
    }
  } else if (warp < 24) {
    // ------------------------------------------------------------ softmax, queries and output of a row tile
    asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
    // Row tile t.  Two threads have row r: half 0 its keys 0 .. 63 of a key tile and channels 0 .. D/2 - 1,
    // half 1 the others.  Their warps are a pair, and meet at a barrier of their own now and then.
    const int t = (warp - 8) >> 3, half = ((warp - 8) >> 2) & 1, r = (warp & 3) * 32 + lane;
    const uint32_t pair = FEM_CB(kCbPair + t * 4 + (warp & 3));
    unsigned met = 0;
    constexpr int kHalfD = D / 2;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + t * 128 + half * 64 + lane_off;  // P goes over the first 32 of these 64 columns
    const uint32_t tO = tmem + 256 + t * D + half * kHalfD + lane_off;
    // per row: a maximum or a sum, or a rise asked for by each half in bf16; per half and warp: the tile of its
    // last request
    float *s_row = reinterpret_cast<float *>(smem + Lay::kRow) + t * 128;
    volatile __nv_bfloat16 *s_top = reinterpret_cast<volatile __nv_bfloat16 *>(s_row);
    volatile unsigned *s_ask = reinterpret_cast<volatile unsigned *>(smem + Lay::kAsk) + (t * 4 + (warp & 3)) * 2;
    const float qk_scale = a.scale * kLog2e;
    unsigned n = 0, ns = 0, seg = 0;
    // (like every wait it gives up in the end; then both warps of the pair do)
    auto meet = [&]() {
      mbar_arrive(pair);
      return __all_sync(0xffffffffu, chunk_wait(pair, met++ & 1, a.err, kErrWaitMma, abort_flag)) != 0;
    };
    // The thread's row of a segment: whether there is one, its place in the output, the keys it sees.
    struct Row {
      bool on;
      int lim, hq;
      int qrow;
    };
    auto row_of = [&](const SplitSeg &g, const ChunkRows &cr) {
      const int ir = t * 128 + r;
      Row w;
      w.on = ir < cr.rows;
      const int tok = cr.tok0 + (w.on ? ir / a.group : 0);
      w.hq = g.h * a.group + (w.on ? ir % a.group : 0);
      w.qrow = g.si.q0 + tok;
      w.lim = w.on ? min(paged_limit(g.si, tok, a.causal), g.si.ctx) : 0;
      return w;
    };
    // Half of the row's query into shared memory, and the arrival that lets the segment's products start.
    auto load_q = [&](const Row &w, bool used) {
      if (used) {
        uint8_t *tQ = smem + Lay::kQ + t * Lay::kTile;
        const uint4 *qp = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.q) + w.qrow * a.q_sn + w.hq * a.q_sh) +
                          half * (kHalfD / 8);
        uint4 x[kHalfD / 8];
#pragma unroll
        for (int c = 0; c < kHalfD / 8; ++c) x[c] = w.on ? __ldg(qp + c) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int c = 0; c < kHalfD / 8; ++c) {
          const int ch = half * (kHalfD / 8) + c;
          *reinterpret_cast<uint4 *>(tQ + (ch >> 3) * 16384 + sw128_offset(r, ch & 7)) = x[c];
        }
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
      const int nk = sg.kt1 - sg.kt0;
      // a row that sees nothing of the segment needs no maximum
      float m = w.lim > sg.kt0 * kChunkKeys ? -INFINITY : 0.f, L = 0.f;
      if (t < cr.tiles) {
        for (int k = 0; k < nk; ++k) {
          ++ns;  // this tile's number; its S is the barrier's phase ns - 1
          ok = __all_sync(0xffffffffu, chunk_wait(FEM_CB(kCbS + t), (ns - 1) & 1, a.err, kErrWaitMma, abort_flag));
          if (!ok) break;
          tc_fence_after_sync();
          const int k0 = (sg.kt0 + k) * kChunkKeys + half * 64;
          const unsigned inv = s_inv[(n + k) % kInvRing];
          const bool masked = __any_sync(0xffffffffu, k0 + 64 > w.lim) || inv;
          auto mask = [&](int c, uint32_t (&sr)[32]) {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const bool seen = k0 + c * 32 + j < w.lim && !((inv >> ((half * 64 + c * 32 + j) >> box_shift)) & 1u);
              sr[j] = seen ? sr[j] : 0xff800000u;
            }
          };
          // the half row's largest score
          auto largest = [&]() {
            float y = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < 2; ++c) {
              uint32_t sr[32];
              tmem_ld32(tS + c * 32, sr);
              tmem_ld_wait();
              if (masked) mask(c, sr);
#pragma unroll
              for (int j = 0; j < 32; j += 2) y = fmax3(y, __uint_as_float(sr[j]), __uint_as_float(sr[j + 1]));
            }
            return y * qk_scale;
          };
          // The row's maximum moves to `top`: its sum, and its half of the products so far (of the key tiles
          // before: see the issue order), are rescaled.  (By up to 2^-128 at once, when the tile before had its
          // weights near the end of the range: they are worth 1 after that.)  Whole warps.
          auto raise = [&](float top, bool products) {
            float root = 1.f;
            if (top > m) {
              root = weight_root(m - top);
              m = top;
              L = L * root * root;
            }
            if (products) {
#pragma unroll 1
              for (int c = 0; c < kHalfD / 32; ++c) {
                uint32_t v[32];
                tmem_ld32(tO + c * 32, v);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * root * root);
                tmem_st32(tO + c * 32, v);
              }
            }
          };
          if (__any_sync(0xffffffffu, m == -INFINITY)) {
            // the first tile with something to see: the two threads agree on the row's maximum, exactly, so
            // that the weight of its key is 1 and not a rounding of it
            float top = largest();
            if (half == 1) s_row[r] = top;
            if (!(ok = meet())) break;
            if (half == 0) s_row[r] = top = fmaxf(top, s_row[r]);
            if (!(ok = meet())) break;
            if (half == 1) top = s_row[r];
            raise(top, k > 0);
          } else {
            // a rise asked for during the tile before: what either thread wrote then is seen by both
            // now, through the arrivals of P and the product they let start
            const unsigned q0 = s_ask[0], q1 = s_ask[1];
            if (q0 == ns - 1 || q1 == ns - 1) {
              const float t0 = q0 == ns - 1 ? __bfloat162float(s_top[2 * r]) : -INFINITY;
              const float t1 = q1 == ns - 1 ? __bfloat162float(s_top[2 * r + 1]) : -INFINITY;
              if (!(ok = meet())) break;  // both have read what the next request overwrites
              raise(m + fmaxf(t0, t1), true);
            }
          }
          // The weights against the maximum so far, and their sum.  bf16 and fp32 hold them however far a
          // score lies above it (to 2^127; where they or their sum are beyond, the row goes to the exact path);
          // a sum over kAskSum asks for a larger one from the next tile on.
          const float mz = m == -INFINITY ? 0.f : m;
          const float2 scale2 = make_float2(qk_scale, qk_scale), negm2 = make_float2(-mz, -mz);
          float2 ls[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          uint32_t both[2][32];
          tmem_ld32(tS, both[0]);
          tmem_ld32(tS + 32, both[1]);
          tmem_ld_wait();
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t p[16];
            uint32_t(&sr)[32] = both[c];
            if (masked) mask(c, sr);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 x = __ffma2_rn(make_float2(__uint_as_float(sr[2 * i]), __uint_as_float(sr[2 * i + 1])), scale2, negm2);
              const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
              ls[i & 1] = __fadd2_rn(ls[i & 1], e);
              p[i] = pack_bf16(e.x, e.y);
            }
            tmem_st16(tS + c * 16, p);  // over columns already read
          }
          const float sum = (ls[0].x + ls[0].y) + (ls[1].x + ls[1].y);
          if (__any_sync(0xffffffffu, sum > kAskSum)) {
            // m + log2(sum) is at least the largest score, and at most 6 more.  The rise, from 40 to 128, goes over in
            // bf16, within 1/2; of a maximum in the tens of thousands bf16 keeps no more than 128.
            s_top[2 * r + half] = __float2bfloat16_rn(sum > kAskSum ? lg2_approx(sum) : -INFINITY);
            if (lane == 0) s_ask[half] = ns;
          }
          L += sum;
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
        // the row's sum: half 1's goes to half 0, and the whole comes back
        if (half == 1) s_row[r] = L;
        if (!(ok = meet())) break;
        if (half == 0) s_row[r] = L = L + s_row[r];
        if (!(ok = meet())) break;
        if (half == 1) L = s_row[r];
        // ---- the row's output (half of its channels), or its piece
        // A row that saw nothing has no weight.  Where the segment held keys for it, the sum lies between 1/2 and
        // the end of the range, or the row is left to the exact path: the last tile's weights may each be within
        // the range, to 2^127, and O with them, and their sum be past it; and scores past 2^24 are rounded to
        // whole numbers, the maximum apart from the weights.  (What paged_out takes for lost is relative to a
        // sum of about 1 or more.)
        if (!(L >= kLeastSum && L < INFINITY)) {
          m = -INFINITY;
          if (w.lim > sg.kt0 * kChunkKeys) L = __int_as_float(0x7fffffff);
        }
        const int ir = t * 128 + r;
        const long long orow = static_cast<long long>(w.qrow) * a.Hq + w.hq;
        const bool whole = sg.kt0 == 0 && sg.kt1 == sg.kt_all;
        const unsigned short *classes = s_class + seg % kSegRing * Lay::kParts * (D / 4);
        auto wide = [&](int j) {
          int c = 0;
#pragma unroll
          for (int i = 0; i < Lay::kParts; ++i) c = max(c, (classes[i * (D / 4) + (j >> 2)] >> (4 * (j & 3))) & 15);
          return c;
        };
        const short *shift = s_shift + (seg % kSegRing) * D + half * kHalfD;
        float *piece = sp.pieces + static_cast<size_t>(cta * 2 + (sg.kt0 == 0 ? 1 : 0)) * piece_floats(256, D);
        const bool empty = L == 0.f;
        const float inv_l = empty ? 0.f : (BETA ? kBankUnit : 1.f) / L;
        bool good = true;
        // 8 channels at a time (a loop of a few lines: the instruction cache serves all roles at once).  Lane l has
        // the coefficients of channel l of a group of 32; every row needs all of them
        OutCoef oc = {};
#pragma unroll 1
        for (int c = 0; c < kHalfD; c += 8) {
          uint32_t v[8];
          tmem_ld8(tO + c, v);
          tmem_ld_wait();
          if (whole) {
            if (BETA && (c & 31) == 0)
              oc = out_coef(__ldg(a.beta + static_cast<long long>(sg.h) * D + half * kHalfD + c + lane), kind_unpack(shift[c + lane]),
                            wide(half * kHalfD + c + lane));
            uint32_t o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float x[2];
#pragma unroll
              for (int u = 0; u < 2; ++u) {
                const float av = __uint_as_float(v[2 * i + u]) * inv_l;
                if (BETA) {
                  const int from = (c & 31) + 2 * i + u;
                  OutCoef kf;
                  kf.g = __shfl_sync(0xffffffffu, oc.g, from);
                  kf.z = __shfl_sync(0xffffffffu, oc.z, from);
                  kf.y = __shfl_sync(0xffffffffu, oc.y, from);
                  kf.w = __shfl_sync(0xffffffffu, oc.w, from);
                  kf.lo = __shfl_sync(0xffffffffu, oc.lo, from);
                  bool fine;
                  x[u] = paged_out(kf, av, &fine);
                  good = good && fine;
                  if (!fine) x[u] = __int_as_float(0x7fffffff);  // the mark, as bf16
                } else {
                  const bool fine = fabsf(av) < kMostA;
                  x[u] = fine ? av : __int_as_float(0x7fffffff);
                  good = good && fine;
                }
              }
              o[i] = empty ? 0u : pack_bf16(x[0], x[1]);
            }
            if (w.on)
              *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) + orow * D + half * kHalfD + c) =
                  make_uint4(o[0], o[1], o[2], o[3]);
          } else if (w.on) {
            float *dst = piece + piece_at(ir, (half * kHalfD + c) >> 2, D);
            *reinterpret_cast<float4 *>(dst) =
                make_float4(__uint_as_float(v[0]), __uint_as_float(v[1]), __uint_as_float(v[2]), __uint_as_float(v[3]));
            *reinterpret_cast<float4 *>(dst + 32) =
                make_float4(__uint_as_float(v[4]), __uint_as_float(v[5]), __uint_as_float(v[6]), __uint_as_float(v[7]));
          }
        }
        // both halves' verdict (and the exchange above is read before the next segment's)
        const bool exact = whole && !good && !empty && w.on;
        if (whole && half == 0 && w.on) sp.exact[orow] = exact;
        if (!(ok = meet())) break;
        if (half == 1 && exact) sp.exact[orow] = 1;
        if (exact) record.any_exact = 1;
        if (w.on && half == 0) {
          if (whole) {
            if (a.lse != nullptr) a.lse[orow] = empty ? -INFINITY : (m + log2f(L)) * kLn2;
          } else {
            piece[256 * D + 2 * ir] = m;
            piece[256 * D + 2 * ir + 1] = L;
          }
        }
        if (!whole && t == 0) {
          const int cls = BETA && half == 0 && r < D ? wide(r) : 0;
          const bool any = __any_sync(0xffffffffu, cls != 0);
          if (half == 0 && r < D) {
            piece[piece_kinds(256, D) + r] = kind_unpack(s_shift[(seg % kSegRing) * D + r]);
            piece[piece_classes(256, D) + r] = static_cast<float>(cls);
          }
          if (half == 0 && lane == 0) piece[piece_wide(256, D) + (warp & 3)] = any ? 1.f : 0.f;
          if (half == 0 && r == 0) {
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
  if (warp == 24) {
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
