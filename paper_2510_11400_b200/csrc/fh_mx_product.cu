// Products of microscaled 4-bit matrices on the tensor cores.
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "fh_launch.cuh"
#include "fh_mx.cuh"
#include "fh_mx_launch.cuh"
#include "fh_tcgen05.cuh"

namespace fh {
namespace {

// C = alpha A B^T (+ C), A m x k and B n x k.  Rows of B lie along the 128 lanes of an accumulator and rows of A along its columns: a lane
// then owns a column of C, so that a warp's store of one row of C is contiguous for any ldc, and the few rows of A that a decoding step
// has cost few accumulator columns while B's 128 rows keep the tensor core's lanes full.
//
// A stage holds 256 elements of the common axis.  Containers are laid out so that this is one contiguous piece of codes and one of
// scales for each operand, in the very order the matrix instruction reads: four bulk copies, no descriptors in memory, no swizzle (eight
// rows' 16 bytes are 128 contiguous ones).  Where fewer rows than the instruction reads are stored, it reads on into the next piece, and the
// rows that come of it are not looked at: a code is always finite, and a NaN scale stays in its row.
constexpr int kProductThreads = 192;  // four warps for the result, one for copies, one for matrix instructions
constexpr int kStepChunks = 8;        // 8 x 32 elements to a stage
constexpr uint32_t kDrainPolls = 1u << 20;  // waits of up to 2 us each, for copies under way

// Waits.  Every wait of a role (loads, matrix instructions, scales, result) has a limit, `polls` (2^26, some seconds); the first one that runs
// out sets a flag, the CTA's or in a pair that of the whole cluster, which ends the others.  What is still under way then is waited for at the
// end, when no role runs any more and the flag no longer changes: nothing may be in flight, in this CTA's memory or the other one's, when a
// CTA ends.  Where no wait has run out, everything has been waited for on the way: copies by the thread that reads them (matrix instructions
// or scales), the instructions by the result's warps, and the word that a stage is free, given only where the stage is used again, by
// the loading thread.  The status is first written by CTA 0, one of the first to run, as it begins; a CTA that has given up writes
// FH_ERR_TIMEOUT as it ends, a wait and a drain later.

// An aligned place for a CTA's stages.  `zero` hides from the compiler that it has this address already: what only the end of the pair
// kernel needs would take registers from its result warps (168 instead of 165; 4096 x 4096 x 4096 42.4 us and 48, 8192 x 16384 x 8192 400 and 428).
__device__ __forceinline__ uint8_t* stages_at(uint8_t* raw, uint32_t zero = 0u) { return raw + ((128u - (smem_u32(raw) & 127u)) & 127u) + zero; }
__device__ __forceinline__ uint32_t hidden_zero() {
  uint32_t r;
  asm volatile("mov.u32 %0, 0;" : "=r"(r));
  return r;
}

// Stage of a ring and the parity of its round.
template <int STAGES>
struct Turn {
  uint32_t stage = 0, round = 0;
  __device__ __forceinline__ void next() {
    if (++stage == (uint32_t)STAGES) {
      stage = 0;
      round ^= 1u;
    }
  }
};

template <int F, int QT>
struct ProductShape {
  static constexpr int kAtoms = F == kMxB32 ? 2 : 4;                     // groups of scales to a stage, each operand
  static constexpr uint32_t kP = 128 * 128, kQ = QT * 128, kS = kAtoms * 512;
  static constexpr uint32_t kStage = kP + kQ + 2 * kS;
  static constexpr int kStages = 4;
  static constexpr uint32_t kScaleCols = kAtoms * 4;                     // columns of tensor memory, each operand
  static constexpr uint32_t kAcc = QT < 32 ? 32 : QT;
  static constexpr uint32_t kCols = kAcc + kStages * 2 * kScaleCols <= 128 ? 128 : 256;
  static_assert(kAcc + kStages * 2 * kScaleCols <= kCols, "tensor memory");
  static constexpr size_t kSmem = 128 + (size_t)kStages * kStage + 256;
  static_assert(kStages * kStage >= (QT + 8) * 512, "partial sums, and rows read behind them");
};

// NR rows of a column of C from row `row` on, those below `end`.  (Addresses step from row to row: a product with ldc for each of them
// made a tile of 128 x 256 take 4 us.)
template <int DT>
using CType = typename std::conditional<DT == kF32, float, __nv_bfloat16>::type;
template <int DT, int NR>
__device__ __forceinline__ void load_c(const uint8_t* c, uint64_t ldc, uint32_t row, uint32_t end, uint32_t col, float (&v)[NR]) {
  const CType<DT>* p = reinterpret_cast<const CType<DT>*>(c) + (uint64_t)row * ldc + col;
#pragma unroll
  for (int x = 0; x < NR; ++x, p += ldc) {
    v[x] = 0.0f;
    if (row + x < end) v[x] = (float)*p;
  }
}
template <int DT, int NR>
__device__ __forceinline__ void store_c(uint8_t* c, uint64_t ldc, uint32_t row, uint32_t end, uint32_t col, const float (&v)[NR]) {
  CType<DT>* p = reinterpret_cast<CType<DT>*>(c) + (uint64_t)row * ldc + col;
  if (row + NR <= end) {
#pragma unroll
    for (int x = 0; x < NR; ++x, p += ldc) *p = (CType<DT>)v[x];
    return;
  }
#pragma unroll
  for (int x = 0; x < NR; ++x, p += ldc)
    if (row + x < end) *p = (CType<DT>)v[x];
}

// What the sums are multiplied by: 2^(ea + eb) and alpha, as one factor where that is exact and no product of it leaves the range of normal
// numbers that the result is in; otherwise alpha's mantissa and then its power of two with the other in three steps of one direction, so
// that nothing over- or underflows on the way that does not in the end.
struct ProductScale {
  float f[4];
  bool one;
  __device__ __forceinline__ ProductScale(int ea, int eb, float alpha) {
    const int e = ea + eb;
    const float m = fabsf(alpha);
    one = e == 0 || (e >= -32 && e <= 32 && m >= 0x1p-60f && m <= 0x1p60f);
    if (one) {
      f[0] = alpha * pow2_f(e);
      return;
    }
    int own = 0;
    f[0] = frexpf(alpha, &own);
    const int t = m > 0.0f ? e + own : 0, t1 = t / 3, t2 = (t - t1) / 2;
    f[1] = pow2_f(t1);
    f[2] = pow2_f(t2);
    f[3] = pow2_f(t - t1 - t2);
  }
  template <int NR>
  __device__ __forceinline__ void apply(float (&v)[NR]) const {
#pragma unroll
    for (int x = 0; x < NR; ++x) v[x] *= f[0];
    if (!one) {
#pragma unroll
      for (int x = 0; x < NR; ++x) v[x] = v[x] * f[1] * f[2] * f[3];
    }
  }
};

// Sums rows of partial sums over the parts of a cluster (CTAs `stride` apart, from `first` on), NR rows at a time, in the order of the parts; four
// parts are asked for at once.
template <int NR>
__device__ __forceinline__ void sum_parts(uint32_t at, uint32_t row_bytes, uint32_t first, uint32_t stride, uint32_t parts, float (&v)[NR]) {
#pragma unroll
  for (int x = 0; x < NR; ++x) v[x] = 0.0f;
  for (uint32_t r0 = 0; r0 < parts; r0 += 4u) {
    float w[4][NR];
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r)
      if (r0 + r < parts) {
#pragma unroll
        for (int x = 0; x < NR; ++x) w[r][x] = ld_cluster(at + x * row_bytes, first + (r0 + r) * stride);
      }
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r)
      if (r0 + r < parts) {
#pragma unroll
        for (int x = 0; x < NR; ++x) v[x] += w[r][x];
      }
  }
}

template <int DT, int F, int QT>
__global__ void __launch_bounds__(kProductThreads) mx_product_kernel(const MxProductArgs g) {
  using S = ProductShape<F, QT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = stages_at(smem_raw);
  uint8_t* tail = smem + S::kStages * S::kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(tail);
  uint64_t* empty = full + S::kStages;
  uint64_t* done = empty + S::kStages;
  uint64_t* idle = done + 1;  // after a wait that ran out: what was issued is complete
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(idle + 1);
  volatile uint32_t* abort = tmem_at + 1;
  uint32_t* loads = tmem_at + 2;  // stages that the loading thread has asked for
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t rank = g.split > 1 ? cluster_rank() : 0u;
  const uint32_t cell = blockIdx.x / g.split, tp = cell % g.tiles_n, tq = cell / g.tiles_n;  // (clusters are along x)
  const MxLayout lp(g.n, g.k, F), lq(g.m, g.k, F);
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    mbar_init(done, 1);
    mbar_init(idle, 1);
    *abort = 0u;
    fence_mbar_init();
  }
  if (warp == 5) {
    tmem_alloc(tmem_at, S::kCols);
    tmem_last_alloc();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  dep_trigger();  // (behind the allocation: no later kernel takes tensor memory that this one still wants)
  dep_wait();
  int32_t ea = 0, eb = 0;
  const bool ok_a = mx_header_ok(g.a, g.a_bytes, lq, &ea), ok_b = mx_header_ok(g.b, g.b_bytes, lp, &eb), ok = ok_a && ok_b;
  if (blockIdx.x == 0 && tid == 0 && g.status) *g.status = ok ? 0ull : status_word(kErrCorrupt);
  const uint32_t chunks = lp.kp / 32u, steps = (chunks + kStepChunks - 1u) / kStepChunks;
  const uint32_t first = (uint32_t)((uint64_t)steps * rank / g.split), last = (uint32_t)((uint64_t)steps * (rank + 1u) / g.split);
  const uint32_t rp = lp.block_rows(tp), rq = lq.block_rows(tq);
  if (ok && warp == 4) {
    if (lane == 0) {
      const uint8_t* p = g.b + lp.code_at(tp * 128u, 0);
      const uint8_t* q = g.a + lq.code_at(tq * 128u, 0);
      const uint8_t* sp = g.b + lp.atom_at(tp, 0);
      const uint8_t* sq = g.a + lq.atom_at(tq, 0);
      uint32_t loaded = 0;
      Turn<S::kStages> at;
      for (uint32_t it = first; it < last && loaded != g.silent; ++it, ++loaded, at.next()) {
        const uint32_t s = at.stage;
        if (loaded >= (uint32_t)S::kStages && !mbar_poll<false>(empty + s, at.round ^ 1u, g.polls, abort)) {
          *abort = 1u;
          break;
        }
        const uint32_t nc = min((uint32_t)kStepChunks, chunks - it * kStepChunks);
        const uint32_t na = min((uint32_t)S::kAtoms, lp.atoms - it * S::kAtoms);
        uint8_t* st = smem + s * S::kStage;
        mbar_expect_tx(full + s, nc * 16u * (rp + rq) + na * 1024u);
        bulk_g2s(st, p + (uint64_t)it * kStepChunks * 16u * rp, nc * 16u * rp, full + s);
        bulk_g2s(st + S::kP, q + (uint64_t)it * kStepChunks * 16u * rq, nc * 16u * rq, full + s);
        bulk_g2s(st + S::kP + S::kQ, sp + (uint64_t)it * S::kAtoms * 512u, na * 512u, full + s);
        bulk_g2s(st + S::kP + S::kQ + S::kS, sq + (uint64_t)it * S::kAtoms * 512u, na * 512u, full + s);
      }
      *loads = loaded;
    }
  } else if (ok && warp == 5) {
    if (lane == 0) {
      Turn<S::kStages> at;
      for (uint32_t it = first; it < last; ++it, at.next()) {
        const uint32_t s = at.stage;
        if (!mbar_poll<false>(full + s, at.round, g.polls, abort)) {
          *abort = 1u;
          break;
        }
        tc_fence_after();
        const uint32_t nc = min((uint32_t)kStepChunks, chunks - it * kStepChunks);
        const uint32_t na = min((uint32_t)S::kAtoms, lp.atoms - it * S::kAtoms);
        const uint32_t st = smem_u32(smem) + s * S::kStage;
        const uint32_t sa = tmem + S::kAcc + s * 2u * S::kScaleCols, sb = sa + S::kScaleCols;
        const uint64_t da = smem_desc(st, rp * 16u, 128u), db = smem_desc(st + S::kP, rq * 16u, 128u), ds = smem_desc(st + S::kP + S::kQ, 128u, 128u);
#pragma unroll
        for (uint32_t x = 0; x < (uint32_t)S::kAtoms; ++x)
          if (x < na) {
            tc_copy_scales(sa + 4u * x, ds + 32u * x);
            tc_copy_scales(sb + 4u * x, ds + S::kS / 16u + 32u * x);
          }
#pragma unroll
        for (uint32_t x = 0; x < kStepChunks / 2u; ++x)
          if (2u * x < nc) {
            const uint32_t word = F == kMxB32 ? x / 2u : x, id = F == kMxB32 ? x % 2u * 2u : 0u;
            tc_mma_mx<F == kMxB32>(tmem, da + 2u * x * rp, db + 2u * x * rq, mx_idesc(128u, QT, F == kMxB32, id), sa + 4u * word, sb + 4u * word,
                                   it > first || x > 0u);
          }
        if (it + (uint32_t)S::kStages < last) tc_commit(empty + s);
      }
      tc_commit(done);
    }
  }
  __syncwarp();
  // the accumulator: lane i of warp w has row 32 w + i of the tile of B, QT columns for the rows of A
  const bool mine = ok && warp < 4;
  bool good = mine;
  if (mine) {
    good = mbar_poll_warp(done, 0u, g.polls, abort);
    if (!good && lane == 0) *abort = 1u;
    tc_fence_after();
  }
  const uint32_t col = tp * 128u + warp * 32u + lane;
  const ProductScale scaled(ea, eb, g.alpha);
  if (g.split == 1u) {
    if (good) {
#pragma unroll 1
      for (uint32_t q0 = 0; q0 < (uint32_t)QT; q0 += 16u) {
        uint32_t v[16];
        float f[16];
        tc_load16(tmem + (warp * 32u << 16) + q0, v);
        tc_load_wait();
#pragma unroll
        for (uint32_t x = 0; x < 16u; ++x) f[x] = bits_f(v[x]);
        scaled.apply(f);
        if (col < g.n) {
          if (g.accumulate) {
            float old[16];
            load_c<DT, 16>(g.c, g.ldc, tq * 128u + q0, g.m, col, old);
#pragma unroll
            for (uint32_t x = 0; x < 16u; ++x) f[x] += old[x];
          }
          store_c<DT, 16>(g.c, g.ldc, tq * 128u + q0, g.m, col, f);
        }
      }
    }
  } else {
    // partial sums of the cluster's CTAs, each over its part of the common axis: to shared memory (all copies into it have been used),
    // then every CTA adds up some rows of C, in the order of the parts
    float* part = reinterpret_cast<float*>(smem);
    if (good) {
#pragma unroll 1
      for (uint32_t q0 = 0; q0 < (uint32_t)QT; q0 += 16u) {
        uint32_t v[16];
        tc_load16(tmem + (warp * 32u << 16) + q0, v);
        tc_load_wait();
#pragma unroll
        for (uint32_t x = 0; x < 16u; ++x) part[(q0 + x) * 128u + tid] = bits_f(v[x]);
      }
    }
    cluster_sync();
    if (good && col < g.n) {
      const uint32_t rows = min((uint32_t)QT, g.m - tq * 128u), end = rows * (rank + 1u) / g.split;
      constexpr int NR = QT < 32 ? 2 : 8;
      for (uint32_t q = rows * rank / g.split; q < end; q += NR) {
        float f[NR], old[NR] = {};
        if (g.accumulate) load_c<DT, NR>(g.c, g.ldc, tq * 128u + q, tq * 128u + end, col, old);
        sum_parts<NR>(smem_u32(part + q * 128u + tid), 512u, 0u, 1u, g.split, f);  // (rows behind the last: stage bytes)
        scaled.apply(f);
        if (g.accumulate) {
#pragma unroll
          for (int x = 0; x < NR; ++x) f[x] += old[x];
        }
        store_c<DT, NR>(g.c, g.ldc, tq * 128u + q, tq * 128u + end, col, f);
      }
    }
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (*abort) {  // (see "Waits" above)
    if (ok && lane == 0 && warp == 4)
      for (uint32_t n = *loads, w = n > (uint32_t)S::kStages ? n - S::kStages : 0u; w < n; ++w) mbar_wait(full + w % S::kStages, w / S::kStages & 1u, kDrainPolls);
    if (ok && lane == 0 && warp == 5) {
      tc_commit(idle);
      mbar_wait(idle, 0u, kDrainPolls);
    }
    if (tid == 0 && g.status) *g.status = status_word(kErrTimeout);
    __syncthreads();
  }
  if (warp == 5) tmem_free(tmem, S::kCols);
}

// Large products: a pair of CTAs on a tile of 256 columns and 256 rows of C, 128 rows of B and 128 of A in the shared memory of each.
// A tile of 128 x 128 moves 34 KB from L2 to an SM for 256 cycles of matrix instructions; this one 36 KB for 512.  Pairs take
// tiles one after the other; the eight warps for the result take the accumulator into registers at once, so that the next tile's matrix
// instructions start while they write.  With a split, a cluster's pairs share one tile.
//
// Scales are copied to tensor memory by a thread of its own.  In the one that issues the matrix instructions the copies (55 cycles each, 6 a
// stage in B32, 12 in B16) stood in line with those, which take 512: 4096 x 4096 x 16384 138 and 182 us, now 103 and 143.
constexpr int kPairThreads = 352;  // eight warps for the result, then one each for loads, matrix instructions and scales

template <int F>
struct PairShape {
  static constexpr int kAtoms = F == kMxB32 ? 2 : 4;
  static constexpr uint32_t kOp = 128 * 128, kS = kAtoms * 512;
  static constexpr uint32_t kStage = 2 * kOp + 3 * kS;  // codes of B and A, scales of B, scales of both halves of A
  static constexpr int kStages = F == kMxB32 ? 6 : 5;
  static constexpr uint32_t kScaleCols = kAtoms * 12;   // columns of tensor memory: B's four and A's eight to a word
  static constexpr uint32_t kCols = 512;
  static_assert(256 + kStages * kScaleCols <= kCols, "tensor memory");
  static constexpr size_t kSmem = 128 + (size_t)kStages * kStage + 256;
  static_assert(kStages * kStage >= (256 + 8) * 512, "partial sums, and rows read behind them");
};

// The barriers behind the stages, and the words behind them.
template <int F>
struct PairBars {
  static constexpr int kStages = PairShape<F>::kStages;
  static constexpr int kFull = 0;                     // even CTA: both CTAs' stages have arrived
  static constexpr int kEmpty = kStages;              // a stage may be loaded again
  static constexpr int kReady = 2 * kStages;          // even CTA: its scales are in both CTAs' tensor memory
  static constexpr int kSums = 3 * kStages;           // the accumulator is complete
  static constexpr int kTaken = kSums + 1;            // even CTA: both CTAs' warps have taken it
  static constexpr int kIdle = kTaken + 1;            // even CTA, after a wait that ran out: what its two threads issued is complete
  static constexpr int kWords = kIdle + 2;
  static_assert(kWords * 8 + (3 + kStages) * 4 <= 256, "room behind the stages");
};

// How the codes and scales of an operand are laid out for the copies, which tell the even CTA's barrier of both CTAs' stages: a plain
// bulk copy cannot reach the other CTA's, and a thread that passed the word on took 0.3 us a stage.
struct OperandMaps {
  CUtensorMap codes;   // of the blocks of 128 rows: 128 bytes (eight rows), 16 of them, every 32 columns
  CUtensorMap rest;    // of the last block, if it has fewer rows: the copies fill up with zeros
  CUtensorMap scales;  // 128 bytes, four to a group
};
struct PairArgs {
  OperandMaps a, b;
  MxProductArgs g;
};

// Tile `t` of the pairs' order: eight rows of tiles at a time, column by column, so that the tiles under way together share rows of A and of B
// in L2 (row by row, 8192 x 16384 x 8192 took 595 us).
struct PairTile {
  uint32_t m, n;
  __device__ __forceinline__ PairTile(uint32_t t, uint32_t tiles_m, uint32_t tiles_n) {
    const uint32_t band = t / (8u * tiles_n), at = t % (8u * tiles_n), high = min(8u, tiles_m - 8u * band);
    m = 8u * band + at % high;
    n = at / high;
  }
};

// What a CTA loads of a tile.
template <int F>
struct PairLoads {
  using S = PairShape<F>;
  uint32_t np, nq;      // blocks of 128 rows that there are of B and of A
  uint32_t bytes, mine; // to a stage, of both CTAs and of this one
  uint32_t zp, zq;      // where the codes of this CTA's blocks begin in their maps ...
  uint32_t yp, yq, ya;  // ... and the scales of its block of B, of both of A, and of A's second one after its first
  bool p_whole, q_whole;
  __device__ __forceinline__ PairLoads(const MxProductArgs& g, uint32_t tile, uint32_t half) {
    const MxLayout lp(g.n, g.k, F), lq(g.m, g.k, F);
    const PairTile where(tile, g.tiles_m, g.tiles_n);
    const uint32_t chunks = lp.kp / 32u, blocks_p = (g.n + 127u) / 128u, blocks_q = (g.m + 127u) / 128u;
    const uint32_t bp0 = where.n * 2u, bq0 = where.m * 2u, bp = bp0 + half, bq = bq0 + half;
    np = min(2u, blocks_p - bp0);
    nq = min(2u, blocks_q - bq0);
    p_whole = lp.block_rows(min(bp, blocks_p - 1u)) == 128u;
    q_whole = lq.block_rows(min(bq, blocks_q - 1u)) == 128u;
    bytes = (np + nq) * S::kOp + (np + 2u * nq) * S::kS;
    mine = ((half < np) + (half < nq)) * S::kOp + ((half < np) + nq) * S::kS;
    zp = p_whole ? bp * chunks : 0u;
    zq = q_whole ? bq * chunks : 0u;
    yp = bp * lp.atoms * 4u;
    yq = bq0 * lq.atoms * 4u;
    ya = lq.atoms * 4u;
  }
  // Stage `it` of the common axis to stage `s` of the ring.
  __device__ __forceinline__ void load(const PairArgs& pa, uint8_t* smem, uint64_t* full, uint32_t it, uint32_t s, uint32_t half, uint32_t even) const {
    const uint32_t st = smem_u32(smem) + s * S::kStage, sc = st + 2u * S::kOp, bar = at_rank(full + s, even);
    if (half == 0u) mbar_expect_tx(full + s, bytes);
    if (half < np) tma_pair_3d(st, p_whole ? &pa.b.codes : &pa.b.rest, 0u, 0u, zp + it * kStepChunks, bar);
    if (half < nq) tma_pair_3d(st + S::kOp, q_whole ? &pa.a.codes : &pa.a.rest, 0u, 0u, zq + it * kStepChunks, bar);
    const uint32_t y = it * S::kAtoms * 4u;
    if (half < np) tma_pair_2d(sc, &pa.b.scales, 0u, yp + y, bar);
    tma_pair_2d(sc + S::kS, &pa.a.scales, 0u, yq + y, bar);
    if (nq > 1u) tma_pair_2d(sc + 2u * S::kS, &pa.a.scales, 0u, yq + ya + y, bar);
  }
};

template <int DT, int F>
__global__ void __launch_bounds__(kPairThreads, 1) mx_product_pair_kernel(const __grid_constant__ PairArgs pa) {
  const MxProductArgs& g = pa.g;
  using S = PairShape<F>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = stages_at(smem_raw);
  using B = PairBars<F>;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  uint64_t *empty = full + B::kEmpty, *ready = full + B::kReady, *sums = full + B::kSums, *taken = full + B::kTaken, *idle = full + B::kIdle;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(full + B::kWords);
  volatile uint32_t* abort = tmem_at + 1;
  uint32_t* loads = tmem_at + 2;  // stages that the loading thread has asked for, and of each stage the odd CTA's bytes
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t crank = cluster_rank(), half = crank & 1u, even = crank & ~1u, rank = crank / 2u;
  const uint32_t pairs = gridDim.x / (2u * g.split), pair = blockIdx.x / (2u * g.split);  // clusters, each on tiles of its own
  const MxLayout lp(g.n, g.k, F), lq(g.m, g.k, F);
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
      mbar_init(ready + i, 1);
    }
    mbar_init(sums, 1);
    mbar_init(taken, 16);
    mbar_init(idle, 1);
    mbar_init(idle + 1, 1);
    *abort = 0u;
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc_pair(tmem_at, S::kCols);
    tmem_last_alloc_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // (both CTAs' barriers stand)
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  dep_trigger();  // (behind the allocation: no later kernel takes tensor memory that this one still wants)
  dep_wait();
  int32_t ea = 0, eb = 0;
  const bool ok_a = mx_header_ok(g.a, g.a_bytes, lq, &ea), ok_b = mx_header_ok(g.b, g.b_bytes, lp, &eb), ok = ok_a && ok_b;
  if (blockIdx.x == 0 && tid == 0 && g.status) *g.status = ok ? 0ull : status_word(kErrCorrupt);
  const uint32_t chunks = lp.kp / 32u, steps = (chunks + kStepChunks - 1u) / kStepChunks;
  const uint32_t first = (uint32_t)((uint64_t)steps * rank / g.split), last = (uint32_t)((uint64_t)steps * (rank + 1u) / g.split);
  const uint32_t tiles = ok ? g.tiles_m * g.tiles_n : 0u;
  bool good = true;
  if (warp == 8) {
    if (lane == 0) {
      uint32_t loaded = 0;
      const uint32_t silent = half ? g.silent : ~0u;
      Turn<S::kStages> turn;
      for (uint32_t tile = pair; tile < tiles && good; tile += pairs) {
        const PairLoads<F> t(g, tile, half);
        for (uint32_t it = first; it < last; ++it, ++loaded, turn.next()) {
          if (loaded == silent) {
            good = false;
            break;
          }
          if (loaded >= (uint32_t)S::kStages && !mbar_poll<true>(empty + turn.stage, turn.round ^ 1u, g.polls, abort)) {
            raise_cluster(abort, 2u * g.split);
            good = false;
            break;
          }
          loads[1u + turn.stage] = half ? t.mine : t.bytes - t.mine;
          t.load(pa, smem, full, it, turn.stage, half, even);
        }
      }
      *loads = loaded;
    }
  } else if (warp == 9) {
    if (lane == 0 && half == 0u) {  // (issues for both)
      const uint16_t both = (uint16_t)(3u << even);
      uint32_t n = 0;
      Turn<S::kStages> turn;
      for (uint32_t tile = pair; tile < tiles && good; tile += pairs, ++n) {
        if (n && !mbar_poll<true>(taken, (n - 1u) & 1u, g.polls, abort)) {
          raise_cluster(abort, 2u * g.split);
          break;
        }
        tc_fence_after();
        for (uint32_t it = first; it < last; ++it, turn.next()) {
          const uint32_t s = turn.stage, ph = turn.round;
          if (!mbar_poll<true>(ready + s, ph, g.polls, abort)) {
            raise_cluster(abort, 2u * g.split);
            good = false;
            break;
          }
          tc_fence_after();
          const uint32_t nc = min((uint32_t)kStepChunks, chunks - it * kStepChunks);
          const uint32_t st = smem_u32(smem) + s * S::kStage;
          const uint32_t sa = tmem + 256u + s * S::kScaleCols, sb = sa + S::kAtoms * 4u;
          const uint64_t da = smem_desc(st, 2048u, 128u), db = smem_desc(st + S::kOp, 2048u, 128u);
#pragma unroll
          for (uint32_t x = 0; x < kStepChunks / 2u; ++x)
            if (2u * x < nc) {
              const uint32_t word = F == kMxB32 ? x / 2u : x, id = F == kMxB32 ? x % 2u * 2u : 0u;
              tc_mma_mx_pair<F == kMxB32>(tmem, da + 256u * x, db + 256u * x, mx_idesc(256u, 256u, F == kMxB32, id), sa + 4u * word, sb + 8u * word,
                                          it > first || x > 0u);
            }
          if (it + (uint32_t)S::kStages < last || tile + pairs < tiles) tc_commit_pair(empty + s, both);
        }
        if (good) tc_commit_pair(sums, both);
      }
    }
  } else if (warp == 10) {
    if (lane == 0 && half == 0u) {
      Turn<S::kStages> turn;
      for (uint32_t tile = pair; tile < tiles && good; tile += pairs)
        for (uint32_t it = first; it < last; ++it, turn.next()) {
          const uint32_t s = turn.stage;
          if (!mbar_poll<true>(full + s, turn.round, g.polls, abort)) {
            raise_cluster(abort, 2u * g.split);
            good = false;
            break;
          }
          tc_fence_after();
          const uint32_t na = min((uint32_t)S::kAtoms, lp.atoms - it * S::kAtoms);
          const uint32_t st = smem_u32(smem) + s * S::kStage;
          const uint32_t sa = tmem + 256u + s * S::kScaleCols, sb = sa + S::kAtoms * 4u;
          const uint64_t ds = smem_desc(st + 2u * S::kOp, 128u, 128u);
#pragma unroll
          for (uint32_t x = 0; x < (uint32_t)S::kAtoms; ++x)
            if (x < na) {
              tc_copy_scales_pair(sa + 4u * x, ds + 32u * x);
              tc_copy_scales_pair(sb + 8u * x, ds + S::kS / 16u + 32u * x);
              tc_copy_scales_pair(sb + 8u * x + 4u, ds + 2u * S::kS / 16u + 32u * x);
            }
          tc_commit_pair(ready + s, (uint16_t)(1u << even));
        }
    }
  } else {
    const ProductScale scaled(ea, eb, g.alpha);
    const uint32_t side = warp / 4u * 128u;  // columns of the accumulator: rows of A
    uint32_t n = 0;
    for (uint32_t tile = pair; tile < tiles && good; tile += pairs, ++n) {
      good = mbar_poll_warp(sums, n & 1u, g.polls, abort);
      if (!good) {
        if (lane == 0) raise_cluster(abort, 2u * g.split);
        break;
      }
      tc_fence_after();
      const PairTile where(tile, g.tiles_m, g.tiles_n);
      const uint32_t col = where.n * 256u + half * 128u + warp % 4u * 32u + lane, row = where.m * 256u + side;
      uint32_t v[8][16];
#pragma unroll
      for (uint32_t x = 0; x < 8u; ++x) tc_load16(tmem + (warp % 4u * 32u << 16) + side + 16u * x, v[x]);
      tc_load_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_at(taken, even);
      if (g.split == 1u) {
#pragma unroll
        for (uint32_t x = 0; x < 8u; ++x) {
          float f[16];
#pragma unroll
          for (uint32_t y = 0; y < 16u; ++y) f[y] = bits_f(v[x][y]);
          scaled.apply(f);
          if (col < g.n) {
            if (g.accumulate) {
              float old[16];
              load_c<DT, 16>(g.c, g.ldc, row + 16u * x, g.m, col, old);
#pragma unroll
              for (uint32_t y = 0; y < 16u; ++y) f[y] += old[y];
            }
            store_c<DT, 16>(g.c, g.ldc, row + 16u * x, g.m, col, f);
          }
        }
      } else {  // (one tile only: all copies into shared memory have been used)
        float* part = reinterpret_cast<float*>(smem) + side * 128u + warp % 4u * 32u + lane;
#pragma unroll
        for (uint32_t x = 0; x < 8u; ++x)
#pragma unroll
          for (uint32_t y = 0; y < 16u; ++y) part[(16u * x + y) * 128u] = bits_f(v[x][y]);
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  if (g.split > 1u) {
    cluster_sync();
    if (warp < 8u && tiles && !*abort) {
      const ProductScale scaled(ea, eb, g.alpha);
      const PairTile where(pair, g.tiles_m, g.tiles_n);
      const uint32_t p = warp % 4u * 32u + lane, col = where.n * 256u + half * 128u + p, row = where.m * 256u;
      const uint32_t rows = min(256u, g.m - row), from = rows * rank / g.split, end = rows * (rank + 1u) / g.split, mid = (from + end) / 2u;
      const uint32_t stop = warp < 4u ? mid : end;
      if (col < g.n)
        for (uint32_t q = warp < 4u ? from : mid; q < stop; q += 8u) {
          float f[8], old[8] = {};
          if (g.accumulate) load_c<DT, 8>(g.c, g.ldc, row + q, row + stop, col, old);
          sum_parts<8>(smem_u32(reinterpret_cast<float*>(smem) + q * 128u + p), 512u, half, 2u, g.split, f);
          scaled.apply(f);
          if (g.accumulate) {
#pragma unroll
            for (int x = 0; x < 8; ++x) f[x] += old[x];
          }
          store_c<DT, 8>(g.c, g.ldc, row + q, row + stop, col, f);
        }
    }
  }
  __syncthreads();
  cluster_sync();  // (a pair's memory serves both until both are done)
  if (*abort) {    // (in all CTAs of the cluster or in none; see "Waits" above)
    uint64_t* bars = reinterpret_cast<uint64_t*>(stages_at(smem_raw, hidden_zero()) + S::kStages * S::kStage);
    const uint32_t me = cluster_rank(), who = threadIdx.x;
    if (me % 2u == 0u && who == 8u * 32u) {
      // The pair's loading threads may have stopped at different stages, and a barrier counts the bytes of both: those that the odd CTA
      // has not asked for are taken off, those that it alone has asked for are expected.
      const uint32_t* count = reinterpret_cast<const uint32_t*>(bars + PairBars<F>::kWords) + 2;
      const uint32_t mine = count[0], other = ld_cluster_u32(count, me ^ 1u), most = max(mine, other);
#pragma unroll 1
      for (uint32_t w = min(mine, other); w < most; ++w) {
        const uint32_t s = w % S::kStages;
        if (mine < other)
          mbar_expect_tx(bars + s, ld_cluster_u32(count + 1 + s, me ^ 1u));
        else
          mbar_complete_tx(bars + s, count[1 + s]);
      }
#pragma unroll 1
      for (uint32_t w = most > (uint32_t)S::kStages ? most - S::kStages : 0u; w < most; ++w) mbar_wait(bars + w % S::kStages, w / S::kStages & 1u, kDrainPolls);
    }
    if (me % 2u == 0u && (who == 9u * 32u || who == 10u * 32u)) {
      uint64_t* bar = bars + PairBars<F>::kIdle + (who / 32u - 9u);
      tc_commit_pair(bar, (uint16_t)(1u << me));
      mbar_wait(bar, 0u, kDrainPolls);
    }
    if (who == 0u && g.status) *g.status = status_word(kErrTimeout);
    __syncthreads();
    cluster_sync();
  }
  if (warp == 9) tmem_free_pair(tmem, S::kCols);
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static std::atomic<void*> fn{nullptr};
  void* f = fn.load();
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
    fn.store(f);
  }
  return (EncodeTiled)f;
}

// A map of `dims` boxes of 128 bytes, `strides` bytes apart, as bytes.
bool encode_map(CUtensorMap* map, const uint8_t* base, uint32_t rank, const cuuint64_t (&dims)[3], const cuuint64_t (&strides)[2], const cuuint32_t (&box)[3]) {
  const EncodeTiled f = encode_tiled();
  const cuuint32_t ones[3] = {1, 1, 1};
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, const_cast<uint8_t*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int F>
bool encode_operand(OperandMaps* m, const uint8_t* c, uint32_t rows, uint32_t k) {
  const MxLayout l(rows, k, F);
  const uint32_t whole = l.r8 / 128u, rest = l.r8 % 128u, chunks = l.kp / 32u;
  const cuuint32_t box[3] = {128, 16, (cuuint32_t)kStepChunks}, sbox[3] = {128, 4 * PairShape<F>::kAtoms, 1};
  bool ok = true;
  if (whole) ok = encode_map(&m->codes, c + kMxHeadBytes, 3, {128, 16, (cuuint64_t)whole * chunks}, {128, 2048}, box);
  if (rest) ok = ok && encode_map(&m->rest, c + l.code_at(whole * 128u, 0), 3, {128, rest / 8u, chunks}, {128, rest * 16u}, box);
  return ok && encode_map(&m->scales, c + l.atom_at(0, 0), 2, {128, (cuuint64_t)(whole + (rest ? 1u : 0u)) * l.atoms * 4u, 1}, {128, 0}, sbox);
}

// Clusters of `size` CTAs of a kernel that the device holds at once (0: an error): fewer than CTAs divided by size, as a cluster stays within
// a part of the device (of 148 CTAs of the pair kernel, 33 clusters of four, 22 of six, 15 of eight).
template <auto Kernel>
int clusters_at_once(int size, int threads, size_t smem) {
  static std::atomic<int> known[64][9];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || size < 1 || size > 8) return 0;
  if (dev < 64 && known[dev][size].load()) return known[dev][size].load();
  if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMxSmemLimit) != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)size);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, Kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  if (dev < 64) known[dev][size].store(n);
  return n;
}

// Into how many parts to split the common axis: what takes the fewest rounds of stages, where a round of clusters costs `fixed` stages besides and a
// split two more than that.  At least two stages to a part.
template <typename AtOnce>
uint32_t choose_split(uint64_t tiles, uint64_t steps, uint32_t most, uint64_t fixed, AtOnce at_once) {
  uint32_t best = 1;
  uint64_t least = ~0ull;
  for (uint32_t s = 1; s <= most && (s == 1 || 2 * s <= steps); ++s) {
    const int n = at_once(s);
    if (n < 1) continue;
    const uint64_t cost = (tiles + n - 1) / n * ((steps + s - 1) / s + fixed + (s > 1 ? fixed / 2 : 0));
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

template <int DT, int F>
int launch_product_pair(const MxProductArgs& a, cudaStream_t stream) {
  PairArgs p = {};
  p.g = a;
  p.g.tiles_m = (a.m + 255u) / 256u;
  p.g.tiles_n = (a.n + 255u) / 256u;
  if (!encode_operand<F>(&p.a, a.a, a.m, a.k) || !encode_operand<F>(&p.b, a.b, a.n, a.k)) return FH_ERR_UNSUPPORTED;
  const uint64_t tiles = (uint64_t)p.g.tiles_m * p.g.tiles_n;
  auto at_once = [](uint32_t s) { return clusters_at_once<mx_product_pair_kernel<DT, F>>((int)(2 * s), kPairThreads, PairShape<F>::kSmem); };
  // (a tile's start and end take about as long as ten stages)
  p.g.split = choose_split(tiles, ((uint64_t)a.k + 255) / 256, 4, 10, at_once);
  const int n = at_once(1);
  if (n < 1) return FH_ERR_CUDA;
  const uint32_t clusters = (uint32_t)(p.g.split > 1 ? tiles : std::min<uint64_t>(tiles, (uint64_t)n));
  return launch_plain<mx_product_pair_kernel<DT, F>>(clusters * 2u * p.g.split, kPairThreads, PairShape<F>::kSmem, (int)(2u * p.g.split), stream, p);
}

template <int DT, int F, int QT>
int launch_product_t(const MxProductArgs& a0, cudaStream_t stream) {
  MxProductArgs a = a0;
  a.tiles_m = (a.m + 127u) / 128u;
  a.tiles_n = (a.n + 127u) / 128u;
  const uint64_t tiles = (uint64_t)a.tiles_m * a.tiles_n;
  // (the runtime counts one CTA of a cluster to an SM; these fit by shared and by tensor memory)
  using S = ProductShape<F, QT>;
  constexpr int kPerSm = std::min<int>((int)(kSmemPerSm / (S::kSmem + 1024)), (int)(512 / S::kCols));
  auto at_once = [](uint32_t s) { return kPerSm * clusters_at_once<mx_product_kernel<DT, F, QT>>((int)s, kProductThreads, S::kSmem); };
  // (a tile's start and end take about as long as eight stages)
  a.split = choose_split(tiles, ((uint64_t)a.k + 255) / 256, 8, 8, at_once);
  return launch_plain<mx_product_kernel<DT, F, QT>>((uint32_t)tiles * a.split, kProductThreads, ProductShape<F, QT>::kSmem, (int)a.split, stream, a);
}
template <int DT, int F>
int launch_product_df(const MxProductArgs& a, cudaStream_t stream) {
  if (a.m <= 16) return launch_product_t<DT, F, 16>(a, stream);
  if (a.m <= 32) return launch_product_t<DT, F, 32>(a, stream);
  if (a.m <= 64) return launch_product_t<DT, F, 64>(a, stream);
  if (a.m <= 128) return launch_product_t<DT, F, 128>(a, stream);
  return launch_product_pair<DT, F>(a, stream);
}

}  // namespace

int launch_mx_product(const MxProductArgs& a, int dtype, int format, cudaStream_t stream) {
  if (((uint64_t)a.m + 127) / 128 * (((uint64_t)a.n + 127) / 128) > 0x7FFFFFFFull / 8) return FH_ERR_UNSUPPORTED;
  if (dtype == kF32)
    return format == kMxB32 ? launch_product_df<kF32, kMxB32>(a, stream) : launch_product_df<kF32, kMxB16>(a, stream);
  return format == kMxB32 ? launch_product_df<kBF16, kMxB32>(a, stream) : launch_product_df<kBF16, kMxB16>(a, stream);
}

}  // namespace fh
