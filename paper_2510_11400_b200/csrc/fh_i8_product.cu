// Products of 8-bit matrices on the tensor cores, and the gated feed-forward block's two at once.
#include "fh_act.cuh"
#include "fh_i8.cuh"
#include "fh_i8_launch.cuh"
#include "fh_product.cuh"

namespace fh {
namespace {

// C = alpha A B^T (+ C), A m x k and B n x k; or, GATED, h = act(A B^T) * (A U^T) with a second weight U.  As in the products of 4-bit matrices rows of B lie
// along the 128 lanes of an accumulator and rows of A along its columns: a lane owns a column of C, and a single token costs 16 columns.
//
// A stage holds 128 elements of the common axis, one contiguous piece of codes for each operand in the very order the matrix instruction reads.
// Where fewer rows than the instruction reads are stored, it reads on into the next piece, and the rows that come of it are not looked at.  Sums
// are 32-bit integers, so that parts of the common axis join exactly, in any order.
constexpr int kI8Threads = 192;   // four warps for the result, one for copies, one for matrix instructions
constexpr int kI8Chunks = 8;      // 8 x 16 elements to a stage
constexpr uint32_t kI8Step = 16 * kI8Chunks;

template <int QT, bool GATED>
struct I8Shape {
  static constexpr int kW = GATED ? 2 : 1;  // weights
  static constexpr uint32_t kP = 128 * kI8Step, kQ = QT * kI8Step;
  static constexpr uint32_t kStage = kW * kP + kQ;
  // (with few rows of A the bytes under way are what counts, and several CTAs to an SM: 3 of 73 KB, or of two weights 2 of 103 KB)
  static constexpr int kStages = GATED && QT <= 32 ? 3 : 4;
  static constexpr uint32_t kCols = kW * QT < 32 ? 32 : kW * QT;
  static constexpr uint32_t kTail = 256 + (QT + 8) * 4;  // barriers and words, factors of A's rows (and of those behind the last)
  static constexpr size_t kSmem = 128 + (size_t)kStages * kStage + kTail;
  static_assert(kStages * kStage >= kW * (QT + 8) * 512, "partial sums, and rows read behind them");
};

// Factors of sums.  In fp32 a sum is multiplied by its column's scale and then by its row's scale times alpha, each rounded once; where a factor
// is beyond 2^90 or below 2^-90, so that the way there could leave fp32's range, the product is made in 64 bits.
__device__ __forceinline__ bool i8_plain(float f) {
  const float m = fabsf(f);
  return m == 0.0f || (m >= 0x1p-90f && m <= 0x1p90f);
}
__device__ __forceinline__ bool any_of(uint32_t bar, uint32_t threads, bool p) {  // of the threads at a named barrier
  uint32_t r;
  asm volatile("{ .reg .pred p, q; setp.ne.b32 p, %1, 0; barrier.cta.red.or.pred q, %2, %3, p; selp.u32 %0, 1, 0, q; }"
               : "=r"(r)
               : "r"((uint32_t)p), "r"(bar), "r"(threads)
               : "memory");
  return r != 0;
}
struct I8Factors {
  const float* rows;  // the scales of the tile's rows times alpha, in shared memory
  const uint8_t* a;   // the first of their magnitudes
  float alpha, col, up;  // scales of the lane's column of C, and of the second weight's
  // NR sums of rows q ... of the tile, of a column of scale `by`.
  template <int NR>
  __device__ __forceinline__ void apply(const uint32_t (&v)[NR], float (&f)[NR], uint32_t q, float by) const {
#pragma unroll
    for (int x = 0; x < NR; ++x) f[x] = (float)(int32_t)v[x] * by * rows[q + x];
  }
  // One, in 64 bits.
  __device__ __forceinline__ float wide(uint32_t v, uint32_t q, float by) const {
    return (float)((double)(int32_t)v * by * (double)i8_scale(reinterpret_cast<const float*>(a)[q]) * alpha);
  }
};

// What becomes of NR results (GATED: of both weights) of a column of C, rows `row` to `end`.
template <int DT, int NR, int ACT>
__device__ __forceinline__ void i8_put(const I8ProductArgs& g, float (&f)[NR], const float (&u)[NR], uint32_t row, uint32_t end, uint32_t col) {
  if (col >= g.n) return;
  if (ACT < 0) {
    if (g.accumulate) {
      float old[NR];
      load_c<DT, NR>(g.c, g.ldc, row, end, col, old);
#pragma unroll
      for (int x = 0; x < NR; ++x) f[x] += old[x];
    }
    store_c<DT, NR>(g.c, g.ldc, row, end, col, f);
  } else {
    if (g.pre) {
      store_c<DT, NR>(g.pre, g.ldp, row, end, col, f);
      store_c<DT, NR>(g.pre, g.ldp, row, end, g.n + col, u);
    }
    if (g.c) {
#pragma unroll
      for (int x = 0; x < NR; ++x) f[x] = act_of<ACT, DT>(f[x]) * u[x];
      store_c<DT, NR>(g.c, g.ldc, row, end, col, f);
    }
  }
}
// Sums of rows q ... of a tile whose first row is row0.
template <int DT, int NR, int ACT>
__device__ __forceinline__ void i8_put_sums(const I8ProductArgs& g, const I8Factors& by, const uint32_t (&v)[NR], const uint32_t (&w)[NR], uint32_t row0, uint32_t end, uint32_t q,
                                            uint32_t col) {
  float f[NR], u[NR];
  by.apply(v, f, q, by.col);
  if (ACT >= 0) by.apply(w, u, q, by.up);
  i8_put<DT, NR, ACT>(g, f, u, row0 + q, end, col);
}
// One row, in 64 bits.  (Where factors need it a tile is gone through row by row: in line with the others it would take registers from those.)
template <int DT, int ACT>
__device__ __forceinline__ void i8_put_wide(const I8ProductArgs& g, const I8Factors& by, uint32_t v, uint32_t w, uint32_t row0, uint32_t q, uint32_t col) {
  float f[1] = {by.wide(v, q, by.col)}, u[1] = {ACT >= 0 ? by.wide(w, q, by.up) : 0.0f};
  i8_put<DT, 1, ACT>(g, f, u, row0 + q, row0 + q + 1u, col);
}

// Adds up rows of partial sums over the parts of a cluster (CTAs `stride` apart, from `first` on); four parts are asked for at once.
template <int NR>
__device__ __forceinline__ void add_parts(uint32_t at, uint32_t first, uint32_t stride, uint32_t parts, uint32_t (&v)[NR]) {
#pragma unroll
  for (int x = 0; x < NR; ++x) v[x] = 0u;
  for (uint32_t r0 = 0; r0 < parts; r0 += 4u) {
    uint32_t w[4][NR];
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r)
      if (r0 + r < parts) {
#pragma unroll
        for (int x = 0; x < NR; ++x) w[r][x] = __float_as_uint(ld_cluster(at + x * 512u, first + (r0 + r) * stride));
      }
#pragma unroll
    for (uint32_t r = 0; r < 4u; ++r)
      if (r0 + r < parts) {
#pragma unroll
        for (int x = 0; x < NR; ++x) v[x] += w[r][x];
      }
  }
}

__device__ __forceinline__ float i8_scale_at(const uint8_t* c, const I8Layout& l, uint32_t row) {
  return row < l.rows ? i8_scale(*reinterpret_cast<const float*>(c + l.magnitude_at(row))) : 0.0f;
}

template <int DT, int QT, int ACT>
__global__ void __launch_bounds__(kI8Threads) i8_product_kernel(const I8ProductArgs g) {
  constexpr bool GATED = ACT >= 0;
  using S = I8Shape<QT, GATED>;
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
  float* factors = reinterpret_cast<float*>(tail + 256);
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t rank = g.split > 1 ? cluster_rank() : 0u;
  const uint32_t cell = blockIdx.x / g.split, tp = cell % g.tiles_n, tq = cell / g.tiles_n;  // (clusters are along x)
  const I8Layout lp(g.n, g.k), lq(g.m, g.k);
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
  // Containers that are large enough are multiplied, whatever their headers say, and the result is written when those are right: waiting for them first is a
  // latency that a single token's product would see.
  const bool sized = g.a_bytes >= lq.total && g.b_bytes >= lp.total && (!GATED || g.up_bytes >= lp.total);
  const uint32_t chunks = lp.chunks(), steps = (chunks + kI8Chunks - 1u) / kI8Chunks;
  const uint32_t first = (uint32_t)((uint64_t)steps * rank / g.split), last = (uint32_t)((uint64_t)steps * (rank + 1u) / g.split);
  const uint32_t rp = lp.block_rows(tp), rq = lq.block_rows(tq);
  if (sized && warp == 4) {
    if (lane == 0) {
      const uint64_t at = lp.code_at(tp * 128u, 0);
      const uint8_t* q = g.a + lq.code_at(tq * 128u, 0);
      uint32_t loaded = 0;
      Turn<S::kStages> turn;
      for (uint32_t it = first; it < last && loaded != g.silent; ++it, ++loaded, turn.next()) {
        const uint32_t s = turn.stage;
        if (loaded >= (uint32_t)S::kStages && !mbar_poll<false>(empty + s, turn.round ^ 1u, g.polls, abort)) {
          *abort = 1u;
          break;
        }
        const uint32_t nc = min((uint32_t)kI8Chunks, chunks - it * kI8Chunks);
        uint8_t* st = smem + s * S::kStage;
        const uint64_t p_at = at + (uint64_t)it * kI8Chunks * 16u * rp;
        mbar_expect_tx(full + s, nc * 16u * (S::kW * rp + rq));
        bulk_g2s(st, g.b + p_at, nc * 16u * rp, full + s);
        if (GATED) bulk_g2s(st + S::kP, g.up + p_at, nc * 16u * rp, full + s);
        bulk_g2s(st + S::kW * S::kP, q + (uint64_t)it * kI8Chunks * 16u * rq, nc * 16u * rq, full + s);
      }
      *loads = loaded;
    }
  } else if (sized && warp == 5) {
    if (lane == 0) {
      Turn<S::kStages> turn;
      for (uint32_t it = first; it < last; ++it, turn.next()) {
        const uint32_t s = turn.stage;
        if (!mbar_poll<false>(full + s, turn.round, g.polls, abort)) {
          *abort = 1u;
          break;
        }
        tc_fence_after();
        const uint32_t nc = min((uint32_t)kI8Chunks, chunks - it * kI8Chunks);
        const uint32_t st = smem_u32(smem) + s * S::kStage;
        const uint64_t dp = smem_desc(st, rp * 16u, 128u), du = smem_desc(st + S::kP, rp * 16u, 128u), dq = smem_desc(st + S::kW * S::kP, rq * 16u, 128u);
#pragma unroll
        for (uint32_t x = 0; x < kI8Chunks / 2u; ++x)
          if (2u * x < nc) {
            tc_mma_i8<false>(tmem, dp + 2u * x * rp, dq + 2u * x * rq, i8_idesc(128u, QT), it > first || x > 0u);
            if (GATED) tc_mma_i8<false>(tmem + QT, du + 2u * x * rp, dq + 2u * x * rq, i8_idesc(128u, QT), it > first || x > 0u);
          }
        if (it + (uint32_t)S::kStages < last) tc_commit(empty + s);
      }
      tc_commit(done);
    }
  }
  __syncwarp();
  // the accumulator: lane i of warp w has row 32 w + i of the tile of B, QT columns for the rows of A
  const bool mine = sized && warp < 4;
  const uint32_t col = tp * 128u + warp * 32u + lane, rows = min((uint32_t)QT, g.m - tq * 128u);
  I8Factors by = {factors, g.a + lq.magnitude_at(tq * 128u), g.alpha, 0.0f, 0.0f};
  bool good = mine, wide = false, ok = false;
  if (warp < 4) {
    const bool ok_a = i8_header_ok(g.a, g.a_bytes, lq), ok_b = i8_header_ok(g.b, g.b_bytes, lp), ok_u = !GATED || i8_header_ok(g.up, g.up_bytes, lp);
    ok = ok_a && ok_b && ok_u;
    if (blockIdx.x == 0 && tid == 0 && g.status) *g.status = ok ? 0ull : status_word(kErrCorrupt);
  }
  if (mine) {
    by.col = i8_scale_at(g.b, lp, col);
    if (GATED) by.up = i8_scale_at(g.up, lp, col);
    wide = !i8_plain(by.col) || !i8_plain(by.up);
    if (tid < (uint32_t)QT) {
      const float s = i8_scale_at(g.a, lq, tq * 128u + tid), f = s * g.alpha;
      factors[tid] = f;
      wide = wide || !i8_plain(f) || !i8_plain(s) || (f == 0.0f && s != 0.0f && g.alpha != 0.0f);
    }
    wide = any_of(1u, 128u, wide);
    good = mbar_poll_warp(done, 0u, g.polls, abort);
    if (!good && lane == 0) *abort = 1u;
    tc_fence_after();
  }
  constexpr int NR = 16;
  const uint32_t at = tmem + (warp * 32u << 16);
  if (g.split == 1u) {
    if (good && ok && !wide) {
#pragma unroll 1
      for (uint32_t q = 0; q < rows; q += NR) {
        uint32_t v[NR], w[NR] = {};
        tc_load16(at + q, v);
        if (GATED) tc_load16(at + QT + q, w);
        tc_load_wait();
        i8_put_sums<DT, NR, ACT>(g, by, v, w, tq * 128u, g.m, q, col);
      }
    } else if (good && ok) {
#pragma unroll 1
      for (uint32_t q = 0; q < rows; ++q) {
        const uint32_t v = tc_load1(at + q), w = GATED ? tc_load1(at + QT + q) : 0u;
        tc_load_wait();
        i8_put_wide<DT, ACT>(g, by, v, w, tq * 128u, q, col);
      }
    }
  } else {
    // partial sums of the cluster's CTAs, each over its part of the common axis: to shared memory (all copies into it have been used),
    // then every CTA adds up some rows of C
    uint32_t* part = reinterpret_cast<uint32_t*>(smem);
    if (good) {
#pragma unroll 1
      for (uint32_t q = 0; q < (uint32_t)(S::kW * QT); q += NR) {
        uint32_t v[NR];
        tc_load16(at + q, v);
        tc_load_wait();
#pragma unroll
        for (uint32_t x = 0; x < (uint32_t)NR; ++x) part[(q + x) * 128u + tid] = v[x];
      }
    }
    cluster_sync();
    if (good && ok) {
      const uint32_t end = rows * (rank + 1u) / g.split;
      constexpr int N = QT < 32 ? 2 : 8;
      const uint32_t step = wide ? 1u : N;
#pragma unroll 1
      for (uint32_t q = rows * rank / g.split; q < end; q += step) {
        uint32_t v[N], w[N] = {};
        add_parts<N>(smem_u32(part + q * 128u + tid), 0u, 1u, g.split, v);  // (rows behind the last: stage bytes)
        if (GATED) add_parts<N>(smem_u32(part + (QT + q) * 128u + tid), 0u, 1u, g.split, w);
        if (wide)
          i8_put_wide<DT, ACT>(g, by, v[0], w[0], tq * 128u, q, col);
        else
          i8_put_sums<DT, N, ACT>(g, by, v, w, tq * 128u, tq * 128u + end, q, col);
      }
    }
    cluster_sync();
  }
  tc_fence_before();
  __syncthreads();
  if (*abort) {  // (see "Waits" in fh_product.cuh)
    if (sized && lane == 0 && warp == 4)
      for (uint32_t n = *loads, w = n > (uint32_t)S::kStages ? n - S::kStages : 0u; w < n; ++w) mbar_wait(full + w % S::kStages, w / S::kStages & 1u, kDrainPolls);
    if (sized && lane == 0 && warp == 5) {
      tc_commit(idle);
      mbar_wait(idle, 0u, kDrainPolls);
    }
    if (tid == 0 && g.status) *g.status = status_word(kErrTimeout);
    __syncthreads();
  }
  if (warp == 5) tmem_free(tmem, S::kCols);
}

// More rows of A: a pair of CTAs on a tile of 256 columns of C, 128 rows of B (and of U) and 128 of the tile's 256 rows of A in the shared memory of each.
// Pairs take tiles one after the other.  The eight warps for the result take the accumulators into registers, 128 columns at a time, before they write: the
// word that tensor memory is free would wait for what the thread has stored.  A product's accumulators alternate between the halves of tensor memory, so that
// the next tile's matrix instructions run meanwhile; two weights' take all of it.  (With 128 rows of A to a tile they alternated too, but a stage then moved
// 80 bytes a clock from L2 to an SM instead of 48: 4096 x 8192 x 4096 253 us and 194.)  With a split, a cluster's pairs share one tile.
constexpr int kI8PairThreads = 320;  // eight warps for the result, then one each for loads and matrix instructions

template <bool GATED>
struct I8PairShape {
  static constexpr int kW = GATED ? 2 : 1;
  static constexpr uint32_t kQ = 256;                              // rows of A to a tile
  static constexpr uint32_t kSums = kW * kQ, kBufs = 512 / kSums;  // columns of tensor memory that a tile takes, tiles that have room
  static constexpr uint32_t kP = 128 * kI8Step;
  static constexpr uint32_t kStage = (kW + 1) * kP;
  static constexpr int kStages = 200 * 1024 / kStage;
  static constexpr uint32_t kTail = 256 + 2 * kQ * 4;
  static constexpr size_t kSmem = 128 + (size_t)kStages * kStage + kTail;
  static constexpr uint32_t kMostSplit = GATED ? 1 : 4;  // (two weights' partial sums do not fit the stages)
  static_assert(kSmem <= kMxSmemLimit && (GATED || kStages * kStage >= (kQ + 8) * 512), "room; partial sums, and rows read behind them");
  // the barriers behind the stages
  static constexpr int kEmpty = kStages;          // a stage may be loaded again
  static constexpr int kDone = 2 * kStages;       // an accumulator is complete (one for each of the two)
  static constexpr int kTaken = kDone + 2;        // even CTA: both CTAs' warps have taken it
  static constexpr int kIdle = kTaken + 2;        // even CTA, after a wait that ran out: what was issued is complete
  static constexpr int kWords = kIdle + 1;
  static_assert(kWords * 8 + 12 <= 256, "room behind the stages");
};

struct I8Maps {
  CUtensorMap codes;  // of the blocks of 128 rows: 128 bytes (eight rows), 16 of them, every chunk
  CUtensorMap rest;   // of the last block, if it has fewer rows: the copies fill up with zeros
};
struct I8PairArgs {
  I8Maps a, b, up;
  I8ProductArgs g;
};

// Where a block of 128 rows of an operand is.  One that the matrix does not have is behind the end of the map: its copies bring zeros.
struct I8Source {
  const CUtensorMap* map;
  uint32_t z;
  __device__ __forceinline__ I8Source(const I8Maps& m, const I8Layout& l, uint32_t block) {
    const uint32_t whole = l.r8 / 128u, c = l.chunks();
    const bool rest = whole == 0u || (block == whole && l.r8 % 128u != 0u);
    map = rest ? &m.rest : &m.codes;
    z = rest ? (block == whole ? 0u : c) : min(block, whole) * c;
  }
};

template <int DT, int ACT>
__global__ void __launch_bounds__(kI8PairThreads, 1) i8_pair_kernel(const __grid_constant__ I8PairArgs pa) {
  constexpr bool GATED = ACT >= 0;
  const I8ProductArgs& g = pa.g;
  using S = I8PairShape<GATED>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = stages_at(smem_raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  uint64_t *empty = full + S::kEmpty, *sums = full + S::kDone, *taken = full + S::kTaken, *idle = full + S::kIdle;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(full + S::kWords);
  volatile uint32_t* abort = tmem_at + 1;
  uint32_t* loads = tmem_at + 2;  // stages that the loading thread has asked for
  float* factors = reinterpret_cast<float*>(smem + S::kStages * S::kStage + 256);
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t crank = cluster_rank(), half = crank & 1u, even = crank & ~1u, rank = crank / 2u;
  const uint32_t pairs = gridDim.x / (2u * g.split), pair = blockIdx.x / (2u * g.split);  // clusters, each on tiles of its own
  const I8Layout lp(g.n, g.k), lq(g.m, g.k);
  if (tid == 0) {
    for (int i = 0; i < S::kStages; ++i) {
      mbar_init(full + i, 1);
      mbar_init(empty + i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(sums + i, 1);
      mbar_init(taken + i, 16);
    }
    mbar_init(idle, 1);
    *abort = 0u;
    fence_mbar_init();
  }
  if (warp == 9) {
    tmem_alloc_pair(tmem_at, 512u);
    tmem_last_alloc_pair();
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // (both CTAs' barriers stand)
  tc_fence_after();
  const uint32_t tmem = *tmem_at;
  dep_trigger();  // (behind the allocation: no later kernel takes tensor memory that this one still wants)
  dep_wait();
  const bool sized = g.a_bytes >= lq.total && g.b_bytes >= lp.total && (!GATED || g.up_bytes >= lp.total);  // (as in the kernel for few rows)
  const uint32_t chunks = lp.chunks(), steps = (chunks + kI8Chunks - 1u) / kI8Chunks;
  const uint32_t first = (uint32_t)((uint64_t)steps * rank / g.split), last = (uint32_t)((uint64_t)steps * (rank + 1u) / g.split);
  const uint32_t tiles = sized ? g.tiles_m * g.tiles_n : 0u;
  bool good = true, ok = false;
  if (warp == 8) {
    if (lane == 0) {
      uint32_t loaded = 0;
      const uint32_t silent = half ? g.silent : ~0u;
      Turn<S::kStages> turn;
      for (uint32_t tile = pair; tile < tiles && good; tile += pairs) {
        const PairTile where(tile, g.tiles_m, g.tiles_n);
        const I8Source p(pa.b, lp, where.n * 2u + half), u(pa.up, lp, where.n * 2u + half);
        const I8Source q(pa.a, lq, where.m * 2u + half);
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
          const uint32_t st = smem_u32(smem) + turn.stage * S::kStage, bar = at_rank(full + turn.stage, even), z = it * kI8Chunks;
          if (half == 0u) mbar_expect_tx(full + turn.stage, 2u * S::kStage);
          tma_pair_3d(st, p.map, 0u, 0u, p.z + z, bar);
          if (GATED) tma_pair_3d(st + S::kP, u.map, 0u, 0u, u.z + z, bar);
          tma_pair_3d(st + S::kW * S::kP, q.map, 0u, 0u, q.z + z, bar);
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
        const uint32_t buf = n % S::kBufs, acc = tmem + buf * S::kSums;
        if (n >= S::kBufs && !mbar_poll<true>(taken + buf, (n / S::kBufs - 1u) & 1u, g.polls, abort)) {
          raise_cluster(abort, 2u * g.split);
          break;
        }
        tc_fence_after();
        for (uint32_t it = first; it < last; ++it, turn.next()) {
          const uint32_t s = turn.stage;
          if (!mbar_poll<true>(full + s, turn.round, g.polls, abort)) {
            raise_cluster(abort, 2u * g.split);
            good = false;
            break;
          }
          tc_fence_after();
          const uint32_t nc = min((uint32_t)kI8Chunks, chunks - it * kI8Chunks);
          const uint32_t st = smem_u32(smem) + s * S::kStage;
          const uint64_t dp = smem_desc(st, 2048u, 128u), du = smem_desc(st + S::kP, 2048u, 128u), dq = smem_desc(st + S::kW * S::kP, 2048u, 128u);
#pragma unroll
          for (uint32_t x = 0; x < kI8Chunks / 2u; ++x)
            if (2u * x < nc) {
              tc_mma_i8<true>(acc, dp + 256u * x, dq + 256u * x, i8_idesc(256u, S::kQ), it > first || x > 0u);
              if (GATED) tc_mma_i8<true>(acc + S::kQ, du + 256u * x, dq + 256u * x, i8_idesc(256u, S::kQ), it > first || x > 0u);
            }
          if (it + (uint32_t)S::kStages < last || tile + pairs < tiles) tc_commit_pair(empty + s, both);
        }
        if (good) tc_commit_pair(sums + buf, both);
      }
    }
  } else {
    constexpr uint32_t kSide = S::kQ / 2u, kRun = 128u / S::kW;  // columns of an accumulator to each four warps: rows of A; those of them in registers at once
    const uint32_t side = warp / 4u * kSide;
    const bool ok_a = i8_header_ok(g.a, g.a_bytes, lq), ok_b = i8_header_ok(g.b, g.b_bytes, lp), ok_u = !GATED || i8_header_ok(g.up, g.up_bytes, lp);
    ok = ok_a && ok_b && ok_u;
    if (blockIdx.x == 0 && tid == 0 && g.status) *g.status = ok ? 0ull : status_word(kErrCorrupt);
    // The magnitudes of a tile are asked for a tile ahead.
    float next_col = 0.0f, next_up = 0.0f, next_row = 0.0f;
    auto ask = [&](uint32_t tile) {
      const PairTile where(tile, g.tiles_m, g.tiles_n);
      const uint32_t col = where.n * 256u + half * 128u + warp % 4u * 32u + lane, row = where.m * S::kQ + tid;
      next_col = col < lp.rows ? *reinterpret_cast<const float*>(g.b + lp.magnitude_at(col)) : 0.0f;
      if (GATED) next_up = col < lp.rows ? *reinterpret_cast<const float*>(g.up + lp.magnitude_at(col)) : 0.0f;
      if (tid < S::kQ) next_row = row < lq.rows ? *reinterpret_cast<const float*>(g.a + lq.magnitude_at(row)) : 0.0f;
    };
    if (pair < tiles) ask(pair);
    uint32_t n = 0;
    for (uint32_t tile = pair; tile < tiles; tile += pairs, ++n) {
      const PairTile where(tile, g.tiles_m, g.tiles_n);
      const uint32_t col = where.n * 256u + half * 128u + warp % 4u * 32u + lane, row0 = where.m * S::kQ, rows = min(S::kQ, g.m - row0), buf = n % S::kBufs;
      const I8Factors by = {factors + (n & 1u) * S::kQ, g.a + lq.magnitude_at(row0), g.alpha, i8_scale(next_col), i8_scale(next_up)};
      float* fa = factors + (n & 1u) * S::kQ;  // (the other half may still be read by warps that are a tile behind)
      if (tid < S::kQ) {
        const float s = i8_scale(next_row), f = s * g.alpha;
        fa[tid] = i8_plain(s) && i8_plain(f) && (f != 0.0f || s == 0.0f || g.alpha == 0.0f) ? f : __uint_as_float(0x7FC00000u);
      }
      if (tile + pairs < tiles) ask(tile + pairs);
      if (any_of(1u, 256u, !good)) break;  // (all warps stay or none does: they meet here)
      bool wide = !i8_plain(by.col) || !i8_plain(by.up);
#pragma unroll
      for (uint32_t q = 0; q < S::kQ; q += 32u) wide = wide || fa[q + lane] != fa[q + lane];
      wide = __any_sync(0xFFFFFFFFu, wide);
      good = mbar_poll_warp(sums + buf, n / S::kBufs & 1u, g.polls, abort);
      if (!good) {
        if (lane == 0) raise_cluster(abort, 2u * g.split);
        continue;
      }
      tc_fence_after();
      const uint32_t at = tmem + buf * S::kSums + (warp % 4u * 32u << 16) + side;
      if (wide && (GATED || g.split == 1u)) {
#pragma unroll 1
        for (uint32_t q = 0; q < kSide; ++q) {
          const uint32_t v = tc_load1(at + q), w = GATED ? tc_load1(at + S::kQ + q) : 0u;
          tc_load_wait();
          if (ok && side + q < rows) i8_put_wide<DT, ACT>(g, by, v, w, row0, side + q, col);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_at(taken + buf, even);
        continue;
      }
#pragma unroll 1
      for (uint32_t run = 0; run < kSide; run += kRun) {
        uint32_t v[kRun / 16u][16], w[GATED ? kRun / 16u : 1u][16];
#pragma unroll
        for (uint32_t x = 0; x < kRun / 16u; ++x) {
          tc_load16(at + run + 16u * x, v[x]);
          if (GATED) tc_load16(at + S::kQ + run + 16u * x, w[x]);
        }
        tc_load_wait();
        if (run + kRun == kSide) {  // (ahead of this tile's stores: the release would wait for them)
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_at(taken + buf, even);
        }
        if (GATED || g.split == 1u) {
#pragma unroll
          for (uint32_t x = 0; x < kRun / 16u; ++x) {
            const uint32_t q = side + run + 16u * x;
            if (ok && q < rows) i8_put_sums<DT, 16, ACT>(g, by, v[x], w[GATED ? x : 0u], row0, g.m, q, col);
          }
        } else {  // (one tile only: all copies into shared memory have been used)
          uint32_t* part = reinterpret_cast<uint32_t*>(smem) + (side + run) * 128u + warp % 4u * 32u + lane;
#pragma unroll
          for (uint32_t x = 0; x < kRun / 16u; ++x)
#pragma unroll
            for (uint32_t y = 0; y < 16u; ++y) part[(16u * x + y) * 128u] = v[x][y];
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  if (!GATED && g.split > 1u) {
    cluster_sync();
    if (warp < 8u && tiles && ok && !*abort) {
      const PairTile where(pair, g.tiles_m, g.tiles_n);
      const uint32_t p = warp % 4u * 32u + lane, col = where.n * 256u + half * 128u + p, row0 = where.m * S::kQ;
      const uint32_t rows = min(S::kQ, g.m - row0), from = rows * rank / g.split, end = rows * (rank + 1u) / g.split, mid = (from + end) / 2u;
      const uint32_t stop = warp < 4u ? mid : end;
      const I8Factors by = {factors, g.a + lq.magnitude_at(row0), g.alpha, i8_scale_at(g.b, lp, col), 0.0f};
      bool wide = !i8_plain(by.col);
      for (uint32_t q = lane; q < rows; q += 32u) wide = wide || factors[q] != factors[q];
      wide = __any_sync(0xFFFFFFFFu, wide);
      const uint32_t step = wide ? 1u : 8u;
#pragma unroll 1
      for (uint32_t q = warp < 4u ? from : mid; q < stop; q += step) {
        uint32_t v[8], w[8] = {};
        add_parts<8>(smem_u32(reinterpret_cast<uint32_t*>(smem) + q * 128u + p), half, 2u, g.split, v);
        if (wide)
          i8_put_wide<DT, ACT>(g, by, v[0], w[0], row0, q, col);
        else
          i8_put_sums<DT, 8, ACT>(g, by, v, w, row0, row0 + stop, q, col);
      }
    }
  }
  __syncthreads();
  cluster_sync();  // (a pair's memory serves both until both are done)
  if (*abort) {    // (in all CTAs of the cluster or in none; see "Waits" in fh_product.cuh)
    uint64_t* bars = reinterpret_cast<uint64_t*>(stages_at(smem_raw, hidden_zero()) + S::kStages * S::kStage);
    const uint32_t me = cluster_rank(), who = threadIdx.x;
    if (me % 2u == 0u && who == 8u * 32u) {
      // The pair's loading threads may have stopped at different stages, and a barrier counts the bytes of both: those that the odd CTA
      // has not asked for are taken off, those that it alone has asked for are expected.
      const uint32_t* count = reinterpret_cast<const uint32_t*>(bars + S::kWords) + 2;
      const uint32_t mine = *count, other = ld_cluster_u32(count, me ^ 1u), most = max(mine, other);
#pragma unroll 1
      for (uint32_t w = min(mine, other); w < most; ++w) {
        if (mine < other)
          mbar_expect_tx(bars + w % S::kStages, S::kStage);
        else
          mbar_complete_tx(bars + w % S::kStages, S::kStage);
      }
#pragma unroll 1
      for (uint32_t w = most > (uint32_t)S::kStages ? most - S::kStages : 0u; w < most; ++w) mbar_wait(bars + w % S::kStages, w / S::kStages & 1u, kDrainPolls);
    }
    if (me % 2u == 0u && who == 9u * 32u) {
      tc_commit_pair(bars + S::kIdle, (uint16_t)(1u << me));
      mbar_wait(bars + S::kIdle, 0u, kDrainPolls);
    }
    if (who == 0u && g.status) *g.status = status_word(kErrTimeout);
    __syncthreads();
    cluster_sync();
  }
  if (warp == 9) tmem_free_pair(tmem, 512u);
}

bool encode_i8(I8Maps* m, const uint8_t* c, uint32_t rows, uint32_t k) {
  const I8Layout l(rows, k);
  const uint32_t whole = l.r8 / 128u, rest = l.r8 % 128u, chunks = l.chunks();
  const cuuint32_t box[3] = {128, 16, (cuuint32_t)kI8Chunks};
  // (coordinates are signed 32-bit numbers, one tile's steps behind the end included)
  if ((uint64_t)(whole + 2u) * chunks + kI8Chunks > 0x7FFFFFFFull) return false;
  bool ok = true;
  if (whole) ok = encode_map(&m->codes, c + kI8HeadBytes, 3, {128, 16, (cuuint64_t)whole * chunks}, {128, 2048}, box);
  if (rest) ok = ok && encode_map(&m->rest, c + l.code_at(whole * 128u, 0), 3, {128, rest / 8u, chunks}, {128, rest * 16u}, box);
  return ok;
}

template <int DT, int ACT>
int launch_i8_pair(const I8ProductArgs& a, cudaStream_t stream) {
  using S = I8PairShape<(ACT >= 0)>;
  I8PairArgs p = {};
  p.g = a;
  p.g.tiles_m = (uint32_t)(((uint64_t)a.m + S::kQ - 1u) / S::kQ);
  p.g.tiles_n = (a.n + 255u) / 256u;
  if (!encode_i8(&p.a, a.a, a.m, a.k) || !encode_i8(&p.b, a.b, a.n, a.k) || (ACT >= 0 && !encode_i8(&p.up, a.up, a.n, a.k)))
    return FH_ERR_UNSUPPORTED;
  const uint64_t tiles = (uint64_t)p.g.tiles_m * p.g.tiles_n;
  auto at_once = [](uint32_t s) { return clusters_at_once<i8_pair_kernel<DT, ACT>>((int)(2 * s), kI8PairThreads, S::kSmem); };
  // (a tile's start and end take about as long as ten stages)
  p.g.split = choose_split(tiles, ((uint64_t)a.k + kI8Step - 1) / kI8Step, S::kMostSplit, 10, at_once);
  const int n = at_once(1);
  if (n < 1) return FH_ERR_CUDA;
  const uint32_t clusters = (uint32_t)(p.g.split > 1 ? tiles : std::min<uint64_t>(tiles, (uint64_t)n));
  return launch_plain<i8_pair_kernel<DT, ACT>>(clusters * 2u * p.g.split, kI8PairThreads, S::kSmem, (int)(2u * p.g.split), stream, p);
}

template <int DT, int QT, int ACT>
int launch_i8_few(const I8ProductArgs& a0, cudaStream_t stream) {
  I8ProductArgs a = a0;
  a.tiles_m = (a.m + 127u) / 128u;
  a.tiles_n = (a.n + 127u) / 128u;
  const uint64_t tiles = (uint64_t)a.tiles_m * a.tiles_n;
  // (the runtime counts one CTA of a cluster to an SM; these fit by shared and by tensor memory)
  using S = I8Shape<QT, (ACT >= 0)>;
  constexpr int kPerSm = std::min<int>((int)(kSmemPerSm / (S::kSmem + 1024)), (int)(512 / S::kCols));
  auto at_once = [](uint32_t s) { return kPerSm * clusters_at_once<i8_product_kernel<DT, QT, ACT>>((int)s, kI8Threads, S::kSmem); };
  // (a tile's start and end take about as long as eight stages)
  a.split = choose_split(tiles, ((uint64_t)a.k + kI8Step - 1) / kI8Step, 8, 8, at_once);
  return launch_plain<i8_product_kernel<DT, QT, ACT>>((uint32_t)tiles * a.split, kI8Threads, S::kSmem, (int)a.split, stream, a);
}

template <int DT, int ACT>
int launch_i8(const I8ProductArgs& a, cudaStream_t stream) {
  if (((uint64_t)a.m + 127) / 128 * (((uint64_t)a.n + 127) / 128) > 0x7FFFFFFFull / 8) return FH_ERR_UNSUPPORTED;
  if (a.m <= 16) return launch_i8_few<DT, 16, ACT>(a, stream);
  if (a.m <= 32) return launch_i8_few<DT, 32, ACT>(a, stream);
  if (a.m <= 64) return launch_i8_few<DT, 64, ACT>(a, stream);
  if (a.m <= 128) return launch_i8_few<DT, 128, ACT>(a, stream);
  return launch_i8_pair<DT, ACT>(a, stream);
}

template <int ACT>
int launch_by_type(const I8ProductArgs& a, int dtype, cudaStream_t stream) {
  return dtype == kF32 ? launch_i8<kF32, ACT>(a, stream) : launch_i8<kBF16, ACT>(a, stream);
}

}  // namespace

int launch_i8_product(const I8ProductArgs& a, int dtype, cudaStream_t stream) { return launch_by_type<-1>(a, dtype, stream); }

int launch_i8_gated(const I8ProductArgs& a, int dtype, int activation, cudaStream_t stream) {
  if (activation == FH_SILU) return launch_by_type<FH_SILU>(a, dtype, stream);
  if (activation == FH_GELU) return launch_by_type<FH_GELU>(a, dtype, stream);
  if (activation == FH_GELU_TANH) return launch_by_type<FH_GELU_TANH>(a, dtype, stream);
  return launch_by_type<FH_RELU>(a, dtype, stream);
}

}  // namespace fh
