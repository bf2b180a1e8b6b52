// Products of microscaled 4-bit matrices on the tensor cores.
#include <algorithm>

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
constexpr uint32_t kWaitPolls = 1u << 20;

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
  static constexpr size_t kSmem = 128 + kStages * kStage + 256;
  static_assert(kStages * kStage >= QT * 512, "partial sums");
};

struct ProductScale {
  float a, b, alpha;
};

template <int DT>
__device__ __forceinline__ void store_c(uint8_t* c, uint64_t at, float v, bool add) {
  if (DT == kF32) {
    float* p = reinterpret_cast<float*>(c) + at;
    *p = add ? *p + v : v;
  } else {
    __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(c) + at;
    *p = __float2bfloat16_rn(add ? __bfloat162float(*p) + v : v);
  }
}

template <int DT, int F, int QT>
__global__ void __launch_bounds__(kProductThreads) mx_product_kernel(const MxProductArgs g) {
  using S = ProductShape<F, QT>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  uint8_t* tail = smem + S::kStages * S::kStage;
  uint64_t* full = reinterpret_cast<uint64_t*>(tail);
  uint64_t* empty = full + S::kStages;
  uint64_t* done = empty + S::kStages;
  uint32_t* tmem_at = reinterpret_cast<uint32_t*>(done + 1);
  volatile uint32_t* abort = tmem_at + 1;
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
      uint32_t i = 0;
      for (uint32_t it = first; it < last; ++it, ++i) {
        const uint32_t s = i % S::kStages;
        if (i >= (uint32_t)S::kStages && !mbar_wait(empty + s, (i / S::kStages - 1u) & 1u, kWaitPolls)) {
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
      // nothing may be in flight when the CTA ends
      for (uint32_t w = i > (uint32_t)S::kStages ? i - S::kStages : 0u; w < i; ++w) mbar_wait(full + w % S::kStages, w / S::kStages & 1u, kWaitPolls);
    }
  } else if (ok && warp == 5) {
    if (lane == 0) {
      uint32_t i = 0;
      for (uint32_t it = first; it < last; ++it, ++i) {
        const uint32_t s = i % S::kStages;
        if (!mbar_wait_abortable(full + s, i / S::kStages & 1u, kWaitPolls, abort)) {
          *abort = 1u;
          break;
        }
        tc_fence_after();
        const uint32_t nc = min((uint32_t)kStepChunks, chunks - it * kStepChunks);
        const uint32_t na = min((uint32_t)S::kAtoms, lp.atoms - it * S::kAtoms);
        const uint32_t st = smem_u32(smem + s * S::kStage);
        const uint32_t sa = tmem + S::kAcc + s * 2u * S::kScaleCols, sb = sa + S::kScaleCols;
        for (uint32_t x = 0; x < na; ++x) {
          tc_copy_scales(sa + 4u * x, smem_desc(st + S::kP + S::kQ + 512u * x, 128u, 128u));
          tc_copy_scales(sb + 4u * x, smem_desc(st + S::kP + S::kQ + S::kS + 512u * x, 128u, 128u));
        }
        for (uint32_t x = 0; x < nc / 2u; ++x) {
          const uint64_t da = smem_desc(st + x * 32u * rp, rp * 16u, 128u), db = smem_desc(st + S::kP + x * 32u * rq, rq * 16u, 128u);
          const uint32_t word = F == kMxB32 ? x / 2u : x, id = F == kMxB32 ? x % 2u * 2u : 0u;
          tc_mma_mx<F == kMxB32>(tmem, da, db, mx_idesc(128u, QT, F == kMxB32, id), sa + 4u * word, sb + 4u * word, i > 0u || x > 0u);
        }
        tc_commit(empty + s);
      }
      tc_commit(done);
    }
  }
  __syncwarp();
  // the accumulator: lane i of warp w has row 32 w + i of the tile of B, QT columns for the rows of A
  const bool mine = ok && warp < 4;
  bool good = mine;
  if (mine) {
    good = __all_sync(0xFFFFFFFFu, mbar_wait_abortable(done, 0u, kWaitPolls, abort) && !*abort);
    tc_fence_after();
  }
  const uint32_t col = tp * 128u + warp * 32u + lane;
  const int e = ea + eb, e1 = e / 2;
  const float f1 = pow2_f(e1), f2 = pow2_f(e - e1);  // (in two steps: neither over- nor underflows where the result does not)
  if (g.split == 1u) {
    if (good) {
#pragma unroll 1
      for (uint32_t q0 = 0; q0 < (uint32_t)QT; q0 += 16u) {
        uint32_t v[16];
        tc_load16(tmem + (warp * 32u << 16) + q0, v);
        tc_load_wait();
#pragma unroll
        for (uint32_t x = 0; x < 16u; ++x) {
          const uint32_t row = tq * 128u + q0 + x;
          if (row < g.m && col < g.n) store_c<DT>(g.c, (uint64_t)row * g.ldc + col, bits_f(v[x]) * f1 * f2 * g.alpha, g.accumulate);
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
      const uint32_t rows = min((uint32_t)QT, g.m - tq * 128u);
      for (uint32_t q = rows * rank / g.split; q < rows * (rank + 1u) / g.split; ++q) {
        float v = 0.0f;
        for (uint32_t r = 0; r < g.split; ++r) v += ld_cluster(smem_u32(part + q * 128u + tid), r);
        store_c<DT>(g.c, (uint64_t)(tq * 128u + q) * g.ldc + col, v * f1 * f2 * g.alpha, g.accumulate);
      }
    }
    cluster_sync();
  }
  if (mine && !good && tid == 0 && g.status) *g.status = status_word(kErrTimeout);
  tc_fence_before();
  __syncthreads();
  if (warp == 5) tmem_free(tmem, S::kCols);
}

template <int DT, int F, int QT>
int launch_product_t(const MxProductArgs& a, cudaStream_t stream) {
  return launch_plain<mx_product_kernel<DT, F, QT>>(a.tiles_m * a.tiles_n * a.split, kProductThreads, ProductShape<F, QT>::kSmem,
                                                    (int)a.split, stream, a);
}
template <int DT, int F>
int launch_product_df(const MxProductArgs& a, cudaStream_t stream) {
  if (a.m <= 16) return launch_product_t<DT, F, 16>(a, stream);
  if (a.m <= 32) return launch_product_t<DT, F, 32>(a, stream);
  if (a.m <= 64) return launch_product_t<DT, F, 64>(a, stream);
  return launch_product_t<DT, F, 128>(a, stream);
}

}  // namespace

int launch_mx_product(const MxProductArgs& a0, int dtype, int format, cudaStream_t stream) {
  MxProductArgs a = a0;
  const uint64_t tm = ((uint64_t)a.m + 127) / 128, tn = ((uint64_t)a.n + 127) / 128;
  const int sms = sm_count();
  if (sms < 1) return FH_ERR_CUDA;
  // parts of the common axis while that leaves SMs idle, each of at least two stages
  const uint64_t steps = ((uint64_t)a.k + 255) / 256;
  uint64_t split = std::min<uint64_t>({8, (uint64_t)sms / (tm * tn), steps / 2});
  if (split < 1) split = 1;
  if (tm * tn * split > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
  a.tiles_m = (uint32_t)tm;
  a.tiles_n = (uint32_t)tn;
  a.split = (uint32_t)split;
  if (dtype == kF32)
    return format == kMxB32 ? launch_product_df<kF32, kMxB32>(a, stream) : launch_product_df<kF32, kMxB16>(a, stream);
  return format == kMxB32 ? launch_product_df<kBF16, kMxB32>(a, stream) : launch_product_df<kBF16, kMxB16>(a, stream);
}

}  // namespace fh
