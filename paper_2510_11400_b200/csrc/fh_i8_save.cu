// Dense matrices into 8-bit containers and back.
#include "fh_i8.cuh"
#include "fh_i8_launch.cuh"
#include "fh_launch.cuh"
#include "fh_tcgen05.cuh"

namespace fh {
namespace {

constexpr int kI8Threads = 256;

template <int DT>
constexpr uint32_t kEs = DT == kF32 ? 4u : 2u;

// ---- by rows ---------------------------------------------------------------------------------------
// A CTA takes R rows.  Lanes of a warp lie R rows by 32 / R chunks of 16 columns: R lanes that write the codes of the same chunk write R x 16 bytes
// side by side, and lanes of the same row read 32 / R chunks side by side.  A lane's I chunks stay in registers from the
// row's maximum to its codes; I = 0: the row is too long for that and is read again, from L2.
template <int DT, int R, int I, bool VEC>
__global__ void __launch_bounds__(512, 2) i8_rows_kernel(const I8SaveArgs g) {
  __shared__ uint32_t tops[16][R];
  constexpr uint32_t kLanes = 32 / R;
  const I8Layout l(g.rows, g.cols);
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = blockDim.x / 32;
  const uint32_t r = lane % R, row = blockIdx.x * R + r, chunks = l.chunks(), first = warp * kLanes + lane / R, step = warps * kLanes;
  dep_trigger();
  dep_wait();
  if (blockIdx.x == 0 && tid < 32) i8_write_header(g.dst, l, tid);
  using Loose = LooseRows<DT, R>;
  __shared__ __align__(16) uint8_t stages[VEC ? 16 : 16 * Loose::kBytes];
  const uint8_t* src = g.src + (uint64_t)(VEC ? row : blockIdx.x * R) * g.ld * kEs<DT>;
  const bool there = row < g.rows;
  const uint32_t rows = blockIdx.x * R < g.rows ? min((uint32_t)R, g.rows - blockIdx.x * R) : 0u;
  auto fetch = [&](Raw16<DT>& x, uint32_t j) {
    const uint32_t c = j * 16u;
    if (VEC)
      x.template load<true>(src + (uint64_t)c * kEs<DT>, there && c < g.cols ? (int)min(16u, g.cols - c) : 0);
    else
      Loose::load(x, stages + warp * Loose::kBytes, src, g.ld, rows, (j - lane / R) * 16u, g.cols, lane);
  };
  constexpr int N = I ? I : 1;
  Raw16<DT> x[N];
  uint32_t top = 0;
  if (I) {
#pragma unroll
    for (int i = 0; i < N; ++i) fetch(x[i], first + i * step);
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, x[i].top());
  } else {
#pragma unroll 2
    for (uint32_t j = first; j < chunks + lane / R; j += step) {  // (all lanes of a warp as often)
      fetch(x[0], j);
      top = max(top, x[0].top());
    }
  }
#pragma unroll
  for (int s = R; s < 32; s *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
  if (lane < R) tops[warp][r] = top;
  __syncthreads();
  for (uint32_t w = 0; w < warps; ++w) top = max(top, tops[w][r]);
  const I8Coder<DT> coder(top);
  uint8_t* dst = g.dst + l.code_at(row, 0);
  const uint64_t pitch = 16ull * l.block_rows(row / 128u);
  auto put = [&](const Raw16<DT>& v, uint32_t j) {
    float f[16];
    v.values(f);
    *reinterpret_cast<uint4*>(dst + j * pitch) = i8_codes16(f, coder);
  };
  if (I) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (first + i * step < chunks) put(x[i], first + i * step);
  } else {
#pragma unroll 2
    for (uint32_t j = first; j < chunks + lane / R; j += step) {
      fetch(x[0], j);
      if (j < chunks) put(x[0], j);
    }
  }
  if (warp == 0 && lane < R) *reinterpret_cast<uint32_t*>(g.dst + l.magnitude_at(row)) = i8_magnitude_bits(top);
}

template <int DT, int R, int I, bool VEC>
int rows_launch(const I8SaveArgs& a, uint32_t warps, cudaStream_t stream) {
  const uint64_t grid = (I8Layout(a.rows, a.cols).r8 + R - 1ull) / R;
  if (grid > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
  return launch_plain<i8_rows_kernel<DT, R, I, VEC>>((uint32_t)grid, (int)warps * 32, 0, 1, stream, a);
}
template <int DT, int R, bool VEC>
int rows_by_length(const I8SaveArgs& a, bool many, cudaStream_t stream) {
  constexpr uint32_t kLanes = 32 / R, kMost = DT == kF32 ? 2 : 4;
  const uint32_t need = (I8Layout(a.rows, a.cols).chunks() + kLanes - 1u) / kLanes;  // steps of a warp in all
  // Four warps to a CTA, or as few as hold the row, where there are many rows: CTAs that load run beside CTAs that write (8192 x 4096 bf16 in two rows to a
  // CTA: 16 warps 26 us, 8 18.5, 4 17.4); as many warps as the row has work for where there are few.
  const uint32_t most = many ? 4u : 16u;
  if (need <= most) return rows_launch<DT, R, 1, VEC>(a, need, stream);
  if (kMost == 4 && need <= 2u * most) return rows_launch<DT, R, 2, VEC>(a, (need + 1u) / 2u, stream);
  if (R == 2 || need <= 16u * kMost) return rows_launch<DT, R, kMost, VEC>(a, (need + kMost - 1u) / kMost, stream);
  return rows_launch<DT, 1, 0, VEC>(a, 16u, stream);  // (R is 1)
}
template <int DT, bool VEC>
int rows_by_group(const I8SaveArgs& a, cudaStream_t stream) {
  // Two rows to a CTA write whole sectors of codes (one row 16384 x 512 17.8 us, two 9.3, four 6.8; 8192 x 4096 20.8, 17.4 and 18.5); one where there are not
  // enough rows for every SM, or where two do not fit the registers of 16 warps.  Four rows have a chunk to a lane.
  const uint32_t chunks = I8Layout(a.rows, a.cols).chunks(), most = DT == kF32 ? 32u : 64u;
  const bool many = a.rows / 2u >= (uint32_t)std::max(1, sm_count());
  if (!many || (chunks + 15u) / 16u > most) return rows_by_length<DT, 1, VEC>(a, many, stream);
  if (chunks > 32u) return rows_by_length<DT, 2, VEC>(a, true, stream);
  return rows_launch<DT, 4, 1, VEC>(a, (chunks + 7u) / 8u, stream);
}

// ---- by columns ------------------------------------------------------------------------------------
// The container of the transpose: its rows are the matrix's columns, its chunks 16 of the matrix's rows.  A lane has C neighbouring columns and 16 rows at
// a time, whose codes are C times 16 bytes side by side in the container, 32 C columns to a warp: both sides are in whole sectors without a detour through
// shared memory.  The scales need whole columns first.
//  Matrices of few rows: one kernel, a cluster's CTAs share the rows of a group of columns, put their maxima together and read their rows again.
//  Others: the maxima by a kernel of their own, bands of rows side by side, which leaves them in the container (a maximum does not depend on the order), then
//  the codes.  (In clusters 8192 x 4096 bf16 took 40 us, 34 in two passes; 65536 x 256, with eight CTAs to a group of columns, 122 and 24.)
constexpr int kColWarps = 8;

template <int DT, int C, bool VEC>
struct ColChunk {
  static constexpr int kWords = C * (int)kEs<DT> / 4 ? C * (int)kEs<DT> / 4 : 1;
  static_assert(!VEC || C * kEs<DT> == 4u, "a word to a row");
  uint32_t w[16][kWords];
  // Rows 16 j ... of the columns from `col` on (n of them there), zeros elsewhere.
  __device__ __forceinline__ void load(const I8SaveArgs& g, uint32_t j, uint32_t col, int n) {
    const uint8_t* p = g.src + ((uint64_t)j * 16u * g.ld + col) * kEs<DT>;
    const uint64_t step = g.ld * kEs<DT>;
#pragma unroll
    for (int i = 0; i < 16; ++i, p += step) {
      const bool there = (uint64_t)j * 16u + i < g.rows;
#pragma unroll
      for (int x = 0; x < kWords; ++x) w[i][x] = 0u;
      if (VEC) {
        if (there && n == C) {
          w[i][0] = *reinterpret_cast<const uint32_t*>(p);  // (two columns of bf16)
          continue;
        }
      }
      if (there) {
#pragma unroll
        for (int x = 0; x < C; ++x)
          if (x < n) {
            if (DT == kF32)
              w[i][x] = reinterpret_cast<const uint32_t*>(p)[x];
            else
              w[i][x / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[x] << (x % 2 * 16);
          }
      }
    }
  }
  __device__ __forceinline__ float at(int row, int col) const {
    if (DT == kF32) return __uint_as_float(w[row][col]);
    return __uint_as_float(col % 2 ? w[row][col / 2] & 0xFFFF0000u : w[row][col / 2] << 16);
  }
};

template <int DT, int C, bool VEC>
__global__ void __launch_bounds__(kColWarps * 32) i8_cols_kernel(const I8SaveArgs g) {
  constexpr uint32_t kCols = 32 * C;
  __shared__ uint32_t tops[kColWarps][kCols];
  __shared__ uint32_t mine[kCols];
  const I8Layout l(g.cols, g.rows);
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t rank = g.parts > 1u ? blockIdx.x % g.parts : 0u, c0 = blockIdx.x / g.parts * kCols, col = c0 + lane * C;
  const uint32_t chunks = l.chunks(), first = (uint32_t)((uint64_t)chunks * rank / g.parts) + warp, last = (uint32_t)((uint64_t)chunks * (rank + 1u) / g.parts);
  const int n = col < g.cols ? (int)min((uint32_t)C, g.cols - col) : 0;
  dep_trigger();
  dep_wait();
  if (blockIdx.x == 0 && tid < 32) i8_write_header(g.dst, l, tid);
  using Chunk = ColChunk<DT, C, VEC>;
  Chunk x;
  uint32_t top[Chunk::kWords] = {};  // (in bf16 two columns' maxima side by side)
  for (uint32_t j = first; j < last; j += kColWarps) {
    x.load(g, j, col, n);
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int w = 0; w < Chunk::kWords; ++w)
        top[w] = DT == kF32 ? max(top[w], x.w[i][w] & 0x7FFFFFFFu) : __vmaxu2(top[w], x.w[i][w] & 0x7FFF7FFFu);
  }
#pragma unroll
  for (int c = 0; c < C; ++c) tops[warp][lane * C + c] = DT == kF32 ? top[c] : c % 2 ? top[c / 2] & 0x7FFF0000u : top[c / 2] << 16;
  __syncthreads();
  if (tid < kCols) {
    uint32_t t = 0;
#pragma unroll
    for (int w = 0; w < kColWarps; ++w) t = max(t, tops[w][tid]);
    mine[tid] = t;
  }
  if (g.parts > 1u) {
    cluster_sync();
    if (tid < kCols) {
      uint32_t t = 0;
      for (uint32_t p = 0; p < g.parts; ++p) t = max(t, ld_cluster_u32(mine + tid, p));
      tops[0][tid] = t;
    }
    cluster_sync();  // (before any CTA ends: others read its maxima)
  } else if (tid < kCols) {
    tops[0][tid] = mine[tid];
  }
  __syncthreads();
  if (rank == 0u && tid < kCols && c0 + tid < l.r8) *reinterpret_cast<uint32_t*>(g.dst + l.magnitude_at(c0 + tid)) = i8_magnitude_bits(tops[0][tid]);
  if (col >= l.r8) return;
  const uint64_t pitch = 16ull * l.block_rows(col / 128u);
  uint8_t* dst = g.dst + l.code_at(col, 0);
  I8Coder<DT> coder[C] = {I8Coder<DT>(tops[0][lane * C])};
#pragma unroll
  for (int c = 1; c < C; ++c) coder[c] = I8Coder<DT>(tops[0][lane * C + c]);
  for (uint32_t j = first; j < last; j += kColWarps) {
    x.load(g, j, col, n);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      float f[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = x.at(i, c);
      *reinterpret_cast<uint4*>(dst + j * pitch + c * 16u) = i8_codes16(f, coder[c]);
    }
  }
}

// The container's header, and zeros where the maxima are gathered.
__global__ void __launch_bounds__(kI8Threads) i8_cols_start_kernel(const I8SaveArgs g) {
  const I8Layout l(g.cols, g.rows);
  dep_trigger();
  dep_wait();
  if (blockIdx.x == 0 && threadIdx.x < 32) i8_write_header(g.dst, l, threadIdx.x);
  uint32_t* top = reinterpret_cast<uint32_t*>(g.dst + l.magnitude_at(0));
  for (uint64_t i = (uint64_t)blockIdx.x * kI8Threads + threadIdx.x; i < l.r8; i += (uint64_t)gridDim.x * kI8Threads) top[i] = 0u;
}

// A CTA takes 256 columns of a band of rows: a lane eight columns (VEC: side by side, in 16-byte vectors), a warp every eighth row.
constexpr uint32_t kBand = 64;
template <int DT, bool VEC>
__global__ void __launch_bounds__(kI8Threads) i8_cols_max_kernel(const I8SaveArgs g) {
  __shared__ uint32_t tops[kI8Threads / 32][256];
  const I8Layout l(g.cols, g.rows);
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, groups = (g.cols + 255u) / 256u, c0 = blockIdx.x % groups * 256u;
  const uint32_t r0 = blockIdx.x / groups * kBand, end = min(g.rows, r0 + kBand);
  uint32_t top[8] = {};
  dep_trigger();
  dep_wait();
  const uint8_t* p = g.src + ((uint64_t)r0 * g.ld + c0) * kEs<DT>;
  if (VEC) {
    const uint32_t n = c0 + lane * 8u < g.cols ? min(8u, g.cols - c0 - lane * 8u) : 0u;
    constexpr int kWords = DT == kF32 ? 8 : 4;
    uint32_t m[kWords] = {};
#pragma unroll 4
    for (uint32_t r = r0 + warp; r < end; r += kI8Threads / 32) {
      const uint8_t* q = p + ((uint64_t)(r - r0) * g.ld + lane * 8u) * kEs<DT>;
      uint32_t w[kWords] = {};
      if (n == 8u) {
#pragma unroll
        for (int x = 0; x < kWords; x += 4) {
          const uint4 v = reinterpret_cast<const uint4*>(q)[x / 4];
          w[x] = v.x;
          w[x + 1] = v.y;
          w[x + 2] = v.z;
          w[x + 3] = v.w;
        }
      } else {
#pragma unroll
        for (uint32_t x = 0; x < 8u; ++x)
          if (x < n) {
            if (DT == kF32)
              w[x] = reinterpret_cast<const uint32_t*>(q)[x];
            else
              w[x / 2u] |= (uint32_t) reinterpret_cast<const uint16_t*>(q)[x] << (x % 2u * 16u);
          }
      }
#pragma unroll
      for (int x = 0; x < kWords; ++x) m[x] = DT == kF32 ? max(m[x], w[x] & 0x7FFFFFFFu) : __vmaxu2(m[x], w[x] & 0x7FFF7FFFu);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) top[x] = DT == kF32 ? m[x % kWords] : x % 2 ? m[x / 2 % kWords] & 0x7FFF0000u : m[x / 2 % kWords] << 16;
#pragma unroll
    for (int x = 0; x < 8; ++x) tops[warp][lane * 8 + x] = top[x];
  } else {
#pragma unroll 2
    for (uint32_t r = r0 + warp; r < end; r += kI8Threads / 32) {
      const uint8_t* q = p + (uint64_t)(r - r0) * g.ld * kEs<DT>;
#pragma unroll
      for (uint32_t x = 0; x < 8u; ++x) {
        const uint32_t c = x * 32u + lane;
        if (c0 + c < g.cols)
          top[x] = max(top[x], DT == kF32 ? reinterpret_cast<const uint32_t*>(q)[c] & 0x7FFFFFFFu : (uint32_t)(reinterpret_cast<const uint16_t*>(q)[c] & 0x7FFFu) << 16);
      }
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) tops[warp][x * 32 + lane] = top[x];
  }
  __syncthreads();
  uint32_t t = 0;
#pragma unroll
  for (int w = 0; w < kI8Threads / 32; ++w) t = max(t, tops[w][threadIdx.x]);
  if (c0 + threadIdx.x < g.cols && t) atomicMax(reinterpret_cast<uint32_t*>(g.dst + l.magnitude_at(c0 + threadIdx.x)), i8_magnitude_bits(t));
}

// A warp takes a chunk of 32 C columns.  (Several, each asked for while the one before it is worked on: 8192 x 4096 bf16 34 -> 35 us with two, 47 with four.  Panels
// of columns that stay in L2 from one pass to the other, 16384 x 8192 with 48 MB to a panel: 121 -> 159.)
template <int DT, int C, bool VEC>
__global__ void __launch_bounds__(kI8Threads) i8_cols_codes_kernel(const I8SaveArgs g) {
  const I8Layout l(g.cols, g.rows);
  const uint32_t lane = threadIdx.x % 32, groups = (l.r8 + 32u * C - 1u) / (32u * C);
  const uint32_t col = blockIdx.x % groups * 32u * C + lane * C, j = blockIdx.x / groups * (kI8Threads / 32) + threadIdx.x / 32;
  const int n = col < g.cols ? (int)min((uint32_t)C, g.cols - col) : 0;
  dep_trigger();
  dep_wait();
  if (j >= l.chunks() || col >= l.r8) return;
  ColChunk<DT, C, VEC> x;
  x.load(g, j, col, n);
  uint8_t* dst = g.dst + l.code_at(col, j);
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (col + c >= l.r8) break;
    const I8Coder<DT> coder(*reinterpret_cast<const uint32_t*>(g.dst + l.magnitude_at(col + c)));
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = x.at(i, c);
    *reinterpret_cast<uint4*>(dst + c * 16u) = i8_codes16(f, coder);
  }
}

template <int DT, int C, bool VEC>
int cols_launch(const I8SaveArgs& a0, cudaStream_t stream) {
  I8SaveArgs a = a0;
  const I8Layout l(a.cols, a.rows);
  const uint32_t chunks = l.chunks();
  const uint64_t groups = ((uint64_t)a.cols + 32u * C - 1u) / (32u * C);
  a.parts = 1u;
  while (a.parts < 8u && chunks >= 2u * kColWarps * a.parts) a.parts *= 2u;
  // (the cluster kernel where a CTA has few rows: 1024 x 4096 bf16 8 us; or not many and the device several CTAs an SM: 4096 x 16384 59 us, in two passes 65)
  if (a.rows <= 1024u || (a.rows <= 4096u && groups * a.parts >= 8ull * std::max(1, sm_count()))) {
    if (groups * a.parts > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
    return launch_plain<i8_cols_kernel<DT, C, VEC>>((uint32_t)(groups * a.parts), kColWarps * 32, 0, (int)a.parts, stream, a);
  }
  const uint64_t max_ctas = ((uint64_t)a.cols + 255u) / 256u * (((uint64_t)a.rows + kBand - 1u) / kBand);
  const uint64_t code_ctas = (l.r8 + 32ull * C - 1u) / (32u * C) * ((chunks + kI8Threads / 32 - 1ull) / (kI8Threads / 32));
  if (max_ctas > 0x7FFFFFFFull || code_ctas > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
  int rc = launch_plain<i8_cols_start_kernel>((uint32_t)std::min<uint64_t>((l.r8 + kI8Threads - 1ull) / kI8Threads, (uint64_t)std::max(1, sm_count())), kI8Threads, 0, 1, stream, a);
  if (rc != FH_OK) return rc;
  if (((uintptr_t)a.src | a.ld * kEs<DT>) % 16u == 0u)
    rc = launch_plain<i8_cols_max_kernel<DT, true>>((uint32_t)max_ctas, kI8Threads, 0, 1, stream, a);
  else
    rc = launch_plain<i8_cols_max_kernel<DT, false>>((uint32_t)max_ctas, kI8Threads, 0, 1, stream, a);
  if (rc != FH_OK) return rc;
  return launch_plain<i8_cols_codes_kernel<DT, C, VEC>>((uint32_t)code_ctas, kI8Threads, 0, 1, stream, a);
}

// ---- and back --------------------------------------------------------------------------------------
// A warp's lanes lie 8 rows by 4 chunks, as in the kernel by rows.  (Four chunks to a lane, asked for at once: the same on large matrices, where two
// thirds of the traffic are writes, and 1 x 8192 2.7 us instead of 1.8.)
template <int DT, bool VEC>
__global__ void __launch_bounds__(kI8Threads) i8_restore_kernel(const I8SaveArgs g) {
  using Loose = LooseRows<DT, 8>;
  __shared__ __align__(16) uint8_t stages[VEC ? 16 : kI8Threads / 32 * Loose::kBytes];
  const I8Layout l(g.rows, g.cols);
  const uint32_t tid = threadIdx.x, lane = tid % 32;
  dep_trigger();
  dep_wait();
  const bool ok = i8_header_ok(g.src, g.src_bytes, l);
  if (blockIdx.x == 0 && tid == 0 && g.status) *g.status = ok ? 0ull : status_word(kErrCorrupt);
  if (!ok) return;
  const uint32_t quads = (l.chunks() + 3u) / 4u;
  const uint64_t items = (uint64_t)(l.r8 / 8u) * quads, step = (uint64_t)gridDim.x * (kI8Threads / 32);
  for (uint64_t it = (uint64_t)blockIdx.x * (kI8Threads / 32) + tid / 32; it < items; it += step) {
    const uint32_t r0 = (uint32_t)(it / quads) * 8u, row = r0 + lane % 8u, j0 = (uint32_t)(it % quads) * 4u, j = j0 + lane / 8u, c = j * 16u;
    const uint4 q = j < l.chunks() ? *reinterpret_cast<const uint4*>(g.src + l.code_at(row, j)) : make_uint4(0u, 0u, 0u, 0u);
    const float s = i8_scale(*reinterpret_cast<const float*>(g.src + l.magnitude_at(row)));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    float f[16];
#pragma unroll
    for (int i = 0; i < 16; ++i)  // (127 scales of a row that has fp32's largest number may be beyond it)
      f[i] = max_nan(min_nan((float)((int32_t)(w[i / 4] << (24 - i % 4 * 8)) >> 24) * s, 3.4028235e38f), -3.4028235e38f);
    Raw16<DT> v;
    v.take(f);
    if (VEC)
      v.template store<true>(g.dst + ((uint64_t)row * g.ld + c) * kEs<DT>, row < g.rows && c < g.cols ? (int)min(16u, g.cols - c) : 0);
    else
      Loose::store(v, stages + tid / 32 * Loose::kBytes, g.dst + (uint64_t)r0 * g.ld * kEs<DT>, g.ld, g.rows > r0 ? min(8u, g.rows - r0) : 0u, j0 * 16u, g.cols, lane);
  }
}

template <int DT>
bool on_grid(const void* p, uint64_t ld) { return ((uintptr_t)p | ld * kEs<DT>) % 16u == 0u; }

template <int DT>
int restore_launch(const I8SaveArgs& a, cudaStream_t stream) {
  const I8Layout l(a.rows, a.cols);
  const uint64_t items = (uint64_t)(l.r8 / 8u) * ((l.chunks() + 3u) / 4u), ctas = (items + kI8Threads / 32 - 1) / (kI8Threads / 32);
  const uint32_t grid = (uint32_t)std::min<uint64_t>(ctas, (uint64_t)std::max(1, sm_count()) * 32u);
  if (on_grid<DT>(a.dst, a.ld)) return launch_plain<i8_restore_kernel<DT, true>>(grid, kI8Threads, 0, 1, stream, a);
  return launch_plain<i8_restore_kernel<DT, false>>(grid, kI8Threads, 0, 1, stream, a);
}

}  // namespace

int launch_i8_rows(const I8SaveArgs& a, int dtype, cudaStream_t stream) {
  if (dtype == kF32) return on_grid<kF32>(a.src, a.ld) ? rows_by_group<kF32, true>(a, stream) : rows_by_group<kF32, false>(a, stream);
  return on_grid<kBF16>(a.src, a.ld) ? rows_by_group<kBF16, true>(a, stream) : rows_by_group<kBF16, false>(a, stream);
}

int launch_i8_cols(const I8SaveArgs& a, int dtype, cudaStream_t stream) {
  if (dtype == kF32) return cols_launch<kF32, 1, false>(a, stream);
  const bool words = ((uintptr_t)a.src | a.ld * 2u) % 4u == 0u;
  return words ? cols_launch<kBF16, 2, true>(a, stream) : cols_launch<kBF16, 1, false>(a, stream);
}

int launch_i8_decompress(const I8SaveArgs& a, int dtype, cudaStream_t stream) {
  return dtype == kF32 ? restore_launch<kF32>(a, stream) : restore_launch<kBF16>(a, stream);
}

}  // namespace fh
