// Layer norm: forward pass into dense and 4-bit outputs, backward pass from a dense or a 4-bit input.
#include <algorithm>

#include "fh_launch.cuh"
#include "fh_mx.cuh"
#include "fh_mx_launch.cuh"

namespace fh {
namespace {

constexpr int kNormThreads = 256, kNormWarps = kNormThreads / 32;

template <int DT>
struct NormVec {
  static constexpr int kE = DT == kF32 ? 4 : 8;  // elements of a 16-byte vector
};

// Which of a row's columns are element e of vector i of thread t of its team: E neighbours, so that they are one access of 16 bytes, or,
// where rows lie off the 16-byte grid (LINES), elements TEAM apart, so that a warp's accesses of one element each are neighbours.
template <int E, int TEAM, bool LINES>
__device__ __forceinline__ uint32_t column(uint32_t i, uint32_t t, int e) {
  return LINES ? (i * E + e) * TEAM + t : (i * TEAM + t) * E + e;
}
template <int DT>
__device__ __forceinline__ uint32_t load_elem(const uint8_t* row, uint32_t col) {
  return DT == kF32 ? reinterpret_cast<const uint32_t*>(row)[col] : reinterpret_cast<const uint16_t*>(row)[col];
}
// Vector i of a row as it lies in memory, zeros behind the last column.  VEC: rows are on the 16-byte grid.
template <int DT, int TEAM, bool VEC, bool LINES>
__device__ __forceinline__ uint4 load_vec(const uint8_t* row, uint32_t i, uint32_t t, uint32_t cols) {
  constexpr int E = NormVec<DT>::kE;
  const uint32_t col = column<E, TEAM, LINES>(i, t, 0);
  if (VEC && col + E <= cols) return *reinterpret_cast<const uint4*>(row + (uint64_t)col * (16 / E));
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint32_t c = column<E, TEAM, LINES>(i, t, e);
    if (c < cols) w[DT == kF32 ? e : e / 2] |= load_elem<DT>(row, c) << (DT == kF32 ? 0 : e % 2 * 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT, int TEAM, bool VEC, bool LINES>
__device__ __forceinline__ void store_vec(uint8_t* row, uint32_t i, uint32_t t, uint32_t cols, const uint4& v) {
  constexpr int E = NormVec<DT>::kE;
  const uint32_t col = column<E, TEAM, LINES>(i, t, 0);
  if (VEC && col + E <= cols) {
    *reinterpret_cast<uint4*>(row + (uint64_t)col * (16 / E)) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if (DT == kBF16 && !VEC && !LINES && col + E <= cols) {  // words, wherever the row begins
    uint16_t* p = reinterpret_cast<uint16_t*>(row) + col;
    uint32_t* q = reinterpret_cast<uint32_t*>((uintptr_t)p + 2u & ~(uintptr_t)3u);
    if ((uintptr_t)p & 2u) {
      p[0] = (uint16_t)w[0];
#pragma unroll
      for (int k = 0; k < 3; ++k) q[k] = __funnelshift_r(w[k], w[k + 1], 16);
      p[7] = (uint16_t)(w[3] >> 16);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) q[k] = w[k];
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint32_t c = column<E, TEAM, LINES>(i, t, e);
    if (c < cols) {
      if (DT == kF32)
        reinterpret_cast<uint32_t*>(row)[c] = w[e];
      else
        reinterpret_cast<uint16_t*>(row)[c] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
    }
  }
}
// The same into the thread's own bytes of shared memory, later: what a thread has asked for so it alone reads, so that no barrier
// stands between.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4u : 0u) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
// Where a thread's vectors of a row lie: 16 bytes each, and off the 16-byte grid in bf16 a fifth word.  An element of bf16 is too small for
// such a copy, so the words that hold the vector are copied, and the vector is shifted out of them: where rows begin in the middle of a word, the
// first word's other half is the end of the row before, which is why the first row's first vector and the last row's last ones are loaded
// when they are used (by_hand).  With LINES nothing is copied, and elements of bf16 are loaded when they are used.
template <int DT, int TEAM, int V, bool VEC, bool LINES>
struct RowRing {
  static constexpr bool kWords = DT == kBF16 && !VEC && !LINES, kNone = DT == kBF16 && !VEC && LINES;
  static constexpr uint32_t kFifth = V * kNormThreads * 16, kBytes = kNone ? 0 : kFifth + (kWords ? V * kNormThreads * 4 : 0);
  static __device__ __forceinline__ bool by_hand(uint32_t row, uint32_t rows, uint32_t col, uint32_t cols) {
    return kWords && ((row == 0u && col == 0u) || (row + 1u == rows && col + 9u >= cols));
  }
  // Vector i, one that begins ahead of the last column.
  static __device__ __forceinline__ void copy(uint32_t at, const uint8_t* p, uint32_t row, uint32_t rows, uint32_t i, uint32_t t, uint32_t cols) {
    constexpr int E = NormVec<DT>::kE;
    const uint32_t col = column<E, TEAM, LINES>(i, t, 0), to = at + (i * kNormThreads + threadIdx.x) * 16u;
    if (VEC) {
      copy16(to, p + (uint64_t)col * (16 / E), min((uint32_t)E, cols - col) * (16 / E));
    } else if (DT == kF32) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t c = column<E, TEAM, LINES>(i, t, e);
        copy4(to + 4 * e, p + (c < cols ? (uint64_t)c * 4u : 0u), c < cols);
      }
    } else if (kWords && !by_hand(row, rows, col, cols)) {
      const uint32_t shift = (uint32_t)((uintptr_t)p >> 1) & 1u;
      const uint8_t* q = p + ((int64_t)col - shift) * 2;
#pragma unroll
      for (uint32_t k = 0; k < 4u; ++k)
        if (col + 2u * k < cols + shift) copy4(to + 4u * k, q + 4u * k, true);
      if (shift && col + 8u < cols + shift) copy4(at + kFifth + (i * kNormThreads + threadIdx.x) * 4u, q + 16, true);
    }
  }
  static __device__ __forceinline__ uint4 get(uint32_t at, const uint8_t* p, uint32_t row, uint32_t rows, uint32_t i, uint32_t t, uint32_t cols);
};
__device__ __forceinline__ uint4 ld_shared16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t ld_shared4(uint32_t at) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}
template <int DT, int TEAM, int V, bool VEC, bool LINES>
__device__ __forceinline__ uint4 RowRing<DT, TEAM, V, VEC, LINES>::get(uint32_t at, const uint8_t* p, uint32_t row, uint32_t rows, uint32_t i,
                                                                       uint32_t t, uint32_t cols) {
  constexpr int E = NormVec<DT>::kE;
  if (kNone) return load_vec<DT, TEAM, VEC, LINES>(p, i, t, cols);
  const uint32_t to = at + (i * kNormThreads + threadIdx.x) * 16u;
  if (!kWords) return ld_shared16(to);
  const uint32_t col = column<E, TEAM, LINES>(i, t, 0);
  if (by_hand(row, rows, col, cols)) return load_vec<DT, TEAM, VEC, LINES>(p, i, t, cols);
  uint4 v = ld_shared16(to);
  if ((uintptr_t)p & 2u) {
    const uint32_t fifth = ld_shared4(at + kFifth + (i * kNormThreads + threadIdx.x) * 4u);
    v = make_uint4(__funnelshift_r(v.x, v.y, 16), __funnelshift_r(v.y, v.z, 16), __funnelshift_r(v.z, v.w, 16), __funnelshift_r(v.w, fifth, 16));
  }
  if (col + 8u > cols) {  // (nothing was copied behind the last column's word)
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (uint32_t k = 0; k < 4u; ++k) w[k] = col + 2u * k + 1u < cols ? w[k] : (col + 2u * k < cols ? w[k] & 0xFFFFu : 0u);
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return v;
}
template <int DT, int E>
__device__ __forceinline__ void unpack(const uint4& v, float (&f)[E]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = DT == kF32 ? bits_f(w[e]) : bits_f(e % 2 ? w[e / 2] & 0xFFFF0000u : w[e / 2] << 16);
}
template <int DT, int E>
__device__ __forceinline__ uint4 pack(const float (&f)[E]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT == kF32) {
      w[i] = __float_as_uint(f[i]);
    } else {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i % E], f[(2 * i + 1) % E]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// The same as pairs for the two-wide instructions.
template <int DT, int H>
__device__ __forceinline__ void unpack(const uint4& v, f32x2 (&f)[H]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int h = 0; h < H; ++h)
    f[h] = DT == kF32 ? pack2(bits_f(w[2 * h % 4]), bits_f(w[(2 * h + 1) % 4])) : pack2(bits_f(w[h % 4] << 16), bits_f(w[h % 4] & 0xFFFF0000u));
}
template <int DT, int H>
__device__ __forceinline__ uint4 pack(const f32x2 (&f)[H]) {
  uint32_t w[4];
#pragma unroll
  for (int h = 0; h < H; ++h) {
    float a, b;
    unpack2(f[h], a, b);
    if (DT == kF32) {
      w[2 * h % 4] = __float_as_uint(a);
      w[(2 * h + 1) % 4] = __float_as_uint(b);
    } else {
      w[h % 4] = f32x2_to_bf16x2(a, b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ f32x2 both(float v) { return pack2(v, v); }
__device__ __forceinline__ float halves(f32x2 v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}

// The weights of vector i in fp32; `none` where there are none.
template <int E, int TEAM, bool LINES>
__device__ __forceinline__ void load_weights(const uint8_t* p, int wdt, uint32_t i, uint32_t t, uint32_t cols, float none, float (&f)[E]) {
  const uint32_t col = column<E, TEAM, LINES>(i, t, 0);
  if (!LINES && p && (uintptr_t)p % 16 == 0 && col + E <= cols) {
    if (wdt == kF32) {
#pragma unroll
      for (int h = 0; h < E / 4; ++h) {
        const float4 v = reinterpret_cast<const float4*>(p)[col / 4u + h];
        f[4 * h] = v.x;
        f[4 * h + 1] = v.y;
        f[4 * h + 2] = v.z;
        f[4 * h + 3] = v.w;
      }
    } else {
#pragma unroll
      for (int h = 0; h < E / 4; ++h) {
        const uint2 v = reinterpret_cast<const uint2*>(p)[col / 4u + h];
        f[4 * h] = bits_f(v.x << 16);
        f[4 * h + 1] = bits_f(v.x & 0xFFFF0000u);
        f[4 * h + 2] = bits_f(v.y << 16);
        f[4 * h + 3] = bits_f(v.y & 0xFFFF0000u);
      }
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const uint32_t c = column<E, TEAM, LINES>(i, t, e);
    f[e] = none;
    if (p && c < cols) f[e] = wdt == kF32 ? reinterpret_cast<const float*>(p)[c] : bits_f((uint32_t) reinterpret_cast<const uint16_t*>(p)[c] << 16);
  }
}

// Barrier of the TEAM threads that share a row.
template <int TEAM>
__device__ __forceinline__ void team_barrier() {
  if (TEAM == kNormThreads)
    __syncthreads();
  else if (TEAM > 32)
    asm volatile("bar.sync %0, %1;" ::"r"(1u + threadIdx.x / TEAM), "n"(TEAM) : "memory");
}

// Sum over the TEAM threads that share a row, in a fixed order, the same in every thread.  `slot`: TEAM / 32 values that the team uses for
// nothing else until another of its barriers has passed.
template <int TEAM>
__device__ __forceinline__ float team_sum(float a, float* slot) {
#pragma unroll
  for (int d = 16; d; d /= 2) a += __shfl_xor_sync(0xFFFFFFFFu, a, d);
  if (TEAM == 32) return a;
  if (threadIdx.x % 32 == 0) slot[threadIdx.x % TEAM / 32] = a;
  team_barrier<TEAM>();
  a = 0.0f;
#pragma unroll
  for (int w = 0; w < TEAM / 32; w += 4) {
    const float4 v = *reinterpret_cast<const float4*>(slot + w);
    a += (v.x + v.y) + (v.z + v.w);
  }
  return a;
}
// NV sums at once (2, 4 or 8): in each of the first steps a lane keeps half of the values it has and hands over the others, so that NV sums
// take NV - 1 exchanges and the steps that are left.  `slot`: NV rows of TEAM / 32 values.
template <int TEAM, int NV>
__device__ __forceinline__ void team_sums(float (&v)[NV], float (*slot)[TEAM / 32]) {
  const uint32_t lane = threadIdx.x % 32;
  uint32_t which = 0;
  int d = 16;
#pragma unroll
  for (int n = NV / 2; n; n /= 2, d /= 2) {
    const bool upper = lane & d;
    which += upper ? n : 0;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float give = upper ? v[j] : v[j + n];
      v[j] = (upper ? v[j + n] : v[j]) + __shfl_xor_sync(0xFFFFFFFFu, give, d);
    }
  }
#pragma unroll
  for (; d; d /= 2) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], d);
  if (TEAM == 32) {
    const float mine = v[0];
#pragma unroll
    for (int j = 0; j < NV; ++j) v[j] = __shfl_sync(0xFFFFFFFFu, mine, j * (32 / NV));
    return;
  }
  if (lane % (32u / NV) == 0u) slot[which][threadIdx.x % TEAM / 32] = v[0];
  team_barrier<TEAM>();
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    v[j] = 0.0f;
#pragma unroll
    for (int w = 0; w < TEAM / 32; w += 4) {
      const float4 u = *reinterpret_cast<const float4*>(&slot[j][w]);
      v[j] += (u.x + u.y) + (u.z + u.w);
    }
  }
}

// sum / cols, rounded once, of a finite sum that is not subnormal; `inv` = rn(1 / cols).  q is off by at most 1.5 of its last places, so what it
// leaves of the sum, a multiple of that place, is below 2^17 of them for cols < 2^15 and comes out exactly; that times inv is the distance from q to
// the quotient within 2^-23 places, and a quotient by cols lies 2^-16 places or more from where rounding turns.  With the
// rounding of q alone a row of 15 times 10000 had the mean 10000.00098, its only spread, and y = 0.3.  (A division in its place:
// 100000 x 64 bf16 23.9 us, this 23.0; 16384 x 4096 and its container 84.5 and 83.8.)
__device__ __forceinline__ float mean_of(float sum, uint32_t cols, float inv) {
  const float q = sum * inv, rest = __fmaf_rn(-q, (float)cols, sum);
  return rest == rest ? __fmaf_rn(rest, inv, q) : q;  // (a sum that is infinite keeps its mean)
}

// ---- codes of a row of the output, E of its columns from `col` on in each lane (neighbouring lanes hold neighbouring columns)
// A lane's codes and, in the lane that has the first of four blocks, their scales.  Every lane of the warp takes part; rows behind the last
// and columns behind the last give zeros.
template <int E>
__device__ __forceinline__ uint32_t top_of(const float (&v)[E]) {
  uint32_t top = 0u;
#pragma unroll
  for (int e = 0; e < E; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
  return top;
}
// (`top`: the largest magnitude of v, as bits)
template <int F, int E>
__device__ __forceinline__ uint2 codes_of_f(const NormArgs& a, uint32_t row, uint32_t col, const float (&v)[E], uint32_t top, float unscale) {
  constexpr int kLanes = (F == kMxB32 ? 32 : 16) / E;  // lanes to a block
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  const MxScale s = mx_scale<F>(top, unscale);
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = e < E ? mx_quotient<F>(v[e % E], s) : 0.0f;
  uint32_t word = row < a.rows && col < a.cols ? s.byte : 0u;
  word |= __shfl_down_sync(0xFFFFFFFFu, word, kLanes) << 8;
  word |= __shfl_down_sync(0xFFFFFFFFu, word, 2 * kLanes) << 16;
  return make_uint2(s.bad ? 0u : mx_codes8(q), word);
}
template <int E>
__device__ __forceinline__ uint2 codes_of(const NormArgs& a, uint32_t format, uint32_t row, uint32_t col, const float (&v)[E], float unscale) {
  return format == kMxB32 ? codes_of_f<kMxB32, E>(a, row, col, v, top_of<E>(v), unscale) : codes_of_f<kMxB16, E>(a, row, col, v, top_of<E>(v), unscale);
}
// ... straight to the container, for rows that are worked on one at a time.  (col is a multiple of E, and kp of 64.)
template <int E>
__device__ __forceinline__ void store_codes(const NormArgs& a, const MxLayout& l, uint32_t row, uint32_t col, const float (&v)[E], float unscale) {
  const uint2 c = codes_of<E>(a, l.format, row, col, v, unscale);
  if (row < l.r8 && col < l.kp) {
    uint8_t* p = a.packed + l.code_at(row, col / 32u) + col % 32u / 2u;
    if (E == 8)
      *reinterpret_cast<uint32_t*>(p) = c.x;
    else
      *reinterpret_cast<uint16_t*>(p) = (uint16_t)c.x;
  }
  const uint32_t cols = l.format == kMxB32 ? 128u : 64u, atom = col / cols;
  if (col % cols == 0u && atom < l.atoms)
    *reinterpret_cast<uint32_t*>(a.packed + l.atom_at(row / 128u, atom) + MxLayout::scale_in_atom(row)) = c.y;
}
// ... or by way of shared memory, four rows of a vector of a warp at `at`, so that a lane writes 16 bytes and four lanes 64 in a row (with 4 bytes a
// lane 16384 x 4096 took 91 us, 29 more than y alone and longer than compressing y).
constexpr uint32_t kStageX = 512 + 64;
template <int F, int E>
__device__ __forceinline__ void stage_codes(const NormArgs& a, uint8_t* at, uint32_t row, uint32_t col, uint32_t k, const float (&v)[E], uint32_t top,
                                            float unscale) {
  constexpr uint32_t cols = F == kMxB32 ? 128u : 64u;
  const uint32_t lane = threadIdx.x % 32u;
  const uint2 c = codes_of_f<F, E>(a, row, col, v, top, unscale);
  if (E == 8)
    reinterpret_cast<uint32_t*>(at)[k * 32u + lane] = c.x;
  else
    reinterpret_cast<uint16_t*>(at)[k * 32u + lane] = (uint16_t)c.x;
  if (col % cols == 0u) reinterpret_cast<uint32_t*>(at + 512)[4u * k + lane * E / cols] = c.y;
}
// Rows row ... row + n - 1 of the vector that begins in column col0.
template <int F, int E>
__device__ __forceinline__ void flush_codes(const NormArgs& a, const MxLayout& l, const uint8_t* at, uint32_t row, uint32_t n, uint32_t col0) {
  const uint32_t lane = threadIdx.x % 32u, k = lane % 4u, c = lane / 4u, chunk = col0 / 32u + c;
  if (c < (uint32_t)E && k < n && row + k < l.r8 && chunk * 32u < l.kp)
    *reinterpret_cast<uint4*>(a.packed + l.code_at(row + k, chunk)) = *reinterpret_cast<const uint4*>(at + k * (16u * E) + c * 16u);
  constexpr uint32_t cols = F == kMxB32 ? 128u : 64u, words = 32u * E / cols;
  const uint32_t ks = lane / words, word = lane % words, atom = col0 / cols + word;
  if (ks < n && atom < l.atoms)
    *reinterpret_cast<uint32_t*>(a.packed + l.atom_at((row + ks) / 128u, atom) + MxLayout::scale_in_atom(row + ks)) =
        reinterpret_cast<const uint32_t*>(at + 512)[4u * ks + word];
}

// Forward.  y = (x - mean) * rstd * gamma + beta, mean and variance from the row as it is held in registers (the squares of the
// distances from the mean, not of the values), sums in fp32.  TEAM threads to a row, V vectors to a thread; a team takes rows in order, with
// the weights of its columns in registers and the next rows on their way into shared memory.  What bounds it is memory; arithmetic is two
// elements to an instruction for that (16384 x 4096 bf16: one element to an instruction 66 us, with the weights read again for every row 153).
constexpr int kAhead = 4;  // rows of a team in shared memory

__device__ __forceinline__ void write_header(const NormArgs& a, const MxLayout& l) {
  if (!a.packed || blockIdx.x != 0 || threadIdx.x >= 8) return;
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (threadIdx.x == 0) v = make_uint4(kMxMagic, 1u | l.format << 16, l.rows, l.cols);
  if (threadIdx.x == 1) v = make_uint4((uint32_t)a.exponent, 0u, (uint32_t)l.total, (uint32_t)(l.total >> 32));
  if (threadIdx.x == 2) v = make_uint4((uint32_t)a.tensor_id, (uint32_t)(a.tensor_id >> 32), 0u, 0u);
  reinterpret_cast<uint4*>(a.packed)[threadIdx.x] = v;
}

// A vector of y as it is in its type, so that its codes are those that compressing y gives; its largest magnitude, as bits.
template <int DT, int E>
__device__ __forceinline__ uint32_t as_stored(const NormArgs& a, uint32_t col, const uint4& out, float (&f)[E]) {
  unpack<DT, E>(out, f);
  if (DT == kBF16 && col + E <= a.cols) {  // two elements at a time
    const uint32_t m = __vmaxu2(__vmaxu2(out.x & 0x7FFF7FFFu, out.y & 0x7FFF7FFFu), __vmaxu2(out.z & 0x7FFF7FFFu, out.w & 0x7FFF7FFFu));
    return max(m << 16, m & 0xFFFF0000u);
  }
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (col + e >= a.cols) f[e] = 0.0f;
  return top_of<E>(f);
}

// P: no container, or 1 + its format.
template <int DT, int TEAM, int V, bool VEC, bool LINES, int P>
__global__ void __launch_bounds__(kNormThreads, 2) norm_forward_kernel(const NormArgs a) {
  constexpr int E = NormVec<DT>::kE, H = E / 2;
  using Row = RowRing<DT, TEAM, V, VEC, LINES>;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float slots[kNormThreads / TEAM][4][TEAM / 32];
  const uint32_t t = threadIdx.x % TEAM, in_cta = threadIdx.x / TEAM, team = blockIdx.x * (kNormThreads / TEAM) + in_cta,
                 teams = gridDim.x * (kNormThreads / TEAM);
  constexpr int F = P > 1 ? kMxB16 : kMxB32;
  const MxLayout l(a.rows, a.cols, F);
  const uint32_t rows = P ? (a.rows + 127u) / 128u * 128u : a.rows;  // (the padding of a container belongs to it)
  const uint32_t begin = (uint32_t)((uint64_t)rows * team / teams), end = (uint32_t)((uint64_t)rows * (team + 1u) / teams);
  const float inv = __frcp_rn((float)a.cols), unscale = F == kMxB32 ? 1.0f : pow2_f(-a.exponent);
  const uint32_t ring = smem_u32(smem);
  auto row_of = [&](uint32_t row) { return a.x + (uint64_t)row * a.ldx * (16 / E); };
  auto column_of = [&](int i, int e) { return column<E, TEAM, LINES>(i, t, e); };
  dep_trigger();
  dep_wait();
  if (P) write_header(a, l);
  auto ask = [&](uint32_t row, uint32_t slot) {
    if (row < end && (!P || row < a.rows)) {
      const uint8_t* p = row_of(row);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (column_of(i, 0) < a.cols) Row::copy(ring + slot * Row::kBytes, p, row, a.rows, i, t, a.cols);
    }
    copy_commit();
  };
#pragma unroll
  for (int k = 0; k < kAhead - 1; ++k) ask(begin + k, k);
  f32x2 gamma[V][H], beta[V][H];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float g[E], b[E];
    load_weights<E, TEAM, LINES>(a.gamma, a.wdtype, i, t, a.cols, 1.0f, g);
    load_weights<E, TEAM, LINES>(a.beta, a.wdtype, i, t, a.cols, 0.0f, b);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      gamma[i][h] = pack2(g[2 * h], g[2 * h + 1]);
      beta[i][h] = pack2(b[2 * h], b[2 * h + 1]);
    }
  }
  // codes of the team's rows, four of them at a time
  uint8_t* stage = smem + kAhead * Row::kBytes + threadIdx.x / 32u * kStageX;
  auto put_codes = [&](int i, uint32_t row, const float(&f)[E], uint32_t top) {
    stage_codes<F, E>(a, stage + i * (kNormWarps * kStageX), row, (i * TEAM + t) * E, (row - begin) % 4u, f, top, unscale);
  };
  auto flush = [&](uint32_t row) {
    const uint32_t k = (row - begin) % 4u;
    if (k != 3u && row + 1u != end) return;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < V; ++i)
      flush_codes<F, E>(a, l, stage + i * (kNormWarps * kStageX), row - k, k + 1u, (i * TEAM + (t - threadIdx.x % 32u)) * E);
    __syncwarp();
  };
  uint32_t turn = 0, slot = 0;
  for (uint32_t row = begin; row < end; ++row, turn ^= 2u, slot = slot + 1u == kAhead ? 0u : slot + 1u) {
    ask(row + kAhead - 1u, slot ? slot - 1u : kAhead - 1u);
    if (P && row >= a.rows) {
      const float zero[E] = {};
#pragma unroll
      for (int i = 0; i < V; ++i) put_codes(i, row, zero, 0u);
      flush(row);
      continue;
    }
    copy_wait<kAhead - 1>();
    f32x2 x[V][H], sum = both(0.0f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      uint4 raw = make_uint4(0u, 0u, 0u, 0u);
      if (column_of(i, 0) < a.cols) raw = Row::get(ring + slot * Row::kBytes, row_of(row), row, a.rows, i, t, a.cols);
      unpack<DT, H>(raw, x[i]);
#pragma unroll
      for (int h = 0; h < H; ++h) sum = add2(sum, x[i][h]);
    }
    const float mean = mean_of(team_sum<TEAM>(halves(sum), slots[in_cta][turn]), a.cols, inv);
    f32x2 sq = both(0.0f);
    float rest = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int h = 0; h < H; ++h) x[i][h] = add2(x[i][h], both(-mean));
      if (column_of(i, E - 1) < a.cols) {
#pragma unroll
        for (int h = 0; h < H; ++h) sq = fma2(x[i][h], x[i][h], sq);
      } else if (column_of(i, 0) < a.cols) {  // part of the vector is behind the last column
#pragma unroll
        for (int h = 0; h < H; ++h) {
          float p, q;
          unpack2(x[i][h], p, q);
          if (column_of(i, 2 * h) < a.cols) rest = __fmaf_rn(p, p, rest);
          if (column_of(i, 2 * h + 1) < a.cols) rest = __fmaf_rn(q, q, rest);
        }
      }
    }
    const float rstd = __frsqrt_rn(team_sum<TEAM>(halves(sq) + rest, slots[in_cta][turn + 1]) * inv + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    uint8_t* y = a.y ? a.y + (uint64_t)row * a.ldy * (16 / E) : nullptr;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
      for (int h = 0; h < H; ++h) x[i][h] = fma2(mul2(x[i][h], both(rstd)), gamma[i][h], beta[i][h]);
      const uint4 out = pack<DT, H>(x[i]);
      if (y && column_of(i, 0) < a.cols) store_vec<DT, TEAM, VEC, LINES>(y, i, t, a.cols, out);
      if (P) {
        float f[E];
        const uint32_t top = as_stored<DT, E>(a, (i * TEAM + t) * E, out, f);
        put_codes(i, row, f, top);
      }
    }
    if (P) flush(row);
  }
  copy_wait<0>();
}

// Rows of more vectors than that: each of the three sweeps reads the row again.
template <int DT, bool VEC>
__global__ void __launch_bounds__(kNormThreads) norm_forward_wide_kernel(const NormArgs a) {
  constexpr int E = NormVec<DT>::kE, TEAM = kNormThreads;
  __shared__ __align__(16) float slots[4][TEAM / 32];
  const uint32_t t = threadIdx.x;
  const MxLayout l(a.rows, a.cols, a.format);
  const uint32_t rows = a.packed ? (a.rows + 127u) / 128u * 128u : a.rows, sweeps = (a.cols + TEAM * E - 1u) / (TEAM * E);
  const float inv = __frcp_rn((float)a.cols), unscale = a.format == kMxB32 ? 1.0f : pow2_f(-a.exponent);
  dep_trigger();
  dep_wait();
  write_header(a, l);
  uint32_t turn = 0;
  for (uint32_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 2u) {
    if (row >= a.rows) {
      const float zero[E] = {};
      for (uint32_t i = 0; i < sweeps; ++i) store_codes<E>(a, l, row, (i * TEAM + t) * E, zero, unscale);
      continue;
    }
    const uint8_t* x = a.x + (uint64_t)row * a.ldx * (16 / E);
    float sum = 0.0f, sq = 0.0f;
    for (uint32_t i = 0; i < sweeps; ++i) {
      float f[E];
      unpack<DT, E>(load_vec<DT, TEAM, VEC, false>(x, i, t, a.cols), f);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += f[e];
    }
    const float mean = mean_of(team_sum<TEAM>(sum, slots[turn]), a.cols, inv);
    for (uint32_t i = 0; i < sweeps; ++i) {
      float f[E];
      unpack<DT, E>(load_vec<DT, TEAM, VEC, false>(x, i, t, a.cols), f);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float d = (i * TEAM + t) * E + e < a.cols ? f[e] - mean : 0.0f;
        sq = __fmaf_rn(d, d, sq);
      }
    }
    const float rstd = __frsqrt_rn(team_sum<TEAM>(sq, slots[turn + 1]) * inv + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[row] = mean;
      if (a.rstd) a.rstd[row] = rstd;
    }
    uint8_t* y = a.y ? a.y + (uint64_t)row * a.ldy * (16 / E) : nullptr;
    for (uint32_t i = 0; i < sweeps; ++i) {
      const uint32_t col = (i * TEAM + t) * E;
      float f[E], g[E], b[E];
      unpack<DT, E>(load_vec<DT, TEAM, VEC, false>(x, i, t, a.cols), f);
      load_weights<E, TEAM, false>(a.gamma, a.wdtype, i, t, a.cols, 1.0f, g);
      load_weights<E, TEAM, false>(a.beta, a.wdtype, i, t, a.cols, 0.0f, b);
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = __fmaf_rn((f[e] - mean) * rstd, g[e], b[e]);
      const uint4 out = pack<DT, E>(f);
      if (y && col < a.cols) store_vec<DT, TEAM, VEC, false>(y, i, t, a.cols, out);
      if (a.packed) {
        as_stored<DT, E>(a, col, out, f);
        store_codes<E>(a, l, row, col, f, unscale);
      }
    }
  }
}

// ---- backward -----------------------------------------------------------------------------------------
// With xhat = (x - mean) * rstd and g = dy * gamma:  dx = rstd * (g - mean(g) - xhat * mean(g * xhat)), dgamma = sum of dy * xhat over the
// rows, dbeta = sum of dy.  A team takes rows one after the other and keeps the sums of its columns, in registers, or in shared memory
// where there are too many; a CTA's teams are added up at the end, and the CTAs' sums, which lie in the caller's workspace, by a second kernel:
// all in a fixed order.

// x of vector i: dense as it lies there, or the word with its codes and the one with its scale.
template <int DT, int TEAM, bool VEC, bool LINES, int X>
__device__ __forceinline__ uint4 load_x(const NormArgs& a, const MxLayout& l, uint32_t row, uint32_t i, uint32_t t) {
  constexpr int E = NormVec<DT>::kE;
  if (X == 0) return load_vec<DT, TEAM, VEC, LINES>(a.x + (uint64_t)row * a.ldx * (16 / E), i, t, a.cols);
  const uint32_t col = column<E, TEAM, LINES>(i, t, 0);
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (col < a.cols) {
    v.x = *reinterpret_cast<const uint32_t*>(a.x + l.code_at(row, col / 32u) + col % 32u / 8u * 4u);
    v.y = *reinterpret_cast<const uint32_t*>(a.x + l.atom_at(row / 128u, col / (X > 1 ? 64u : 128u)) + MxLayout::scale_in_atom(row));
  }
  return v;
}
template <int DT, int X, int E>
__device__ __forceinline__ void unpack_x(const uint4& v, uint32_t col, float scale, float (&f)[E]) {
  if (X == 0) {
    unpack<DT, E>(v, f);
    return;
  }
  const float s = mx_factor<(X > 1 ? kMxB16 : kMxB32)>(v.y >> (col / (X > 1 ? 16u : 32u) % 4u * 8u) & 255u, scale);
  if constexpr (E == 8)
    mx_values8(v.x, f);
  else
    mx_values4(v.x >> (col % 8u * 4u), f);
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] *= s;
}
// The same as pairs; `shift`: where the vector's scale is in its word (fixed for a thread).
template <int X, int H>
__device__ __forceinline__ void unpack_x2(uint32_t codes, uint32_t word, uint32_t shift, uint32_t col, float scale, f32x2 (&f)[H]) {
  float v[2 * H];
  if constexpr (H == 4)
    mx_values8(codes, v);
  else
    mx_values4(codes >> (col % 8u * 4u), v);
  const f32x2 s = both(mx_factor<(X > 1 ? kMxB16 : kMxB32)>(word >> shift & 255u, scale));
#pragma unroll
  for (int h = 0; h < H; ++h) f[h] = mul2(pack2(v[2 * h], v[2 * h + 1]), s);
}
// The kernels' starts and ends in common: the header of a container (false: another one), and the CTA's sums to the workspace.
template <int X>
__device__ __forceinline__ bool backward_begin(const NormArgs& a, const MxLayout& l, float* scale) {
  int32_t exponent = 0;
  const bool ok = X == 0 || mx_header_ok(a.x, a.x_bytes, l, &exponent);
  if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) *a.status = ok ? 0ull : status_word(kErrCorrupt);
  *scale = ok && X == 1 + kMxB16 ? pow2_f(exponent) : 1.0f;
  return ok;
}
__device__ __forceinline__ void sums_to_work(const NormArgs& a, const float* acc, uint32_t wide) {
  float* out = a.work + (uint64_t)blockIdx.x * 2u * a.cols;
  for (uint32_t c = threadIdx.x; c < a.cols; c += kNormThreads) {
    out[c] = acc[c];
    out[a.cols + c] = acc[wide + c];
  }
}

template <int DT, int TEAM, int V, bool VEC, int X>
struct BackRing {
  static constexpr bool kLines = !VEC && X == 0;  // (bf16: 16384 x 4095 154 us, by words 171)
  using Row = RowRing<DT, TEAM, V, VEC, kLines>;
  static constexpr int kGroup = X ? 4 : (V < 4 ? 2 : 1);      // rows worked on together ...
  static constexpr int kRows = X || V < 4 ? 2 * kGroup : 3;   // ... and in shared memory
  static constexpr uint32_t kX = Row::kBytes, kSlot = X ? kX : 2 * kX;  // bytes of a slot: dy, and a dense x
  static constexpr uint32_t kWarpX = 512 + 64;                // of a vector of a warp, four rows: codes, scales
  static constexpr uint32_t kPacked = kRows * kSlot, kGroupX = V * kNormWarps * kWarpX;
  static constexpr size_t kBytes = kPacked + (X ? 2 * kGroupX : 0);
};

// Rows of up to V vectors a thread, a group of them at a time: their sums first, with one reduction and one barrier for all, then, from shared
// memory again, dx.  Rows come through a ring there, of which each thread asks for what it alone reads; a team's rows follow one another,
// so that a container's 128-byte pieces (eight rows) are found in L1.  Of a container a warp asks for 16 bytes a lane, four rows of eight
// chunks, and each lane reads its words of them.  Arithmetic is two elements to an instruction.
// (16384 x 4096 bf16 from 4 bits: each lane asking for its own words 105 us; element by element 138.)
template <int DT, int TEAM, int V, bool VEC, int X>
__global__ void __launch_bounds__(kNormThreads, V < 4 ? 2 : 1) norm_backward_kernel(const NormArgs a) {
  constexpr int E = NormVec<DT>::kE, H = E / 2;
  using R = BackRing<DT, TEAM, V, VEC, X>;
  using Row = typename R::Row;
  constexpr bool kLines = R::kLines;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float slots[kNormThreads / TEAM][2][2 * R::kGroup][TEAM / 32];
  const uint32_t t = threadIdx.x % TEAM, in_cta = threadIdx.x / TEAM, team = blockIdx.x * (kNormThreads / TEAM) + in_cta,
                 teams = gridDim.x * (kNormThreads / TEAM);
  const uint32_t begin = (uint32_t)((uint64_t)a.rows * team / teams), end = (uint32_t)((uint64_t)a.rows * (team + 1u) / teams);
  const MxLayout l(a.rows, a.cols, a.format);
  const float inv = __frcp_rn((float)a.cols);
  const uint32_t ring = smem_u32(smem);
  auto column_of = [&](int i, int e) { return column<E, TEAM, kLines>(i, t, e); };
  dep_trigger();
  dep_wait();
  float scale;
  if (!backward_begin<X>(a, l, &scale)) return;
  auto ask = [&](uint32_t row, uint32_t slot) {
    if (row < end) {
      const uint32_t at = ring + slot * R::kSlot;
      const uint8_t* dyr = a.dy + (uint64_t)row * a.ldy * (16 / E);
      const uint8_t* xr = a.x + (uint64_t)row * a.ldx * (16 / E);
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (column_of(i, 0) < a.cols) {
          Row::copy(at, dyr, row, a.rows, i, t, a.cols);
          if (X == 0) Row::copy(at + R::kX, xr, row, a.rows, i, t, a.cols);
        }
    }
    copy_commit();
  };
  constexpr int G = R::kGroup, kAsked = R::kRows - G;  // rows asked for ahead of a group
  // four rows of a container, vector i of the warp: lane 4 c + k asks for chunk c of row k
  constexpr uint32_t kAtomCols = X > 1 ? 64u : 128u, kWords = 32u * E / kAtomCols;  // columns to a word of scales, words to a warp's vector
  const uint32_t lane = threadIdx.x % 32u, warp_x = ring + R::kPacked + threadIdx.x / 32u * R::kWarpX;
  auto x_at = [&](int i, uint32_t half) { return warp_x + half * R::kGroupX + i * (kNormWarps * R::kWarpX); };
  auto ask_x = [&](uint32_t row, uint32_t half) {
    if (X) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const uint32_t col0 = (i * TEAM + (t - lane)) * E, k = lane % 4u, c = lane / 4u, chunk = col0 / 32u + c;
        if (c < (uint32_t)E && row + k < end && chunk * 32u < a.cols) copy16(x_at(i, half) + k * (16u * E) + c * 16u, a.x + l.code_at(row + k, chunk), 16u);
        const uint32_t ks = lane / kWords, word = lane % kWords, atom = col0 / kAtomCols + word;
        if (ks < 4u && row + ks < end && atom < l.atoms)
          copy4(x_at(i, half) + 512u + (4u * ks + word) * 4u, a.x + l.atom_at((row + ks) / 128u, atom) + MxLayout::scale_in_atom(row + ks), true);
      }
    }
  };
  ask_x(begin, 0u);
#pragma unroll
  for (int k = 0; k < kAsked; ++k) ask(begin + k, k);
  f32x2 dg[V][H], db[V][H], gamma[V][H];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    float g[E];
    load_weights<E, TEAM, kLines>(a.gamma, a.wdtype, i, t, a.cols, 1.0f, g);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      gamma[i][h] = pack2(g[2 * h], g[2 * h + 1]);
      dg[i][h] = db[i][h] = both(0.0f);
    }
  }
  float next_mean[G], next_rstd[G];
  auto ask_stats = [&](uint32_t row) {
#pragma unroll
    for (int k = 0; k < G; ++k)
      if (row + k < end) {
        next_mean[k] = a.mean[row + k];
        next_rstd[k] = a.rstd[row + k];
      }
  };
  ask_stats(begin);
  // dy, xhat and g = dy * gamma of vector i of a row (one that begins ahead of the last column; columns behind it have dy = 0 and add nothing)
  auto vec = [&](int i, uint32_t row, uint32_t slot, uint32_t k, uint32_t half, float mean, float rstd, f32x2(&dy)[H], f32x2(&xh)[H], f32x2(&g)[H]) {
    const uint32_t at = ring + slot * R::kSlot, col = column_of(i, 0);
    uint4 rx = make_uint4(0u, 0u, 0u, 0u);
    const uint4 ry = Row::get(at, a.dy + (uint64_t)row * a.ldy * (16 / E), row, a.rows, i, t, a.cols);
    if (X == 0) {
      rx = Row::get(at + R::kX, a.x + (uint64_t)row * a.ldx * (16 / E), row, a.rows, i, t, a.cols);
    } else {
      rx.x = ld_shared4(x_at(i, half) + k * (16u * E) + lane * E / 8u * 4u);
      rx.y = ld_shared4(x_at(i, half) + 512u + (4u * k + lane * E / kAtomCols) * 4u);
    }
    unpack<DT, H>(ry, dy);
    if (X == 0)
      unpack<DT, H>(rx, xh);
    else
      unpack_x2<X, H>(rx.x, rx.y, col / (X > 1 ? 16u : 32u) % 4u * 8u, col, scale, xh);
#pragma unroll
    for (int h = 0; h < H; ++h) {
      xh[h] = mul2(add2(xh[h], both(-mean)), both(rstd));
      g[h] = mul2(dy[h], gamma[i][h]);
    }
  };
  uint32_t turn = 0, slot = 0;
  for (uint32_t row = begin; row < end; row += G, turn ^= 1u) {
    uint32_t ahead = slot + kAsked;
    if (X) {
      __syncwarp();  // (nobody of the warp reads the group before any more)
      ask_x(row + G, turn ^ 1u);
    }
#pragma unroll
    for (int k = 0; k < G; ++k) {
      if (ahead >= (uint32_t)R::kRows) ahead -= R::kRows;
      ask(row + kAsked + k, ahead++);
    }
    float mean[G], rstd[G], s[2 * G];
#pragma unroll
    for (int k = 0; k < G; ++k) {
      mean[k] = next_mean[k];
      rstd[k] = next_rstd[k];
    }
    ask_stats(row + G);
    copy_wait<kAsked>();
    if (X) __syncwarp();  // (what the other lanes have asked for)
#pragma unroll
    for (int k = 0; k < G; ++k) {
      f32x2 s1 = both(0.0f), s2 = both(0.0f);
      if (row + k < end) {
        const uint32_t here = slot + k < (uint32_t)R::kRows ? slot + k : slot + k - R::kRows;
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (column_of(i, 0) < a.cols) {
            f32x2 dy[H], xh[H], g[H];
            vec(i, row + k, here, (uint32_t)k, turn, mean[k], rstd[k], dy, xh, g);
#pragma unroll
            for (int h = 0; h < H; ++h) {
              s1 = add2(s1, g[h]);
              s2 = fma2(g[h], xh[h], s2);
              dg[i][h] = fma2(dy[h], xh[h], dg[i][h]);
              db[i][h] = add2(db[i][h], dy[h]);
            }
          }
      }
      s[2 * k] = halves(s1);
      s[2 * k + 1] = halves(s2);
    }
    if (a.dx) {
      team_sums<TEAM, 2 * G>(s, slots[in_cta][turn]);
#pragma unroll
      for (int k = 0; k < G; ++k)
        if (row + k < end) {
          const uint32_t here = slot + k < (uint32_t)R::kRows ? slot + k : slot + k - R::kRows;
          const f32x2 m1 = both(-(s[2 * k] * inv)), m2 = both(-(s[2 * k + 1] * inv));
          uint8_t* dxr = a.dx + (uint64_t)(row + k) * a.ldx * (16 / E);
#pragma unroll
          for (int i = 0; i < V; ++i)
            if (column_of(i, 0) < a.cols) {
              f32x2 dy[H], xh[H], g[H];
              vec(i, row + k, here, (uint32_t)k, turn, mean[k], rstd[k], dy, xh, g);
#pragma unroll
              for (int h = 0; h < H; ++h) g[h] = mul2(fma2(xh[h], m2, add2(g[h], m1)), both(rstd[k]));
              store_vec<DT, TEAM, VEC, kLines>(dxr, i, t, a.cols, pack<DT, H>(g));
            }
        }
    }
    slot += G;
    if (slot >= (uint32_t)R::kRows) slot -= R::kRows;
  }
  copy_wait<0>();
  if (!a.work) return;
  float* acc = reinterpret_cast<float*>(smem);
  float* out = a.work + (uint64_t)blockIdx.x * 2u * a.cols;
  constexpr uint32_t wide = V * TEAM * E;
  for (uint32_t w = 0; w < (uint32_t)(kNormThreads / TEAM); ++w) {  // the CTA's teams one after the other
    if (TEAM < kNormThreads) __syncthreads();                       // (the first one: nobody reads its rows any more)
    if (in_cta == w) {
#pragma unroll
      for (int i = 0; i < V; ++i)
#pragma unroll
        for (int h = 0; h < H; ++h) {
          float p[2], q[2];
          unpack2(dg[i][h], p[0], p[1]);
          unpack2(db[i][h], q[0], q[1]);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t c = column_of(i, 2 * h + k);
            if (TEAM < kNormThreads) {
              acc[c] = w ? acc[c] + p[k] : p[k];
              acc[wide + c] = w ? acc[wide + c] + q[k] : q[k];
            } else if (c < a.cols) {
              out[c] = p[k];
              out[a.cols + c] = q[k];
            }
          }
        }
    }
  }
  if (TEAM < kNormThreads) {
    __syncthreads();
    sums_to_work(a, acc, wide);
  }
}

// Rows of more vectors than that: read twice, the sums of the columns in shared memory, where element e of vector i of thread t is at
// (i E + e) * TEAM + t, so that a warp's accesses are neighbours.  (4096 x 16000 bf16: half the threads, and sums in the order of the columns,
// 422 us.)
constexpr int kWideThreads = 512;
// Vectors of a row whose sums the kernel holds.
constexpr uint32_t wide_vecs(uint32_t vecs) { return (vecs + kWideThreads - 1u) / kWideThreads * kWideThreads; }
template <int DT, bool VEC, int X>
__global__ void __launch_bounds__(kWideThreads) norm_backward_wide_kernel(const NormArgs a) {
  constexpr int E = NormVec<DT>::kE, TEAM = kWideThreads;
  constexpr bool kLines = !VEC && X == 0;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ __align__(16) float slots[2][2][TEAM / 32];
  float* acc = reinterpret_cast<float*>(smem);
  const uint32_t t = threadIdx.x, sweeps = (a.cols + TEAM * E - 1u) / (TEAM * E), wide = sweeps * TEAM * E;
  const MxLayout l(a.rows, a.cols, a.format);
  const float inv = __frcp_rn((float)a.cols);
  dep_trigger();
  dep_wait();
  float scale;
  if (!backward_begin<X>(a, l, &scale)) return;
  for (uint32_t i = t; i < 2u * wide; i += TEAM) acc[i] = 0.0f;
  __syncthreads();
  uint32_t turn = 0;
  for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1u) {
    const uint8_t* dyr = a.dy + (uint64_t)row * a.ldy * (16 / E);
    const float mean = a.mean[row], rstd = a.rstd[row];
    auto vec = [&](uint32_t i, float(&xh)[E], float(&dy)[E], float(&g)[E]) {
      unpack<DT, E>(load_vec<DT, TEAM, VEC, kLines>(dyr, i, t, a.cols), dy);
      unpack_x<DT, X, E>(load_x<DT, TEAM, VEC, kLines, X>(a, l, row, i, t), column<E, TEAM, kLines>(i, t, 0), scale, xh);
      load_weights<E, TEAM, kLines>(a.gamma, a.wdtype, i, t, a.cols, 1.0f, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[e] = (xh[e] - mean) * rstd;
        g[e] = dy[e] * g[e];
      }
    };
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 2
    for (uint32_t i = 0; i < sweeps; ++i) {
      float xh[E], dy[E], g[E];
      vec(i, xh, dy, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s1 += g[e];
        s2 = __fmaf_rn(g[e], xh[e], s2);
        const uint32_t at = (i * E + e) * TEAM + t;
        acc[at] = __fmaf_rn(dy[e], xh[e], acc[at]);
        acc[wide + at] += dy[e];
      }
    }
    if (!a.dx) continue;
    float m[2] = {s1, s2};
    team_sums<TEAM, 2>(m, slots[turn]);
    const float m1 = m[0] * inv, m2 = m[1] * inv;
    uint8_t* dxr = a.dx + (uint64_t)row * a.ldx * (16 / E);
#pragma unroll 2
    for (uint32_t i = 0; i < sweeps; ++i) {
      float xh[E], dy[E], g[E];
      vec(i, xh, dy, g);
#pragma unroll
      for (int e = 0; e < E; ++e) g[e] = rstd * (g[e] - m1 - xh[e] * m2);
      if (column<E, TEAM, kLines>(i, t, 0) < a.cols) store_vec<DT, TEAM, VEC, kLines>(dxr, i, t, a.cols, pack<DT, E>(g));
    }
  }
  if (!a.work) return;
  float* out = a.work + (uint64_t)blockIdx.x * 2u * a.cols;
  for (uint32_t i = 0; i < sweeps; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const uint32_t c = column<E, TEAM, kLines>(i, t, e), at = (i * E + e) * TEAM + t;
      if (c < a.cols) {
        out[c] = acc[at];
        out[a.cols + c] = acc[wide + at];
      }
    }
}

// The CTAs' sums of 32 columns: eight warps take every eighth CTA, then the eight are added up.
__global__ void __launch_bounds__(kNormThreads) norm_columns_kernel(const NormArgs a) {
  __shared__ float part[kNormWarps][32];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, c = blockIdx.x * 32u + lane;  // of 2 * cols
  dep_trigger();
  dep_wait();
  int32_t exponent;
  if (a.x_bytes && !mx_header_ok(a.x, a.x_bytes, MxLayout(a.rows, a.cols, a.format), &exponent)) return;
  float s = 0.0f;
  if (c < 2u * a.cols) {
    const float* p = a.work + c;
    const uint64_t step = (uint64_t)kNormWarps * 2u * a.cols;
    uint32_t i = warp;
    p += (uint64_t)warp * 2u * a.cols;
    for (; i + 7u * kNormWarps < a.parts; i += 8u * kNormWarps) {  // (eight asked for at once: one at a time took 15 us for 296 CTAs)
      float v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k, p += step) v[k] = *p;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
    float v[7];
#pragma unroll
    for (int k = 0; k < 7; ++k, p += step) v[k] = i + k * kNormWarps < a.parts ? *p : 0.0f;
#pragma unroll
    for (int k = 0; k < 7; ++k) s += v[k];
  }
  part[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < 2u * a.cols) {
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < kNormWarps; ++w) v += part[w][lane];
    uint8_t* p = c < a.cols ? a.dgamma : a.dbeta;
    const uint32_t at = c < a.cols ? c : c - a.cols;
    if (p) {
      if (a.wdtype == kF32)
        reinterpret_cast<float*>(p)[at] = v;
      else
        reinterpret_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
    }
  }
}

template <int DT, int TEAM, int V, bool VEC, bool LINES, int P>
int launch_forward_t(const NormArgs& a, cudaStream_t stream) {
  const uint64_t rows = P ? ((uint64_t)a.rows + 127) / 128 * 128 : a.rows;
  const uint32_t grid = (uint32_t)std::min<uint64_t>((rows * TEAM + kNormThreads - 1) / kNormThreads, (uint64_t)sm_count() * 4);
  constexpr size_t smem = (size_t)kAhead * RowRing<DT, TEAM, V, VEC, LINES>::kBytes + (P ? (size_t)V * kNormWarps * kStageX : 0);
  return launch_plain<norm_forward_kernel<DT, TEAM, V, VEC, LINES, P>>(grid, kNormThreads, smem, 1, stream, a);
}
template <int DT, bool VEC, bool LINES, int P>
int launch_forward_dv(const NormArgs& a, cudaStream_t stream) {
  const uint32_t vecs = (a.cols + NormVec<DT>::kE - 1) / NormVec<DT>::kE;
  // a row's two reductions cost a thread some 30 instructions each, so few threads to a row, as long as registers hold their columns' weights
  if (vecs <= 32) return launch_forward_t<DT, 32, 1, VEC, LINES, P>(a, stream);
  if (vecs <= 64) return launch_forward_t<DT, 32, 2, VEC, LINES, P>(a, stream);
  if (vecs <= 128) return launch_forward_t<DT, 32, 4, VEC, LINES, P>(a, stream);
  if (vecs <= 256) return launch_forward_t<DT, 128, 2, VEC, LINES, P>(a, stream);
  if (vecs <= 512) return launch_forward_t<DT, P ? 256 : 128, P ? 2 : 4, VEC, LINES, P>(a, stream);
  if (vecs <= 1024) return launch_forward_t<DT, 256, 4, VEC, LINES, P>(a, stream);
  const uint64_t rows = a.packed ? ((uint64_t)a.rows + 127) / 128 * 128 : a.rows;
  return launch_plain<norm_forward_wide_kernel<DT, VEC>>((uint32_t)std::min<uint64_t>(rows, (uint64_t)sm_count() * 8), kNormThreads, 0, 1, stream, a);
}
template <int DT>
int launch_forward_d(const NormArgs& a, bool vec, cudaStream_t stream) {
  if (a.packed) {
    if (a.format == kMxB32) return vec ? launch_forward_dv<DT, true, false, 1>(a, stream) : launch_forward_dv<DT, false, false, 1>(a, stream);
    return vec ? launch_forward_dv<DT, true, false, 2>(a, stream) : launch_forward_dv<DT, false, false, 2>(a, stream);
  }
  if (vec) return launch_forward_dv<DT, true, false, 0>(a, stream);
  // Off the grid, bf16 comes by words for long rows and element by element for short ones: 16384 x 4095 105 and 256 us, x 1501 49 and 50, x 1001
  // 28.5 and 26.8.
  if constexpr (DT == kBF16) {
    if (a.cols > 1024) return launch_forward_dv<DT, false, false, 0>(a, stream);
  }
  return launch_forward_dv<DT, false, true, 0>(a, stream);
}

template <int DT, int TEAM, int V, bool VEC, int X>
int launch_backward_t(const NormArgs& a, cudaStream_t stream) {
  constexpr size_t ring = BackRing<DT, TEAM, V, VEC, X>::kBytes, sums = TEAM < kNormThreads ? (size_t)8 * V * TEAM * NormVec<DT>::kE : 0;
  return launch_plain<norm_backward_kernel<DT, TEAM, V, VEC, X>>(a.parts, kNormThreads, std::max(ring, sums), 1, stream, a);
}
template <int DT, bool VEC, int X>
int launch_backward_dx(const NormArgs& a, cudaStream_t stream) {
  const uint32_t vecs = (a.cols + NormVec<DT>::kE - 1) / NormVec<DT>::kE;
  if (vecs <= 32) return launch_backward_t<DT, 32, 1, VEC, X>(a, stream);
  if (vecs <= 128) return launch_backward_t<DT, 128, 1, VEC, X>(a, stream);
  if (vecs <= 256) return launch_backward_t<DT, 256, 1, VEC, X>(a, stream);
  if (vecs <= 512) return launch_backward_t<DT, 256, 2, VEC, X>(a, stream);
  if (vecs <= 1024) return launch_backward_t<DT, 256, 4, VEC, X>(a, stream);
  return launch_plain<norm_backward_wide_kernel<DT, VEC, X>>(a.parts, kWideThreads, (size_t)8 * wide_vecs(vecs) * NormVec<DT>::kE, 1, stream, a);
}
template <int DT>
int launch_backward_d(const NormArgs& a, bool vec, cudaStream_t stream) {
  if (a.x_bytes == 0) return vec ? launch_backward_dx<DT, true, 0>(a, stream) : launch_backward_dx<DT, false, 0>(a, stream);
  if (a.format == kMxB32) return vec ? launch_backward_dx<DT, true, 1>(a, stream) : launch_backward_dx<DT, false, 1>(a, stream);
  return vec ? launch_backward_dx<DT, true, 2>(a, stream) : launch_backward_dx<DT, false, 2>(a, stream);
}

bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

}  // namespace

uint32_t norm_parts(uint32_t rows, uint32_t cols, int dtype) {
  // rows that make a CTA worth its sums: four to a team of a warp, of half a CTA, of a CTA (see launch_backward_dx), and one where a row takes
  // 10 us (106 x 11902 fp32: 13 us, 37 with four)
  const uint32_t e = dtype == kF32 ? 4u : 8u, vecs = (cols + e - 1u) / e;
  const uint32_t each = vecs <= 32u ? 32u : (vecs <= 128u ? 8u : (vecs <= 1024u ? 4u : 1u));
  // Two CTAs to an SM; one where rows keep their sums in shared memory and those of two do not fit (4096 x 16000 bf16 215 us and 236,
  // 4096 x 13000, whose columns are rounded up to as many, 211 and 229).
  const uint32_t wide = vecs > 1024u ? wide_vecs(vecs) * e : 0u;
  const uint32_t n = rows / each + (rows % each ? 1u : 0u), most = wide <= 14336u ? 296u : 148u;
  return n < most ? n : most;
}

int launch_norm_forward(const NormArgs& a, int dtype, cudaStream_t stream) {
  if (sm_count() < 1) return FH_ERR_CUDA;
  const uint64_t es = dtype == kF32 ? 4 : 2;
  const bool vec = aligned16(a.x) && aligned16(a.y) && a.ldx * es % 16 == 0 && (!a.y || a.ldy * es % 16 == 0);
  return dtype == kF32 ? launch_forward_d<kF32>(a, vec, stream) : launch_forward_d<kBF16>(a, vec, stream);
}

int launch_norm_backward(const NormArgs& a0, int dtype, cudaStream_t stream) {
  NormArgs a = a0;
  const uint64_t es = dtype == kF32 ? 4 : 2;
  const bool vec = aligned16(a.x) && aligned16(a.dy) && aligned16(a.dx) && a.ldx * es % 16 == 0 && a.ldy * es % 16 == 0;
  a.parts = norm_parts(a.rows, a.cols, dtype);
  const int rc = dtype == kF32 ? launch_backward_d<kF32>(a, vec, stream) : launch_backward_d<kBF16>(a, vec, stream);
  if (rc != FH_OK || !a.work) return rc;
  return launch_plain<norm_columns_kernel>((2u * a.cols + 31u) / 32u, kNormThreads, 0, 1, stream, a);
}

}  // namespace fh
