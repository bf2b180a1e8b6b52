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

// A vector of a row as it lies in memory, zeros behind the last column.  VEC: on a 16-byte boundary.
template <int DT, bool VEC>
__device__ __forceinline__ uint4 load_vec(const uint8_t* row, uint32_t col, uint32_t cols) {
  constexpr int E = NormVec<DT>::kE;
  if (VEC && col + E <= cols) return *reinterpret_cast<const uint4*>(row + (uint64_t)col * (16 / E));
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (col + e < cols) {
      if (DT == kF32)
        w[e] = reinterpret_cast<const uint32_t*>(row)[col + e];
      else
        w[e / 2] |= (uint32_t) reinterpret_cast<const uint16_t*>(row)[col + e] << (e % 2 * 16);
    }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int DT, bool VEC>
__device__ __forceinline__ void store_vec(uint8_t* row, uint32_t col, uint32_t cols, const uint4& v) {
  constexpr int E = NormVec<DT>::kE;
  if (VEC && col + E <= cols) {
    *reinterpret_cast<uint4*>(row + (uint64_t)col * (16 / E)) = v;
    return;
  }
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int e = 0; e < E; ++e)
    if (col + e < cols) {
      if (DT == kF32)
        reinterpret_cast<uint32_t*>(row)[col + e] = w[e];
      else
        reinterpret_cast<uint16_t*>(row)[col + e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
    }
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
// E weights from `col` on, in fp32; `none` where there are none.
template <int E>
__device__ __forceinline__ void load_weights(const uint8_t* p, int wdt, uint32_t col, uint32_t cols, float none, float (&f)[E]) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    f[e] = none;
    if (p && col + e < cols)
      f[e] = wdt == kF32 ? reinterpret_cast<const float*>(p)[col + e] : bits_f((uint32_t) reinterpret_cast<const uint16_t*>(p)[col + e] << 16);
  }
}

// Sum over the TEAM threads that share a row, in a fixed order, the same in every thread.  `slot`: kNormWarps floats that the CTA
// uses for nothing else until two more of its barriers have passed.
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float* slot) {
#pragma unroll
  for (int d = 16; d; d /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if (TEAM == 32) return v;
  if (threadIdx.x % 32 == 0) slot[threadIdx.x / 32] = v;
  __syncthreads();
  float s = 0.0f;
#pragma unroll
  for (int w = 0; w < kNormWarps; ++w) s += slot[w];
  return s;
}

// ---- codes of a row of the output, E of its columns from `col` on in each lane (neighbouring lanes hold neighbouring columns)
// Every lane of the warp takes part; rows behind the last and columns behind the last give zeros.
template <int DT, int F, int E>
__device__ __forceinline__ void store_codes_f(const NormArgs& a, const MxLayout& l, uint32_t row, uint32_t col, const float (&v)[E], float unscale) {
  constexpr int kLanes = (F == kMxB32 ? 32 : 16) / E;  // lanes to a block
  uint32_t top = 0u;
#pragma unroll
  for (int e = 0; e < E; ++e) top = max(top, __float_as_uint(v[e]) & 0x7FFFFFFFu);
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
  const MxScale s = mx_scale<F>(top, unscale);
  float q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = e < E ? mx_quotient<F>(v[e % E], s) : 0.0f;
  const uint32_t codes = s.bad ? 0u : mx_codes8(q);
  // (col is a multiple of E, and kp of 64)
  if (row < l.r8 && col < l.kp) {
    uint8_t* p = a.packed + l.code_at(row, col / 32u) + col % 32u / 2u;
    if (E == 8)
      *reinterpret_cast<uint32_t*>(p) = codes;
    else
      *reinterpret_cast<uint16_t*>(p) = (uint16_t)codes;
  }
  // four blocks' scales to the lane that has the first of them
  uint32_t word = row < a.rows && col < a.cols ? s.byte : 0u;
  word |= __shfl_down_sync(0xFFFFFFFFu, word, kLanes) << 8;
  word |= __shfl_down_sync(0xFFFFFFFFu, word, 2 * kLanes) << 16;
  const uint32_t atom = col / (F == kMxB32 ? 128u : 64u);
  if (col % (F == kMxB32 ? 128u : 64u) == 0u && atom < l.atoms)
    *reinterpret_cast<uint32_t*>(a.packed + l.atom_at(row / 128u, atom) + MxLayout::scale_in_atom(row)) = word;
}
template <int DT, int E>
__device__ __forceinline__ void store_codes(const NormArgs& a, const MxLayout& l, uint32_t row, uint32_t col, const float (&v)[E], float unscale) {
  if (l.format == kMxB32)
    store_codes_f<DT, kMxB32, E>(a, l, row, col, v, unscale);
  else
    store_codes_f<DT, kMxB16, E>(a, l, row, col, v, unscale);
}

// Forward.  y = (x - mean) * rstd * gamma + beta, mean and variance from the row as it is held in registers (the squares of the
// distances from the mean, not of the values), sums in fp32.  TEAM threads to a row, V vectors to a thread; V = 0: any number, the row is
// read again for each of the three sweeps.
template <int DT, int TEAM, int V, bool VEC>
__global__ void __launch_bounds__(kNormThreads) norm_forward_kernel(const NormArgs a) {
  constexpr int E = NormVec<DT>::kE, N = V ? V : 1;
  __shared__ float slots[4][kNormWarps];
  const uint32_t t = threadIdx.x % TEAM, team = blockIdx.x * (kNormThreads / TEAM) + threadIdx.x / TEAM, teams = gridDim.x * (kNormThreads / TEAM);
  const MxLayout l(a.rows, a.cols, a.format);
  const uint32_t rows = a.packed ? (a.rows + 127u) / 128u * 128u : a.rows;  // (the padding of a container belongs to it)
  const uint32_t sweeps = V ? V : (a.cols + TEAM * E - 1u) / (TEAM * E);
  const uint32_t psweeps = a.packed ? sweeps : 0u;
  const float inv = __frcp_rn((float)a.cols), unscale = a.format == kMxB32 ? 1.0f : pow2_f(-a.exponent);
  dep_trigger();
  dep_wait();
  if (a.packed && blockIdx.x == 0 && threadIdx.x < 8) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (threadIdx.x == 0) v = make_uint4(kMxMagic, 1u | l.format << 16, l.rows, l.cols);
    if (threadIdx.x == 1) v = make_uint4((uint32_t)a.exponent, 0u, (uint32_t)l.total, (uint32_t)(l.total >> 32));
    if (threadIdx.x == 2) v = make_uint4((uint32_t)a.tensor_id, (uint32_t)(a.tensor_id >> 32), 0u, 0u);
    reinterpret_cast<uint4*>(a.packed)[threadIdx.x] = v;
  }
  uint32_t turn = 0;
  for (uint32_t row = team; row < rows; row += teams, turn ^= 2u) {
    if (row >= a.rows) {
      const float zero[E] = {};
      for (uint32_t i = 0; i < psweeps; ++i) store_codes<DT, E>(a, l, row, (i * TEAM + t) * E, zero, unscale);
      continue;
    }
    const uint8_t* x = a.x + (uint64_t)row * a.ldx * (16 / E);
    uint4 raw[N];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (V) raw[i] = load_vec<DT, VEC>(x, (i * TEAM + t) * E, a.cols);
    auto vec = [&](uint32_t i) { return V ? raw[i % N] : load_vec<DT, VEC>(x, (i * TEAM + t) * E, a.cols); };
#pragma unroll
    for (uint32_t i = 0; i < sweeps; ++i) {
      float f[E];
      unpack<DT, E>(vec(i), f);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += f[e];
    }
    const float mean = team_sum<TEAM>(sum, slots[turn]) * inv;
    float sq = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < sweeps; ++i) {
      float f[E];
      unpack<DT, E>(vec(i), f);
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
#pragma unroll
    for (uint32_t i = 0; i < sweeps; ++i) {
      const uint32_t col = (i * TEAM + t) * E;
      float f[E], g[E], b[E];
      unpack<DT, E>(vec(i), f);
      load_weights<E>(a.gamma, a.wdtype, col, a.cols, 1.0f, g);
      load_weights<E>(a.beta, a.wdtype, col, a.cols, 0.0f, b);
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = __fmaf_rn((f[e] - mean) * rstd, g[e], b[e]);
      const uint4 out = pack<DT, E>(f);
      if (y && col < a.cols) store_vec<DT, VEC>(y, col, a.cols, out);
      if (a.packed) {
        // codes of what y is in its type, so that they are those that compressing y gives
        unpack<DT, E>(out, f);
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (col + e >= a.cols) f[e] = 0.0f;
        store_codes<DT, E>(a, l, row, col, f, unscale);
      }
    }
  }
}

// ---- backward -----------------------------------------------------------------------------------------
// With xhat = (x - mean) * rstd and g = dy * gamma:  dx = rstd * (g - mean(g) - xhat * mean(g * xhat)), dgamma = sum of dy * xhat over the
// rows, dbeta = sum of dy.  A team takes rows one after the other and keeps the sums of its columns, in registers, or in shared memory
// where there are too many; a CTA's teams are added up at the end, and the CTAs' sums, which lie in the caller's workspace, by a second kernel:
// all in a fixed order.

// x of a row's columns from `col` on: dense, or four bits and the scale.
template <int DT, bool VEC, int X>
__device__ __forceinline__ uint4 load_x(const NormArgs& a, const MxLayout& l, uint32_t row, uint32_t col) {
  constexpr int E = NormVec<DT>::kE;
  if (X == 0) return load_vec<DT, VEC>(a.x + (uint64_t)row * a.ldx * (16 / E), col, a.cols);
  uint4 v = make_uint4(0u, 0u, 0u, 0u);
  if (col < a.cols) {
    constexpr int F = X - 1;
    v.x = *reinterpret_cast<const uint32_t*>(a.x + l.code_at(row, col / 32u) + col % 32u / 8u * 4u) >> (col % 8u * 4u);
    const uint32_t b = col / (F == kMxB32 ? 32u : 16u);
    v.y = a.x[l.atom_at(row / 128u, b / 4u) + MxLayout::scale_in_atom(row) + b % 4u];
  }
  return v;
}
template <int DT, int X, int E>
__device__ __forceinline__ void unpack_x(const uint4& v, float scale, float (&f)[E]) {
  if (X == 0) {
    unpack<DT, E>(v, f);
    return;
  }
  const float s = mx_factor<(X > 1 ? kMxB16 : kMxB32)>(v.y, scale);
  if constexpr (E == 8)
    mx_values8(v.x, f);
  else
    mx_values4(v.x, f);
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] *= s;
}

template <int DT, int TEAM, int V, bool VEC, int X>
__global__ void __launch_bounds__(kNormThreads) norm_backward_kernel(const NormArgs a) {
  constexpr int E = NormVec<DT>::kE, N = V ? V : 1;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ float slots[4][kNormWarps];
  float* acc = reinterpret_cast<float*>(smem);  // V = 0: dgamma and dbeta of the CTA; otherwise room for the other teams' sums
  const uint32_t t = threadIdx.x % TEAM, in_cta = threadIdx.x / TEAM, team = blockIdx.x * (kNormThreads / TEAM) + in_cta,
                 teams = gridDim.x * (kNormThreads / TEAM);
  const MxLayout l(a.rows, a.cols, a.format);
  const uint32_t sweeps = V ? V : (a.cols + TEAM * E - 1u) / (TEAM * E), wide = sweeps * TEAM * E;
  const float inv = __frcp_rn((float)a.cols);
  dep_trigger();
  dep_wait();
  int32_t exponent = 0;
  if (X) {
    const bool ok = mx_header_ok(a.x, a.x_bytes, l, &exponent);
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) *a.status = ok ? 0ull : status_word(kErrCorrupt);
    if (!ok) return;
  } else if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) {
    *a.status = 0ull;
  }
  const float scale = X == 1 + kMxB16 ? pow2_f(exponent) : 1.0f;
  float dg[N][E] = {}, db[N][E] = {}, gamma[N][E];
  if (V) {
#pragma unroll
    for (int i = 0; i < N; ++i) load_weights<E>(a.gamma, a.wdtype, (i * TEAM + t) * E, a.cols, 1.0f, gamma[i]);
  } else {
    for (uint32_t i = threadIdx.x; i < 2u * wide; i += kNormThreads) acc[i] = 0.0f;
    __syncthreads();
  }
  uint32_t turn = 0;
  for (uint32_t row = team; row < a.rows; row += teams, turn ^= 2u) {
    const uint8_t* dyr = a.dy + (uint64_t)row * a.ldy * (16 / E);
    const float mean = a.mean[row], rstd = a.rstd[row];
    uint4 rx[N], ry[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (V) {
        const uint32_t col = (i * TEAM + t) * E;
        ry[i] = load_vec<DT, VEC>(dyr, col, a.cols);
        rx[i] = load_x<DT, VEC, X>(a, l, row, col);
      }
    // xhat, dy and g = dy * gamma of vector i (zeros behind the last column, as dy is zero there)
    auto vec = [&](uint32_t i, float(&xh)[E], float(&dy)[E], float(&g)[E]) {
      const uint32_t col = (i * TEAM + t) * E;
      unpack<DT, E>(V ? ry[i % N] : load_vec<DT, VEC>(dyr, col, a.cols), dy);
      unpack_x<DT, X, E>(V ? rx[i % N] : load_x<DT, VEC, X>(a, l, row, col), scale, xh);
      if (!V) load_weights<E>(a.gamma, a.wdtype, col, a.cols, 1.0f, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        xh[e] = (xh[e] - mean) * rstd;
        g[e] = dy[e] * (V ? gamma[i % N][e] : g[e]);
        if (col + e >= a.cols) xh[e] = 0.0f;  // (a NaN mean or rstd must not come back through 0 * NaN)
      }
    };
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (uint32_t i = 0; i < sweeps; ++i) {
      float xh[E], dy[E], g[E];
      vec(i, xh, dy, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        s1 += g[e];
        s2 = __fmaf_rn(g[e], xh[e], s2);
      }
    }
    const float m1 = team_sum<TEAM>(s1, slots[turn]) * inv, m2 = team_sum<TEAM>(s2, slots[turn + 1]) * inv;
    uint8_t* dxr = a.dx ? a.dx + (uint64_t)row * a.ldx * (16 / E) : nullptr;
#pragma unroll
    for (uint32_t i = 0; i < sweeps; ++i) {
      const uint32_t col = (i * TEAM + t) * E;
      float xh[E], dy[E], g[E];
      vec(i, xh, dy, g);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (V) {
          dg[i % N][e] = __fmaf_rn(dy[e], xh[e], dg[i % N][e]);
          db[i % N][e] += dy[e];
        } else {  // (a team is the CTA; thread t alone has these columns)
          acc[col + e] = __fmaf_rn(dy[e], xh[e], acc[col + e]);
          acc[wide + col + e] += dy[e];
        }
        g[e] = rstd * (g[e] - m1 - xh[e] * m2);
      }
      if (dxr && col < a.cols) store_vec<DT, VEC>(dxr, col, a.cols, pack<DT, E>(g));
    }
  }
  if (!a.work) return;
  float* out = a.work + (uint64_t)blockIdx.x * 2u * a.cols;
  if (V == 0) {
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < a.cols; c += kNormThreads) {
      out[c] = acc[c];
      out[a.cols + c] = acc[wide + c];
    }
    return;
  }
  if (TEAM == 32) {  // the CTA's teams one after the other
    for (uint32_t w = 0; w < (uint32_t)kNormWarps; ++w) {
      if (in_cta == w) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const uint32_t at = (i * TEAM + t) * E + e;
            acc[at] = w ? acc[at] + dg[i][e] : dg[i][e];
            acc[wide + at] = w ? acc[wide + at] + db[i][e] : db[i][e];
          }
      }
      __syncthreads();
    }
    for (uint32_t c = threadIdx.x; c < a.cols; c += kNormThreads) {
      out[c] = acc[c];
      out[a.cols + c] = acc[wide + c];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t at = (i * TEAM + t) * E + e;
        if (at < a.cols) {
          out[at] = dg[i][e];
          out[a.cols + at] = db[i][e];
        }
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
  if (c < 2u * a.cols)
    for (uint32_t i = warp; i < a.parts; i += kNormWarps) s += a.work[(uint64_t)i * 2u * a.cols + c];
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

template <int DT, int TEAM, int V, bool VEC>
int launch_forward_t(const NormArgs& a, cudaStream_t stream) {
  const uint64_t rows = a.packed ? ((uint64_t)a.rows + 127) / 128 * 128 : a.rows;
  const uint32_t grid = (uint32_t)std::min<uint64_t>((rows * TEAM + kNormThreads - 1) / kNormThreads, (uint64_t)sm_count() * 8);
  return launch_plain<norm_forward_kernel<DT, TEAM, V, VEC>>(grid, kNormThreads, 0, 1, stream, a);
}
template <int DT, bool VEC>
int launch_forward_dv(const NormArgs& a, cudaStream_t stream) {
  const uint32_t vecs = (a.cols + NormVec<DT>::kE - 1) / NormVec<DT>::kE;
  if (vecs <= 32) return launch_forward_t<DT, 32, 1, VEC>(a, stream);
  if (vecs <= 128) return launch_forward_t<DT, 32, 4, VEC>(a, stream);
  if (vecs <= 256) return launch_forward_t<DT, 256, 1, VEC>(a, stream);
  if (vecs <= 512) return launch_forward_t<DT, 256, 2, VEC>(a, stream);
  if (vecs <= 1024) return launch_forward_t<DT, 256, 4, VEC>(a, stream);
  if (vecs <= 2048) return launch_forward_t<DT, 256, 8, VEC>(a, stream);
  return launch_forward_t<DT, 256, 0, VEC>(a, stream);
}

template <int DT, int TEAM, int V, bool VEC, int X>
int launch_backward_t(const NormArgs& a, cudaStream_t stream) {
  constexpr uint32_t E = NormVec<DT>::kE;
  const uint32_t sweeps = V ? V : (a.cols + TEAM * E - 1u) / (TEAM * E);
  const size_t smem = V == 0 || TEAM == 32 ? (size_t)8 * sweeps * TEAM * E : 0;
  return launch_plain<norm_backward_kernel<DT, TEAM, V, VEC, X>>(a.parts, kNormThreads, smem, 1, stream, a);
}
template <int DT, bool VEC, int X>
int launch_backward_dx(const NormArgs& a, cudaStream_t stream) {
  const uint32_t vecs = (a.cols + NormVec<DT>::kE - 1) / NormVec<DT>::kE;
  if (vecs <= 32) return launch_backward_t<DT, 32, 1, VEC, X>(a, stream);
  if (vecs <= 128) return launch_backward_t<DT, 32, 4, VEC, X>(a, stream);
  if (vecs <= 256) return launch_backward_t<DT, 256, 1, VEC, X>(a, stream);
  if (vecs <= 512) return launch_backward_t<DT, 256, 2, VEC, X>(a, stream);
  if (vecs <= 1024) return launch_backward_t<DT, 256, 4, VEC, X>(a, stream);
  return launch_backward_t<DT, 256, 0, VEC, X>(a, stream);
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
  const uint32_t each = cols <= (dtype == kF32 ? 512u : 1024u) ? 32u : 4u;  // rows that make a CTA worth its sums (a warp or a CTA to a row)
  const uint32_t n = rows / each + (rows % each ? 1u : 0u);
  return n < 296u ? n : 296u;
}

int launch_norm_forward(const NormArgs& a, int dtype, cudaStream_t stream) {
  if (sm_count() < 1) return FH_ERR_CUDA;
  const uint64_t es = dtype == kF32 ? 4 : 2;
  const bool vec = aligned16(a.x) && aligned16(a.y) && a.ldx * es % 16 == 0 && (!a.y || a.ldy * es % 16 == 0);
  if (dtype == kF32) return vec ? launch_forward_dv<kF32, true>(a, stream) : launch_forward_dv<kF32, false>(a, stream);
  return vec ? launch_forward_dv<kBF16, true>(a, stream) : launch_forward_dv<kBF16, false>(a, stream);
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
