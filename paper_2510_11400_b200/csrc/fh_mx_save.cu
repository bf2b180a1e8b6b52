// Dense matrices into microscaled 4-bit containers and back.
#include "fh_launch.cuh"
#include "fh_mx.cuh"
#include "fh_mx_launch.cuh"

namespace fh {
namespace {

constexpr int kTile = 128;      // rows and columns of a tile: one group of scales either way
constexpr int kSaveThreads = 256;

template <int DT>
struct Elem;
template <>
struct Elem<kF32> {
  static constexpr int kBytes = 4, kVec = 4;  // elements of a 16-byte vector
};
template <>
struct Elem<kBF16> {
  static constexpr int kBytes = 2, kVec = 8;
};
// A tile in shared memory: rows 16 bytes longer than their data, so that 16-byte accesses of consecutive rows and 4-byte accesses
// of consecutive columns both fall on different banks.
template <int DT>
constexpr int kPitch = kTile * Elem<DT>::kBytes + 16;

// Two neighbouring elements of bf16 of a row of a tile, in one word of memory wherever the row begins (off the 16-byte grid): pair `q` of the
// 128 x 64 of the tile.  Rows that begin in the middle of a word have their first element besides.
struct BfPair {
  uint32_t r, c;            // of the tile; c is the pair's first column
  uint64_t place;           // element of the matrix
  bool whole, half, first;  // both elements exist, the first of them does, and the row's first one, ahead of the pair
  __device__ __forceinline__ BfPair(const void* base, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t r0, uint32_t c0, uint32_t q) {
    r = q / (kTile / 2);
    const uint64_t row = (uint64_t)(r0 + r) * ld + c0;
    const uint32_t shift = (uint32_t)(((uintptr_t)base >> 1) + row) & 1u, end = min((uint32_t)kTile, cols - c0);
    c = q % (kTile / 2) * 2 + shift;
    place = row + c;
    const bool in = r0 + r < rows;
    whole = in && c + 1u < end;
    half = in && c < end;
    first = in && c == 1u;
  }
};

// Loads the tile at (r0, c0), zeros outside the matrix, and waits for it.  VEC: rows start on 16-byte boundaries.  Copies go straight to shared
// memory, all of them under way at once; an element of bf16 is too small for one, so rows off the 16-byte grid come by way of registers.
template <int DT, bool VEC>
__device__ __forceinline__ void load_tile(uint8_t* tile, const uint8_t* src, uint64_t ld, uint32_t rows, uint32_t cols, uint32_t r0,
                                          uint32_t c0) {
  constexpr int ES = Elem<DT>::kBytes, VE = Elem<DT>::kVec, V = kTile / VE;  // V vectors a row
  const uint32_t base = smem_u32(tile);
  if (VEC) {
#pragma unroll
    for (int i = 0; i < kTile * V / kSaveThreads; ++i) {
      const uint32_t at = threadIdx.x + i * kSaveThreads, r = at / V, c = at % V * VE;
      const uint32_t n = r0 + r < rows && c0 + c < cols ? min((uint32_t)VE, cols - (c0 + c)) : 0u;
      const uint8_t* p = src + (n ? ((uint64_t)(r0 + r) * ld + c0 + c) * ES : 0u);
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(base + r * kPitch<DT> + c * ES), "l"(p), "r"(n * ES) : "memory");
    }
  } else if (DT == kF32) {
#pragma unroll 8
    for (int i = 0; i < kTile * kTile / kSaveThreads; ++i) {
      const uint32_t at = threadIdx.x + i * kSaveThreads, r = at / kTile, c = at % kTile;
      const bool there = r0 + r < rows && c0 + c < cols;
      const uint8_t* p = src + (there ? ((uint64_t)(r0 + r) * ld + c0 + c) * ES : 0u);
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(base + r * kPitch<DT> + c * ES), "l"(p), "r"(there ? 4u : 0u) : "memory");
    }
  } else {
    const uint16_t* s16 = reinterpret_cast<const uint16_t*>(src);
#pragma unroll 1
    for (int i = 0; i < kTile * kTile / 2 / kSaveThreads; i += 8) {
      uint32_t w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t at = threadIdx.x + (i + k) * kSaveThreads, r = at / (kTile / 2), c = at % (kTile / 2) * 2;
        const uint16_t* p = s16 + (uint64_t)(r0 + r) * ld + c0 + c;
        const uint32_t lo = r0 + r < rows && c0 + c < cols ? p[0] : 0u, hi = r0 + r < rows && c0 + c + 1u < cols ? p[1] : 0u;
        w[k] = lo | hi << 16;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t at = threadIdx.x + (i + k) * kSaveThreads, r = at / (kTile / 2), c = at % (kTile / 2) * 2;
        *reinterpret_cast<uint32_t*>(tile + r * kPitch<DT> + c * ES) = w[k];
      }
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
}

// Philox-4x32-10 with the ten rounds' keys made on the host (see philox4x32_10).
struct MxKey {
  const uint32_t* rounds;
  uint32_t id_lo, id_hi;
  __device__ __forceinline__ void draw(uint32_t c0, uint32_t c1, uint32_t (&out)[4]) const {
    uint32_t c2 = id_lo, c3 = id_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
      const uint32_t h0 = __umulhi(0xD2511F53u, c0), l0 = 0xD2511F53u * c0, h1 = __umulhi(0xCD9E8D57u, c2), l1 = 0xCD9E8D57u * c2;
      c0 = h1 ^ c1 ^ rounds[2 * r];
      c1 = l1;
      c2 = h0 ^ c3 ^ rounds[2 * r + 1];
      c3 = l0;
    }
    out[0] = c0;
    out[1] = c1;
    out[2] = c2;
    out[3] = c3;
  }
};

// The block of NB elements get(0) ... get(NB - 1) of a matrix's row, from column `col` on, to NB / 8 words of codes; its scale byte.
// `scale`: 2^exponent, `unscale` its inverse.
template <int F, bool RANDOM, int NB, typename G>
__device__ __forceinline__ uint32_t encode_block(G get, uint32_t top, float scale, float unscale, uint32_t row, uint32_t col, const MxKey& key,
                                                 uint32_t* codes) {
  const MxScale s = mx_scale<F>(top, unscale);
  const float s_full = s.s * scale;
#pragma unroll
  for (int i = 0; i < NB / 8; ++i) {
    float v[8];
    if (RANDOM) {
      uint32_t w[4];
      key.draw(col / 8u + i, row, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = get(8 * i + 2 * e);
        v[2 * e + 1] = get(8 * i + 2 * e + 1);
        mx_random2<F>(v[2 * e], v[2 * e + 1], s, s_full, 0x3F800000u | (w[e] << 7 & 0x007FFF80u), 0x3F800000u | (w[e] >> 9 & 0x007FFF80u));
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = mx_quotient<F>(get(8 * i + e), s);
    }
    codes[i] = s.bad ? 0u : mx_codes8(v);
  }
  return s.byte;
}

// Random rounding, blocks of 16: magnitudes beyond eight times the largest scale become that, which is stored as 6 all the same; mx_random2's
// arithmetic holds for quotients up to 2^105 only.  (Blocks that have such a value are rare, and the others pay one comparison.)
// `top`: bits of the block's largest magnitude, in bf16 of both columns' that a word holds.
template <int F, bool RANDOM, int DT, int W>
__device__ __forceinline__ void clip_far(uint32_t (&w)[W], uint32_t top, int32_t exponent) {
  if (F != kMxB16 || !RANDOM) return;
  const uint32_t far = (uint32_t)(138 + exponent) << 23 | 0x00600000u;  // 8 * 448 * 2^exponent = 1.75 * 2^(11 + exponent)
  if (top <= far) return;
#pragma unroll
  for (int i = 0; i < W; ++i)
    w[i] = DT == kF32 ? (w[i] & 0x80000000u) | min(w[i] & 0x7FFFFFFFu, far) : (w[i] & 0x80008000u) | __vminu2(w[i] & 0x7FFF7FFFu, far >> 16 | far);
}

__device__ __forceinline__ float bf_lo(uint32_t w) { return bits_f(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return bits_f(w & 0xFFFF0000u); }

// One tile of 128 x 128 elements a CTA: read once into shared memory, from there blocks along rows (a thread for 32 columns of a
// row) and blocks along columns (a thread for 32 rows of a column, in bf16 of two columns), each written as 16 bytes next to its
// neighbours'.
template <int DT, int F, bool RANDOM, bool VEC>
__global__ void __launch_bounds__(kSaveThreads) mx_compress_kernel(const __grid_constant__ MxSaveArgs a) {
  constexpr int ES = Elem<DT>::kBytes, NB = F == kMxB32 ? 32 : 16, NS = 32 / NB;  // NS scales to 32 elements
  extern __shared__ __align__(16) uint8_t smem[];
  uint8_t* tile = smem;
  uint8_t* scales = smem + kTile * kPitch<DT>;  // two groups of 512 bytes along rows, two along columns
  const uint32_t tid = threadIdx.x;
  const MxLayout lr(a.rows, a.cols, F), lc(a.cols, a.rows, F);
  const uint32_t tiles_c = (a.cols + kTile - 1u) / kTile, tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const uint32_t r0 = tr * kTile, c0 = tc * kTile;
  const float unscale = F == kMxB32 ? 1.0f : pow2_f(-a.exponent);
  const float scale = F == kMxB32 ? 1.0f : pow2_f(a.exponent);
  const MxKey key = {a.round_keys, (uint32_t)a.tensor_id, (uint32_t)(a.tensor_id >> 32)};
  dep_trigger();
  for (uint32_t i = tid; i < 128; i += kSaveThreads) reinterpret_cast<uint4*>(scales)[i] = make_uint4(0u, 0u, 0u, 0u);
  dep_wait();
  load_tile<DT, VEC>(tile, a.src, a.ld, a.rows, a.cols, r0, c0);
  if (blockIdx.x == 0 && tid < 16) {
    const bool col = tid >= 8;
    uint8_t* dst = col ? a.by_cols : a.by_rows;
    const uint64_t total = col ? lc.total : lr.total;
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (tid % 8 == 0) v = make_uint4(kMxMagic, 1u | (uint32_t)F << 16 | (uint32_t)RANDOM << 24, col ? a.cols : a.rows, col ? a.rows : a.cols);
    if (tid % 8 == 1) v = make_uint4((uint32_t)a.exponent, 0u, (uint32_t)total, (uint32_t)(total >> 32));
    if (tid % 8 == 2) v = make_uint4(key.id_lo, key.id_hi, 0u, 0u);
    if (dst) reinterpret_cast<uint4*>(dst)[tid % 8] = v;
  }
  __syncthreads();
  if (a.by_rows) {
#pragma unroll 1
    for (uint32_t t = tid; t < 4 * kTile; t += kSaveThreads) {
      const uint32_t r = t % kTile, j = t / kTile, row = r0 + r, col = c0 + 32u * j;
      if (row >= lr.r8 || col >= lr.kp) continue;
      const uint4* p = reinterpret_cast<const uint4*>(tile + r * kPitch<DT> + 32 * ES * j);
      uint32_t codes[4];
#pragma unroll
      for (int h = 0; h < NS; ++h) {
        constexpr int W = NB * ES / 4;
        uint32_t w[W], top = 0u, byte;
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
          const uint4 v = p[h * (W / 4) + i];
          w[4 * i] = v.x;
          w[4 * i + 1] = v.y;
          w[4 * i + 2] = v.z;
          w[4 * i + 3] = v.w;
        }
        if (DT == kF32) {
#pragma unroll
          for (int i = 0; i < W; ++i) top = max(top, w[i] & 0x7FFFFFFFu);
          clip_far<F, RANDOM, DT>(w, top, a.exponent);
          byte = encode_block<F, RANDOM, NB>([&](int i) { return bits_f(w[i]); }, top, scale, unscale, row, col + h * NB, key, codes + h * (NB / 8));
        } else {
#pragma unroll
          for (int i = 0; i < W; ++i) top = __vmaxu2(top, w[i] & 0x7FFF7FFFu);
          top = max(top << 16, top & 0xFFFF0000u);
          clip_far<F, RANDOM, DT>(w, top, a.exponent);
          byte = encode_block<F, RANDOM, NB>([&](int i) { return i % 2 ? bf_hi(w[i / 2]) : bf_lo(w[i / 2]); }, top, scale, unscale, row,
                                             col + h * NB, key, codes + h * (NB / 8));
        }
        if (row < a.rows && col + h * NB < a.cols)
          scales[(j * NS + h) / 4 * 512 + MxLayout::scale_in_atom(r) + (j * NS + h) % 4] = (uint8_t)byte;
      }
      *reinterpret_cast<uint4*>(a.by_rows + lr.code_at(row, col / 32u)) = make_uint4(codes[0], codes[1], codes[2], codes[3]);
    }
  }
  if (a.by_cols) {
    constexpr int CW = 4 / ES;  // columns to a 4-byte word
#pragma unroll 1
    for (uint32_t t = tid; t < 4 * kTile / CW; t += kSaveThreads) {
      const uint32_t c = t % (kTile / CW) * CW, j = t / (kTile / CW), row = c0 + c, col = r0 + 32u * j;  // of the transpose
      if (row >= lc.r8 || col >= lc.kp) continue;
      const uint8_t* p = tile + 32 * j * kPitch<DT> + c * ES;
      uint32_t codes[CW][4];
#pragma unroll
      for (int h = 0; h < NS; ++h) {
        uint32_t w[NB], top = 0u;
#pragma unroll
        for (int i = 0; i < NB; ++i) w[i] = *reinterpret_cast<const uint32_t*>(p + (h * NB + i) * kPitch<DT>);
#pragma unroll
        for (int i = 0; i < NB; ++i) top = DT == kF32 ? max(top, w[i] & 0x7FFFFFFFu) : __vmaxu2(top, w[i] & 0x7FFF7FFFu);
        clip_far<F, RANDOM, DT>(w, DT == kF32 ? top : max(top << 16, top & 0xFFFF0000u), a.exponent);
#pragma unroll
        for (int q = 0; q < CW; ++q) {
          uint32_t byte;
          if (DT == kF32)
            byte = encode_block<F, RANDOM, NB>([&](int i) { return bits_f(w[i]); }, top, scale, unscale, row, col + h * NB, key, codes[q] + h * (NB / 8));
          else
            byte = encode_block<F, RANDOM, NB>([&](int i) { return q ? bf_hi(w[i]) : bf_lo(w[i]); }, q ? top & 0xFFFF0000u : top << 16,
                                               scale, unscale, row + q, col + h * NB, key, codes[q] + h * (NB / 8));
          if (row + q < a.cols && col + h * NB < a.rows)
            scales[1024 + (j * NS + h) / 4 * 512 + MxLayout::scale_in_atom(c + q) + (j * NS + h) % 4] = (uint8_t)byte;
        }
      }
#pragma unroll
      for (int q = 0; q < CW; ++q)  // (r8 is even, and so is row in bf16)
        *reinterpret_cast<uint4*>(a.by_cols + lc.code_at(row + q, col / 32u)) = make_uint4(codes[q][0], codes[q][1], codes[q][2], codes[q][3]);
    }
  }
  __syncthreads();
  if (tid < 128) {
    constexpr uint32_t A = F == kMxB32 ? 1 : 2;  // groups of scales to a tile
    const bool col = tid >= 64;
    const uint32_t atom = tid % 64 / 32, at = col ? tr * A + atom : tc * A + atom;
    uint8_t* dst = col ? a.by_cols : a.by_rows;
    if (dst && atom < A && at < (col ? lc.atoms : lr.atoms))
      *reinterpret_cast<uint4*>(dst + (col ? lc.atom_at(tc, at) : lr.atom_at(tr, at)) + tid % 32 * 16) = reinterpret_cast<const uint4*>(scales)[tid];
  }
}

// The way back: codes and scales of a tile to shared memory as values, and from there to the matrix in whole lines.
template <int DT, int F, bool VEC>
__global__ void __launch_bounds__(kSaveThreads) mx_decompress_kernel(const MxSaveArgs a) {
  constexpr int ES = Elem<DT>::kBytes, VE = Elem<DT>::kVec, V = kTile / VE;
  extern __shared__ __align__(16) uint8_t smem[];
  const uint32_t tid = threadIdx.x;
  const MxLayout l(a.rows, a.cols, F);
  const uint32_t tiles_c = (a.cols + kTile - 1u) / kTile, tr = blockIdx.x / tiles_c, tc = blockIdx.x % tiles_c;
  const uint32_t r0 = tr * kTile, c0 = tc * kTile;
  dep_trigger();
  dep_wait();
  int32_t exponent;
  const bool ok = mx_header_ok(a.src, a.src_bytes, l, &exponent);
  if (blockIdx.x == 0 && tid == 0 && a.status) *a.status = ok ? 0ull : status_word(kErrCorrupt);
  if (!ok) return;
  const float scale = F == kMxB32 ? 1.0f : pow2_f(exponent);
#pragma unroll
  for (uint32_t k = 0; k < 4 * kTile / kSaveThreads; ++k) {
    const uint32_t t = tid + k * kSaveThreads, r = t % kTile, j = t / kTile, row = r0 + r, col = c0 + 32u * j;
    if (row >= a.rows || col >= a.cols) continue;
    const uint4 q = *reinterpret_cast<const uint4*>(a.src + l.code_at(row, col / 32u));
    const uint32_t word = *reinterpret_cast<const uint32_t*>(a.src + l.atom_at(tr, F == kMxB32 ? tc : 2u * tc + j / 2u) +
                                                              MxLayout::scale_in_atom(r));
    const uint32_t at = F == kMxB32 ? 8u * j : 16u * (j % 2u);
    const float f0 = mx_factor<F>(word >> at & 255u, scale), f1 = F == kMxB32 ? f0 : mx_factor<F>(word >> (at + 8u) & 255u, scale);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint4* p = reinterpret_cast<uint4*>(smem + r * kPitch<DT> + 32 * ES * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float v[8];
      mx_values8(w[i], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= i < 2 ? f0 : f1;
      if (DT == kF32) {
        p[2 * i] = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        p[2 * i + 1] = make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7]));
      } else {  // (exact: a value has two significant bits, times four of a scale of B16)
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
          o[e] = *reinterpret_cast<const uint32_t*>(&b);
        }
        p[i] = make_uint4(o[0], o[1], o[2], o[3]);
      }
    }
  }
  __syncthreads();
  if (VEC) {
#pragma unroll
    for (int i = 0; i < kTile * V / kSaveThreads; ++i) {
      const uint32_t at = tid + i * kSaveThreads, r = at / V, c = at % V * VE;
      if (r0 + r >= a.rows || c0 + c >= a.cols) continue;
      const uint8_t* s = smem + r * kPitch<DT> + c * ES;
      uint8_t* p = a.dst + ((uint64_t)(r0 + r) * a.ld + c0 + c) * ES;
      if (c0 + c + VE <= a.cols) {
        *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(s);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (c0 + c + e < a.cols) {
            if (DT == kF32)
              reinterpret_cast<uint32_t*>(p)[e] = reinterpret_cast<const uint32_t*>(s)[e];
            else
              reinterpret_cast<uint16_t*>(p)[e] = reinterpret_cast<const uint16_t*>(s)[e];
          }
      }
    }
  } else if (DT == kF32) {  // rows off the 16-byte grid: neighbouring lanes store neighbouring words (16384 x 4095 bf16: 158 us with 16 bytes a lane)
#pragma unroll 8
    for (int i = 0; i < kTile * kTile / kSaveThreads; ++i) {
      const uint32_t at = tid + i * kSaveThreads, r = at / kTile, c = at % kTile;
      if (r0 + r < a.rows && c0 + c < a.cols)
        reinterpret_cast<uint32_t*>(a.dst)[(uint64_t)(r0 + r) * a.ld + c0 + c] = *reinterpret_cast<const uint32_t*>(smem + r * kPitch<DT> + c * ES);
    }
  } else {
#pragma unroll 8
    for (int i = 0; i < kTile * kTile / 2 / kSaveThreads; ++i) {
      const BfPair at(a.dst, a.ld, a.rows, a.cols, r0, c0, tid + i * kSaveThreads);
      const uint16_t* s = reinterpret_cast<const uint16_t*>(smem + at.r * kPitch<DT>) + at.c;
      uint16_t* p = reinterpret_cast<uint16_t*>(a.dst) + at.place;
      if (at.whole)
        *reinterpret_cast<uint32_t*>(p) = s[0] | (uint32_t)s[1] << 16;
      else if (at.half)
        *p = s[0];
      if (at.first) p[-1] = s[-1];
    }
  }
}

template <int DT, int F, bool RANDOM, bool VEC>
int launch_compress_t(const MxSaveArgs& a, uint32_t grid, cudaStream_t stream) {
  constexpr size_t smem = kTile * kPitch<DT> + 2048;
  return launch_plain<mx_compress_kernel<DT, F, RANDOM, VEC>>(grid, kSaveThreads, smem, 1, stream, a);
}
template <int DT, int F, bool VEC>
int launch_decompress_t(const MxSaveArgs& a, uint32_t grid, cudaStream_t stream) {
  constexpr size_t smem = kTile * kPitch<DT>;
  return launch_plain<mx_decompress_kernel<DT, F, VEC>>(grid, kSaveThreads, smem, 1, stream, a);
}
template <int DT, int F>
int launch_save_df(const MxSaveArgs& a, bool compress, bool random, bool vec, uint32_t grid, cudaStream_t stream) {
  if (!compress) return vec ? launch_decompress_t<DT, F, true>(a, grid, stream) : launch_decompress_t<DT, F, false>(a, grid, stream);
  if (random) return vec ? launch_compress_t<DT, F, true, true>(a, grid, stream) : launch_compress_t<DT, F, true, false>(a, grid, stream);
  return vec ? launch_compress_t<DT, F, false, true>(a, grid, stream) : launch_compress_t<DT, F, false, false>(a, grid, stream);
}

}  // namespace

int launch_mx_save(const MxSaveArgs& a, int dtype, int format, bool compress, bool random, cudaStream_t stream) {
  const uint64_t tiles = (((uint64_t)a.rows + kTile - 1) / kTile) * (((uint64_t)a.cols + kTile - 1) / kTile);
  if (tiles > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
  const int es = dtype == kF32 ? 4 : 2;
  const uintptr_t dense = (uintptr_t)(compress ? a.src : a.dst);
  const bool vec = dense % 16 == 0 && a.ld * es % 16 == 0;
  const uint32_t grid = (uint32_t)tiles;
  if (dtype == kF32)
    return format == kMxB32 ? launch_save_df<kF32, kMxB32>(a, compress, random, vec, grid, stream)
                            : launch_save_df<kF32, kMxB16>(a, compress, random, vec, grid, stream);
  return format == kMxB32 ? launch_save_df<kBF16, kMxB32>(a, compress, random, vec, grid, stream)
                          : launch_save_df<kBF16, kMxB16>(a, compress, random, vec, grid, stream);
}

}  // namespace fh
