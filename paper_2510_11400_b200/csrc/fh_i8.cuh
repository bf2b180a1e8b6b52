// Matrices in 8-bit integers with a scale for each row: the container's layout and the conversions, shared by the kernels that write
// containers (fh_i8_save.cu, fh_gated.cu) and those that read them (fh_i8_save.cu, fh_i8_product.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fh_device.cuh"

namespace fh {

constexpr uint32_t kI8Magic = 0x38494846u;  // "FHI8"
constexpr uint32_t kI8HeadBytes = 128;

// The container of a rows x cols matrix (fh.h describes it).  A chunk is 16 columns.
struct I8Layout {
  uint32_t rows, cols;
  uint32_t r8, kp;  // rows padded to 8, columns to 32: what codes are stored for
  uint64_t code_bytes, total;

  __host__ __device__ I8Layout() {}
  __host__ __device__ I8Layout(uint32_t rows_, uint32_t cols_) : rows(rows_), cols(cols_) {
    r8 = (rows + 7u) & ~7u;
    kp = (cols + 31u) & ~31u;
    code_bytes = (uint64_t)r8 * kp;
    total = kI8HeadBytes + code_bytes + 4ull * r8;
  }
  __host__ __device__ uint32_t chunks() const { return kp / 16u; }
  // Rows of codes that block b of 128 rows has.
  __host__ __device__ uint32_t block_rows(uint32_t b) const {
    const uint32_t left = r8 - b * 128u;
    return left < 128u ? left : 128u;
  }
  // The 16 bytes of the codes of chunk j of a row; the next chunk's are 16 * block_rows behind them.
  __host__ __device__ uint64_t code_at(uint32_t row, uint32_t j) const {
    const uint32_t b = row / 128u;
    return kI8HeadBytes + (uint64_t)b * 128u * kp + ((uint64_t)j * block_rows(b) + row % 128u) * 16u;
  }
  __host__ __device__ uint64_t magnitude_at(uint32_t row) const { return kI8HeadBytes + code_bytes + 4ull * row; }
};

__device__ __forceinline__ void i8_write_header(uint8_t* dst, const I8Layout& l, uint32_t i) {  // word i of 32
  uint32_t w = 0u;
  if (i == 0u) w = kI8Magic;
  if (i == 1u) w = 1u;
  if (i == 2u) w = l.rows;
  if (i == 3u) w = l.cols;
  if (i == 6u) w = (uint32_t)l.total;
  if (i == 7u) w = (uint32_t)(l.total >> 32);
  reinterpret_cast<uint32_t*>(dst)[i] = w;
}
// Whether a container is the one expected.  (That it is large enough the host knows too: then the header is there to be read, and what the layout has.)
__device__ __forceinline__ bool i8_header_ok(const uint8_t* src, uint64_t src_bytes, const I8Layout& l) {
  if (src_bytes < l.total) return false;  // (so that the header is there to be read)
  const uint4 a = *reinterpret_cast<const uint4*>(src), b = *reinterpret_cast<const uint4*>(src + 16);
  return a.x == kI8Magic && a.y == 1u && a.z == l.rows && a.w == l.cols && b.x == 0u && b.y == 0u && ((uint64_t)b.w << 32 | b.z) == l.total;
}

// The scale of a row of magnitude `a`.
__device__ __forceinline__ float i8_scale(float a) {
  const float s = a * (1.0f / 127.0f);
  return a == 0.0f ? 0.0f : s < 1.17549435e-38f ? 1.17549435e-38f : s;  // (a NaN stays one)
}

constexpr float kI8Magic23 = 12582912.0f;  // 1.5 * 2^23

// How the elements of a row become codes: t = x * inv, rounded to a whole number k by adding 1.5 * 2^23, whose last bits then hold it.  inv is 1 / s
// to within 2^-24, and |x / s| <= 127 (1 + 2^-22), so t is within 2^-16 of x / s: k is right unless x / s lies that near to the middle between two whole
// numbers.
//
// fp32: what is left over, r = x - k s, is exact (a multiple of the last place of x or of s, at most 0.51 s), so that comparing 2 |r| with s settles the
// few elements whose |r| is next to s / 2.
//
// bf16: only half of the row's magnitude is that near to a middle (63.5), and elements whose quotient is a middle exactly.  With x = X 2^p and the
// magnitude M 2^q, X and M of eight bits, 127 x / magnitude is |254 X - (2 k + 1) M 2^(q - p)| / (2 M 2^(q - p)) away from the middle above k: nothing, or at
// least 1 / (2 M 2^(q - p)), which is thirty times what t may be off by (127 * 255 / (M 2^(q - p)) times 2^-21).  Nothing: 127 divides M, which then
// is 254, so that s is a power of two and everything is exact; or it divides 2 k + 1, which then is 127: x is half of the magnitude.  So inv is moved
// by a last place where half the magnitude would come out on the wrong side, and no element is looked at again.  (Half of the magnitude is no rare
// value: looking again at 16 elements where one of them is near a middle made 8192 x 4096 by rows take 60 us instead of 29.)
template <int DT>
struct I8Coder {
  float inv, s, edge;
  __device__ __forceinline__ I8Coder() {}
  // `bits`: of the row's largest magnitude.  A row with a NaN or an infinity has codes 0, whatever x is.
  __device__ __forceinline__ explicit I8Coder(uint32_t bits) {
    const bool bad = bits >= 0x7F800000u;
    s = bad ? 0.0f : i8_scale(__uint_as_float(bits));
    inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
    edge = s > 0.0f ? s * 0.49997f : __uint_as_float(0x7F800000u);
    if (DT == kBF16 && s > 1.17549435e-38f) {  // (the smallest scale is a power of two)
      // (127 s, not 63.5: what is left over of the smallest scales would be half of the smallest number)
      const float a = __uint_as_float(bits);
      const bool up = __fmaf_rn(-127.0f, s, a) >= 0.0f, got = __fmaf_rn(0.5f * a, inv, -63.5f) >= 0.0f;
      if (up != got) inv = __uint_as_float(__float_as_uint(inv) + (up ? 1u : ~0u));
    }
  }
};
__device__ __forceinline__ uint32_t i8_magnitude_bits(uint32_t top) { return top >= 0x7F800000u ? 0x7FC00000u : top; }

// One element, exactly.
__device__ __forceinline__ uint32_t i8_code_exact(float x, const I8Coder<kF32>& c) {
  if (!(c.s > 0.0f)) return 0u;
  float k = __fmaf_rn(x, c.inv, kI8Magic23) - kI8Magic23;
  const float r = __fmaf_rn(-k, c.s, x), twice = 2.0f * fabsf(r);
  if (twice > c.s || (twice == c.s && ((int)k & 1))) k += r > 0.0f ? 1.0f : -1.0f;
  return (uint32_t)(int)k & 255u;
}
// 16 elements, those of a row in bf16 all of that type, to 16 bytes.
template <int DT>
__device__ __forceinline__ uint4 i8_codes16(const float (&x)[16], const I8Coder<DT>& c) {
  const f32x2 inv = pack2(c.inv, c.inv), magic = pack2(kI8Magic23, kI8Magic23), less = pack2(-kI8Magic23, -kI8Magic23), ms = pack2(-c.s, -c.s);
  uint32_t t[16];
  float far = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; i += 2) {
    const f32x2 v = pack2(x[i], x[i + 1]), w = fma2(v, inv, magic);
    unpack2u(w, t[i], t[i + 1]);
    if (DT == kF32) {
      float r0, r1;
      unpack2(fma2(add2(w, less), ms, v), r0, r1);
      far = fmaxf(fmaxf(far, fabsf(r0)), fabsf(r1));
    }
  }
  if (DT == kF32 && !(far <= c.edge)) {
    if constexpr (DT == kF32) {
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i] = i8_code_exact(x[i], c);
    }
  } else if (c.s == 0.0f) {
    return make_uint4(0u, 0u, 0u, 0u);
  }
  uint4 r;
  r.x = __byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410);
  r.y = __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410);
  r.z = __byte_perm(__byte_perm(t[8], t[9], 0x0040), __byte_perm(t[10], t[11], 0x0040), 0x5410);
  r.w = __byte_perm(__byte_perm(t[12], t[13], 0x0040), __byte_perm(t[14], t[15], 0x0040), 0x5410);
  return r;
}

// 16 elements of a row of a dense matrix, as they are in memory, and as fp32.
template <int DT>
struct Raw16 {
  static constexpr int kWords = DT == kF32 ? 16 : 8;
  uint32_t w[kWords];

  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
  }
  // Elements 0 ... n - 1 (n <= 16, zeros behind them) at p.  VEC: p is on a 16-byte boundary.
  template <bool VEC>
  __device__ __forceinline__ void load(const uint8_t* p, int n) {
    if (VEC && n == 16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 v = reinterpret_cast<const uint4*>(p)[i / 4];
        w[i] = v.x;
        w[i + 1] = v.y;
        w[i + 2] = v.z;
        w[i + 3] = v.w;
      }
      return;
    }
    if (DT == kF32) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = i < n ? reinterpret_cast<const uint32_t*>(p)[i] : 0u;
    } else {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        const uint32_t lo = 2 * i < n ? h[2 * i] : 0u, hi = 2 * i + 1 < n ? h[2 * i + 1] : 0u;
        w[i] = lo | hi << 16;
      }
    }
  }
  template <bool VEC>
  __device__ __forceinline__ void store(uint8_t* p, int n) const {
    if (VEC && n == 16) {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
      return;
    }
    if (DT == kF32) {
#pragma unroll
      for (int i = 0; i < kWords; ++i)
        if (i < n) reinterpret_cast<uint32_t*>(p)[i] = w[i];
    } else {
      uint16_t* h = reinterpret_cast<uint16_t*>(p);
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        if (2 * i < n) h[2 * i] = (uint16_t)w[i];
        if (2 * i + 1 < n) h[2 * i + 1] = (uint16_t)(w[i] >> 16);
      }
    }
  }
  __device__ __forceinline__ void values(float (&v)[16]) const {
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      if (DT == kF32) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
  }
  // Rounded to the type.
  __device__ __forceinline__ void take(const float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = DT == kF32 ? __float_as_uint(v[i]) : f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
  }
  // Bits of the largest magnitude, as fp32's (in bf16 two columns' maxima side by side until the end).
  __device__ __forceinline__ uint32_t top() const {
    uint32_t m = w[0] & (DT == kF32 ? 0x7FFFFFFFu : 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < kWords; ++i) m = DT == kF32 ? max(m, w[i] & 0x7FFFFFFFu) : __vmaxu2(m, w[i] & 0x7FFF7FFFu);
    return DT == kF32 ? m : max(m << 16, m & 0x7FFF0000u);
  }
};

// Rows off the 16-byte grid: a warp's R rows by 512 / R columns go through shared memory, so that neighbouring lanes touch neighbouring elements of the
// matrix (element by element where each lane needs its 16, a warp's access met 32 sectors: restoring 8192 x 4095 bf16 203 us).
template <int DT, int R>
struct LooseRows {
  static constexpr uint32_t kEsize = DT == kF32 ? 4u : 2u, kCols = 512u / R, kPitch = kCols * kEsize + 16u, kBytes = R * kPitch;
  using E = typename std::conditional<DT == kF32, uint32_t, uint16_t>::type;
  // Columns c0 ... of `rows` rows at p, `ld` elements apart, those below `cols`, zeros elsewhere: each lane gets the 16 of row lane % R, chunk lane / R.
  static __device__ __forceinline__ void load(Raw16<DT>& x, uint8_t* stage, const uint8_t* p, uint64_t ld, uint32_t rows, uint32_t c0, uint32_t cols, uint32_t lane) {
    E v[16];
#pragma unroll
    for (uint32_t i = 0; i < 16u; ++i) {
      const uint32_t at = i * 32u + lane, r = at / kCols, c = c0 + at % kCols;
      v[i] = r < rows && c < cols ? reinterpret_cast<const E*>(p)[r * ld + c] : (E)0;
    }
    __syncwarp();  // (what was read of the stage before has been)
#pragma unroll
    for (uint32_t i = 0; i < 16u; ++i) {
      const uint32_t at = i * 32u + lane;
      reinterpret_cast<E*>(stage + at / kCols * kPitch)[at % kCols] = v[i];
    }
    __syncwarp();
    x.template load<true>(stage + lane % R * kPitch + lane / R * 16u * kEsize, 16);
  }
  static __device__ __forceinline__ void store(const Raw16<DT>& x, uint8_t* stage, uint8_t* p, uint64_t ld, uint32_t rows, uint32_t c0, uint32_t cols, uint32_t lane) {
    __syncwarp();
    x.template store<true>(stage + lane % R * kPitch + lane / R * 16u * kEsize, 16);
    __syncwarp();
#pragma unroll
    for (uint32_t i = 0; i < 16u; ++i) {
      const uint32_t at = i * 32u + lane, r = at / kCols, c = c0 + at % kCols;
      if (r < rows && c < cols) reinterpret_cast<E*>(p)[r * ld + c] = reinterpret_cast<const E*>(stage + r * kPitch)[at % kCols];
    }
  }
};

}  // namespace fh
