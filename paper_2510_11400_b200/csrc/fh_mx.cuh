// Matrices in microscaled 4-bit floating point: the container's layout and the conversions, shared by the kernels that
// write containers (fh_mx_save.cu, fh_norm.cu) and those that read them (fh_mx_save.cu, fh_mx_product.cu, fh_norm.cu).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "fh_device.cuh"

namespace fh {

constexpr uint32_t kMxMagic = 0x344D4846u;  // "FHM4"
constexpr uint32_t kMxHeadBytes = 128;
constexpr int kMxB32 = 0, kMxB16 = 1;       // fh_mx_format
constexpr int kMxRows = 128;                // rows of a block of codes, and of a group of scales

// The container of a rows x cols matrix (fh.h describes it).
struct MxLayout {
  uint32_t rows, cols;
  uint32_t r8, kp;        // rows padded to 8, columns to 64: what codes are stored for
  uint32_t atoms;         // groups of four blocks along a row
  uint32_t format;
  uint64_t code_bytes, total;

  __host__ __device__ MxLayout() {}
  __host__ __device__ MxLayout(uint32_t rows_, uint32_t cols_, uint32_t format_) : rows(rows_), cols(cols_), format(format_) {
    r8 = (rows + 7u) & ~7u;
    kp = (cols + 63u) & ~63u;
    atoms = (kp / 32u * (format == kMxB32 ? 1u : 2u) + 3u) / 4u;
    code_bytes = (uint64_t)r8 * (kp / 2u);
    total = kMxHeadBytes + code_bytes + (uint64_t)((rows + 127u) / 128u) * atoms * 512u;
  }
  // Rows of codes that block b of 128 rows has.
  __host__ __device__ uint32_t block_rows(uint32_t b) const {
    const uint32_t left = r8 - b * 128u;
    return left < 128u ? left : 128u;
  }
  // The 16 bytes of the codes of columns 32 j ... 32 j + 31 of a row.
  __host__ __device__ uint64_t code_at(uint32_t row, uint32_t j) const {
    const uint32_t b = row / 128u;
    return kMxHeadBytes + (uint64_t)b * 128u * (kp / 2u) + ((uint64_t)j * block_rows(b) + row % 128u) * 16u;
  }
  // The 512 bytes of the scales of four blocks of 128 rows; row r's are the four bytes at scale_in_atom(r).
  __host__ __device__ uint64_t atom_at(uint32_t block, uint32_t atom) const {
    return kMxHeadBytes + code_bytes + ((uint64_t)block * atoms + atom) * 512u;
  }
  __host__ __device__ static uint32_t scale_in_atom(uint32_t row) { return row % 32u * 16u + row % 128u / 32u * 4u; }
};

struct MxHeader {
  uint32_t magic, kind;  // kind: version 1 | format << 16 | rounding << 24
  uint32_t rows, cols;
  int32_t exponent;
  uint32_t zero;
  uint64_t total, tensor_id;
  uint32_t pad[22];
};
static_assert(sizeof(MxHeader) == kMxHeadBytes, "MxHeader layout");

// Whether a container is the one expected, and its exponent.  (Rounding and tensor id do not matter to a reader.)
__device__ __forceinline__ bool mx_header_ok(const uint8_t* src, uint64_t src_bytes, const MxLayout& l, int32_t* exponent) {
  if (src_bytes < l.total) return false;  // (so that the header is there to be read)
  const uint4 a = *reinterpret_cast<const uint4*>(src), b = *reinterpret_cast<const uint4*>(src + 16);
  *exponent = (int32_t)b.x;
  return a.x == kMxMagic && (a.y & 0x00FFFFFFu) == (1u | l.format << 16) && a.z == l.rows && a.w == l.cols && b.y == 0u &&
         ((uint64_t)b.w << 32 | b.z) == l.total && (l.format == kMxB32 ? *exponent == 0 : *exponent >= -64 && *exponent <= 64);
}

__device__ __forceinline__ float bits_f(uint32_t u) { return __uint_as_float(u); }
// 2^k for -126 <= k <= 127.
__device__ __forceinline__ float pow2_f(int k) { return bits_f((uint32_t)(k + 127) << 23); }

// ---- scales ---------------------------------------------------------------------------------------
// What an element of a block is multiplied by before it is rounded to a code.
//  B32: x * 2^-k, exact.
//  B16: x * 2^-exponent / s for a scale s of four significant bits, as the sum of two products: hi, 1 / s rounded towards zero, and lo,
//  what hi lacks (not negative, so that a zero keeps its sign), so that rn(x * hi + rn(x * lo)) is the quotient to within 2^-46 ahead
//  of its last rounding.  That is enough: a
//  boundary m between two codes is a number of three bits, so m * s has seven, and a quotient whose x is not m * s lies at least
//  2^-24 (1 + 2^-7) away from m, relative: its rounding is on the same side, and m itself comes out where x = m * s.
struct MxScale {
  float hi, lo;   // factors (lo: B16 only)
  float s;        // the scale (B16: without 2^exponent; B32: unused)
  uint32_t byte;
  bool bad;       // the block holds a NaN or an infinity
};

// `top`: bit pattern of the block's largest magnitude.
template <int F>
__device__ __forceinline__ MxScale mx_scale(uint32_t top, float unscale) {
  MxScale r;
  r.bad = top >= 0x7F800000u;
  if (F == kMxB32) {
    // smallest k with 6 * 2^k = 1.5 * 2^(k + 2) >= top: the exponent of top less 2, one more when its mantissa is beyond 1.5
    int b = (int)((top + 0x3FFFFFu) >> 23) - 2;
    b = b < 0 ? 0 : (b > 252 ? 252 : b);
    r.byte = r.bad ? 255u : (uint32_t)b;
    r.hi = bits_f((uint32_t)(254 - b) << 23);
    r.lo = 0.0f;
    r.s = 0.0f;
  } else {
    // a sixth, rounded, and that rounded up to E4M3: t is on the right side of every E4M3 number v, as 6 v has at most six
    // bits, and the next fp32 number beyond it is a sixth of an ulp of 6 v away, at least 4/6 of an ulp of v
    const float t = __fdiv_rn(bits_f(top) * unscale, 6.0f);
    uint32_t c;
    if (t >= 0.015625f)
      c = ((__float_as_uint(t) + 0xFFFFFu) >> 20) - (120u << 3);
    else
      c = (uint32_t)ceilf(t * 512.0f);
    c = c < 1u ? 1u : (c > 126u ? 126u : c);
    r.s = c < 8u ? (float)c * 0.001953125f : bits_f((c + (120u << 3)) << 20);
    r.byte = r.bad ? 127u : c;
    const float hi = __frcp_rz(r.s);
    r.lo = __fmaf_rn(-hi, r.s, 1.0f) * hi * unscale;
    r.hi = hi * unscale;
  }
  return r;
}

template <int F>
__device__ __forceinline__ float mx_quotient(float x, const MxScale& s) {
  return F == kMxB32 ? x * s.hi : __fmaf_rn(x, s.hi, x * s.lo);
}

// Random rounding (of finite x with quotients below 2^105): x between two neighbouring magnitudes L and L + step (times the scale) goes up when what it is beyond L is
// more than (r + 1/2) / 2^16 of the step, r a uniform 16-bit integer; exact, as the left side is an fp32 number and the right
// side has at most 17 + 4 bits.  Leaves the magnitude with x's sign.  `draw`: bits of 1 + r / 2^16; `s_full`: the
// scale with 2^exponent (B16; exact, as x is then compared as it is).
// (The step comes from the exponent, L from an addition that rounds down at 2^23 steps: no conversions, which take a scheduler four
// times as long; two elements to an instruction.  8192 x 4096 both ways: 125 us with one element to an instruction and conversions.)
__device__ __forceinline__ f32x2 add2_down(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rm.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
template <int F>
__device__ __forceinline__ void mx_random2(float& x0, float& x1, const MxScale& s, float s_full, uint32_t draw0, uint32_t draw1) {
  const f32x2 x = pack2(fabsf(x0), fabsf(x1)), hi = pack2(s.hi, s.hi), less = pack2(-1.0f, -1.0f);
  const f32x2 u = F == kMxB32 ? mul2(x, hi) : fma2(x, hi, mul2(x, pack2(s.lo, s.lo)));
  uint32_t u0, u1;
  unpack2u(u, u0, u1);
  const uint32_t b0 = (max(u0, 0x3F800000u) & 0x7F800000u) - 0x00800000u, b1 = (max(u1, 0x3F800000u) & 0x7F800000u) - 0x00800000u;
  const f32x2 step = pack2(bits_f(b0), bits_f(b1)), at = pack2(bits_f(b0 + (23u << 23)), bits_f(b1 + (23u << 23)));
  const f32x2 low = fma2(less, at, add2_down(u, at)), high = add2(low, step);
  const f32x2 part = mul2(add2(pack2(bits_f(draw0), bits_f(draw1)), pack2(-0.99999237060546875f, -0.99999237060546875f)), step);
  const f32x2 rest = F == kMxB32 ? fma2(less, low, u) : fma2(low, pack2(-s_full, -s_full), x);
  const f32x2 most = F == kMxB32 ? part : mul2(part, pack2(s_full, s_full));
  float r0, r1, m0, m1, l0, l1, h0, h1;
  unpack2(rest, r0, r1);
  unpack2(most, m0, m1);
  unpack2(low, l0, l1);
  unpack2(high, h0, h1);
  x0 = copysignf(r0 > m0 ? h0 : l0, x0);
  x1 = copysignf(r1 > m1 ? h1 : l1, x1);
}

// Eight values to codes, the first in the lowest bits: round to nearest, ties to even, beyond 6 is 6.
__device__ __forceinline__ uint32_t mx_codes8(const float (&v)[8]) {
  uint32_t r;
  asm("{ .reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d}; }"
      : "=r"(r)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}

// Eight codes to values, by way of fp16, which holds them: exact.
__device__ __forceinline__ void mx_values8(uint32_t codes, float (&v)[8]) {
  uint32_t h[4];
  asm("{ .reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d; }"
      : "=&r"(h[0]), "=&r"(h[1]), "=&r"(h[2]), "=&r"(h[3])
      : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
    v[2 * i] = p.x;
    v[2 * i + 1] = p.y;
  }
}

// Four codes (the low 16 bits) to values: the upper two bytes of an fp32 number picked from tables of the eight magnitudes, and the
// sign.  (With the conversion instruction on the lower two of a word's four bytes and the upper two unused, the upper two's values came
// out; why was not found.)
__device__ __forceinline__ void mx_values4(uint32_t codes, float (&v)[4]) {
  const uint32_t m = codes & 0x7777u;
  const uint32_t hi = __byte_perm(0x3F3F3F00u, 0x40404040u, m), lo = __byte_perm(0xC0800000u, 0xC0804000u, m);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    v[e] = bits_f((__byte_perm(lo, hi, (uint32_t)((4 + e) << 12 | e << 8)) & 0xFFFF0000u) | (codes << (28 - 4 * e) & 0x80000000u));
}

// A scale byte as a factor; `scale`: 2^exponent (B16).
template <int F>
__device__ __forceinline__ float mx_factor(uint32_t byte, float scale) {
  if (F == kMxB32) {
    // 2^(byte - 127): byte 0 is half the smallest normal number, byte 255 a NaN
    return bits_f(byte == 255u ? 0x7FC00000u : max(byte << 23, 0x00400000u));
  }
  const float v = byte < 8u ? (float)byte * 0.001953125f : bits_f((byte + (120u << 3)) << 20);
  return (byte & 127u) == 127u ? bits_f(0x7FC00000u) : v * scale;
}

}  // namespace fh
