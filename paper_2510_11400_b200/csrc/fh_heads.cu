// Norms of queries and keys for each head with the rotation by position, forward and backward.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "fh_i8_launch.cuh"
#include "fh_launch.cuh"

namespace fh {
namespace {

constexpr int kHeadThreads = 128;
constexpr uint32_t kHeadWarps = kHeadThreads / 32;

template <int DT>
constexpr uint32_t kEs = DT == kF32 ? 4u : 2u;
template <int DT>
constexpr uint32_t kV = 16u / kEs<DT>;  // elements of a 16-byte vector

// Memory bounds both passes: a row of a head is read and written once.  Nothing is kept between them: the backward pass has the row in registers
// and makes its mean and rstd again, which costs less than reading them.
//
// A slot is two vectors of 16 bytes that hold both elements of their pairs: a vector of the first half and its partner of the second, or two neighbouring
// vectors; where a part of a head is not rotated, it is made of slots too, whose angle is zero.  A team of T lanes has a row, a slot to a lane, so
// that a row needs no exchange but its sums', and a lane's cosines, sines and weights stay in registers from head to head of a token.
template <int DT>
struct Slot {
  uint32_t a, b;   // first element of its two vectors
  uint32_t pair;   // its first pair in the table
  bool there, turned;
  __device__ __forceinline__ Slot(uint32_t s, uint32_t dim, uint32_t rotary, bool halves) {
    constexpr uint32_t V = kV<DT>;
    there = s < dim / (2u * V);
    turned = s < rotary / (2u * V);
    pair = s * V;
    if (!halves) {
      a = 2u * V * s;
      b = a + V;
    } else if (turned) {
      a = V * s;
      b = rotary / 2u + a;
    } else {
      a = rotary + V * (s - rotary / (2u * V));
      b = a + (dim - rotary) / 2u;
    }
  }
};

// The values of a 16-byte vector.
template <int DT>
__device__ __forceinline__ void vec_values(const uint4& w, float* v) {
  if (DT == kF32) {
    v[0] = __uint_as_float(w.x);
    v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z);
    v[3] = __uint_as_float(w.w);
  } else {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
}
// A slot of a row as it is in memory (as values it would take twice the registers in bf16, of which there are several rows at once).
struct RawSlot {
  uint4 a, b;
  __device__ __forceinline__ void zero() { a = b = make_uint4(0u, 0u, 0u, 0u); }
  template <int DT>
  __device__ __forceinline__ void load(const uint8_t* p, uint32_t at, uint32_t bt) {
    a = *reinterpret_cast<const uint4*>(p + at * kEs<DT>);
    b = *reinterpret_cast<const uint4*>(p + bt * kEs<DT>);
  }
  template <int DT>
  __device__ __forceinline__ void values(float (&v)[2 * kV<DT>]) const {
    vec_values<DT>(a, v);
    vec_values<DT>(b, v + kV<DT>);
  }
};
template <int DT>
__device__ __forceinline__ void store_vec(uint8_t* p, const float* v) {
  uint4 w;
  if (DT == kF32)
    w = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
  else
    w = make_uint4(f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3]), f32x2_to_bf16x2(v[4 % kV<DT>], v[5 % kV<DT>]), f32x2_to_bf16x2(v[6 % kV<DT>], v[7 % kV<DT>]));
  *reinterpret_cast<uint4*>(p) = w;
}
__device__ __forceinline__ float weight_at(const uint8_t* gamma, int wdtype, uint32_t i) {
  if (!gamma) return 1.0f;
  return wdtype == kF32 ? reinterpret_cast<const float*>(gamma)[i] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(gamma)[i]);
}
// The weights of a slot.
template <int DT>
__device__ __forceinline__ void load_weights(const uint8_t* gamma, const HeadsArgs& g, uint32_t a, uint32_t b, float (&w)[2 * kV<DT>]) {
  constexpr uint32_t V = kV<DT>;
  if (gamma && (uintptr_t)gamma % 16u == 0u && g.wdtype == kF32) {
#pragma unroll
    for (uint32_t e = 0; e < 2 * V; e += 4) vec_values<kF32>(*reinterpret_cast<const uint4*>(gamma + ((e < V ? a : b - V) + e) * 4u), w + e);
  } else if (gamma && (uintptr_t)gamma % 16u == 0u && DT == kBF16) {
#pragma unroll
    for (uint32_t e = 0; e < 2 * V; e += 8) vec_values<kBF16>(*reinterpret_cast<const uint4*>(gamma + ((e < V ? a : b - V) + e) * 2u), w + e % (2 * V));
  } else {
#pragma unroll
    for (uint32_t e = 0; e < 2 * V; ++e) w[e] = weight_at(gamma, g.wdtype, (e < V ? a : b - V) + e);
  }
}
template <int DT>
__device__ __forceinline__ float elem_at(const uint8_t* p, uint32_t i) {
  return DT == kF32 ? reinterpret_cast<const float*>(p)[i] : bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(p)[i]);
}
template <int DT>
__device__ __forceinline__ void put_elem(uint8_t* p, uint32_t i, float v) {
  if (DT == kF32)
    reinterpret_cast<float*>(p)[i] = v;
  else
    reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_bits(v);
}

// Sum over the T lanes of a team (all lanes of the warp take part).
template <int T>
__device__ __forceinline__ float team_sum(float v) {
#pragma unroll
  for (int s = 1; s < T; s *= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, s);
  return v;
}

// The pairs of a slot: `first` and `second` of pair i of its V pairs among its 2 V elements.
template <bool HALVES, uint32_t V>
__device__ __forceinline__ constexpr uint32_t first_of(uint32_t i) { return HALVES ? i : 2 * i; }
template <bool HALVES, uint32_t V>
__device__ __forceinline__ constexpr uint32_t second_of(uint32_t i) { return HALVES ? V + i : 2 * i + 1; }

// A token's position: -1 for one that is left out.
__device__ __forceinline__ int32_t position_of(const HeadsArgs& g, uint32_t token) {
  if (g.rotary == 0u) return 0;
  if (!g.at) return (int32_t)token;  // (the host has seen that the table has them all)
  const int32_t p = g.at[token];
  return (uint32_t)p >= g.positions ? -1 : p;
}
// The status, by one CTA that does nothing else (the others' order is not known).
__device__ __forceinline__ void report_positions(const HeadsArgs& g) {
  __shared__ uint32_t bad;
  if (threadIdx.x == 0) bad = 0u;
  __syncthreads();
  bool mine = false;
  if (g.at && g.rotary) {
#pragma unroll 16
    for (uint32_t t = threadIdx.x; t < g.tokens; t += blockDim.x) mine |= (uint32_t)g.at[t] >= g.positions;
  }
  if (mine) bad = 1u;
  __syncthreads();
  if (threadIdx.x == 0) *g.status = bad ? status_word(kErrCorrupt) : 0ull;
}

// Cosines and sines of a slot's pairs at a position.
template <int DT>
__device__ __forceinline__ void load_turn(const HeadsArgs& g, const Slot<DT>& s, int32_t at, float (&c)[kV<DT>], float (&n)[kV<DT>]) {
  if (s.turned) {
    const float4* p = reinterpret_cast<const float4*>(g.table + (uint64_t)at * (g.rotary / 2u) + s.pair);
#pragma unroll
    for (uint32_t i = 0; i < kV<DT> / 2u; ++i) {
      const float4 v = p[i];
      c[2 * i] = v.x;
      n[2 * i] = v.y;
      c[2 * i + 1] = v.z;
      n[2 * i + 1] = v.w;
    }
  } else {
#pragma unroll
    for (uint32_t i = 0; i < kV<DT>; ++i) {
      c[i] = 1.0f;
      n[i] = 0.0f;
    }
  }
}

// Two elements to an instruction: instructions bound the bf16 kernels as much as memory does.
__device__ __forceinline__ f32x2 twice(float x) { return pack2(x, x); }
__device__ __forceinline__ float sum2(f32x2 v) {
  float a, b;
  unpack2(v, a, b);
  return a + b;
}
// First and second elements of the V pairs of a slot.
template <bool HALVES, uint32_t V>
__device__ __forceinline__ void split(const float (&x)[2 * V], f32x2 (&a)[V / 2], f32x2 (&b)[V / 2]) {
#pragma unroll
  for (uint32_t p = 0; p < V; p += 2) {
    a[p / 2] = pack2(x[first_of<HALVES, V>(p)], x[first_of<HALVES, V>(p + 1)]);
    b[p / 2] = pack2(x[second_of<HALVES, V>(p)], x[second_of<HALVES, V>(p + 1)]);
  }
}
template <bool HALVES, uint32_t V>
__device__ __forceinline__ void join(const f32x2 (&a)[V / 2], const f32x2 (&b)[V / 2], float (&x)[2 * V]) {
#pragma unroll
  for (uint32_t p = 0; p < V; p += 2) {
    unpack2(a[p / 2], x[first_of<HALVES, V>(p)], x[first_of<HALVES, V>(p + 1)]);
    unpack2(b[p / 2], x[second_of<HALVES, V>(p)], x[second_of<HALVES, V>(p + 1)]);
  }
}

// Row `u` of all: whether it is of queries or keys, its token and its head.
struct HeadUnit {
  uint32_t side, token, head;
  __device__ __forceinline__ HeadUnit(uint64_t u, const HeadsArgs& g) {
    const uint32_t nq = g.side[0].heads, n = nq + g.side[1].heads;
    // (a division in 64 bits takes as long as a row)
    token = u >> 32 ? (uint32_t)(u / n) : (uint32_t)u / n;
    const uint32_t at = (uint32_t)(u - (uint64_t)token * n);
    side = at >= nq;
    head = side ? at - nq : at;
  }
};

template <int DT>
__device__ __forceinline__ const uint8_t* row_of(const HeadsSide& s, uint32_t token, uint32_t head) {
  return s.x + ((uint64_t)token * s.token + (uint64_t)head * s.head) * kEs<DT>;
}
template <int DT>
__device__ __forceinline__ uint64_t out_at(const HeadsSide& s, uint32_t token, uint32_t head) {
  return ((uint64_t)token * s.out_token + (uint64_t)head * s.out_head) * kEs<DT>;
}

// T lanes to a row.  A team takes U heads of a token at once, which are asked for together and share what the token and the side have; the teams of a warp go on
// where their neighbours end, at the next heads or the next tokens.
template <int DT, int T, int U, bool HALVES>
__global__ void __launch_bounds__(kHeadThreads) heads_forward_kernel(const HeadsArgs g) {
  constexpr uint32_t V = kV<DT>, kTeams = 32 / T;
  dep_trigger();
  dep_wait();
  const uint32_t extra = g.status ? 1u : 0u;
  if (blockIdx.x < extra) {
    report_positions(g);
    return;
  }
  const uint32_t cta = blockIdx.x - extra, which = cta >= g.side[0].parts, lane = threadIdx.x % 32;
  const HeadsSide& s = g.side[which];
  const uint32_t blocks = (s.heads + U - 1u) / U;
  const uint64_t units = (uint64_t)g.tokens * blocks, u = ((uint64_t)(cta - (which ? g.side[0].parts : 0u)) * kHeadWarps + threadIdx.x / 32) * kTeams + lane / T;
  // (a division in 64 bits takes as long as a row)
  const uint32_t token = u >> 32 ? (uint32_t)(u / blocks) : (uint32_t)u / blocks, head0 = (uint32_t)(u - (uint64_t)token * blocks) * U;
  const Slot<DT> slot(lane % T, g.dim, g.rotary, HALVES);
  RawSlot raw[U];
  bool there[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    there[i] = slot.there && u < units && head0 + i < s.heads;
    raw[i].zero();
    if (there[i]) raw[i].load<DT>(row_of<DT>(s, token, head0 + i), slot.a, slot.b);
  }
  float c[V], n[V], w[2 * V];
  if (slot.there) load_weights<DT>(s.gamma, g, slot.a, slot.b, w);
  const int32_t at = u < units ? position_of(g, token) : -1;
  if (slot.there && at >= 0) load_turn<DT>(g, slot, at, c, n);
  // weights and rotation as one factor each: y = rstd (xa (wa c) - xb (wb n)), rstd (xb (wb c) + xa (wa n))
  f32x2 ac[V / 2], an[V / 2], bc[V / 2], bn[V / 2];
  {
    f32x2 wa[V / 2], wb[V / 2];
    split<HALVES, V>(w, wa, wb);
#pragma unroll
    for (uint32_t p = 0; p < V / 2; ++p) {
      const f32x2 cc = pack2(c[2 * p], c[2 * p + 1]), nn = pack2(n[2 * p], n[2 * p + 1]), minus = pack2(-n[2 * p], -n[2 * p + 1]);
      ac[p] = mul2(wa[p], cc);
      an[p] = mul2(wa[p], nn);
      bc[p] = mul2(wb[p], cc);
      bn[p] = mul2(wb[p], minus);
    }
  }
  const float size = (float)g.dim, part = 1.0f / size;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (i && !__any_sync(0xFFFFFFFFu, there[i])) break;
    float x[2 * V];
    raw[i].values<DT>(x);
    f32x2 a[V / 2], b[V / 2];
    split<HALVES, V>(x, a, b);
    if (g.layer) {
      f32x2 sum = add2(a[0], b[0]);
#pragma unroll
      for (uint32_t p = 1; p < V / 2; ++p) sum = add2(sum, add2(a[p], b[p]));
      const float mean = __fdiv_rn(team_sum<T>(sum2(sum)), size);
      const f32x2 less = twice(slot.there ? -mean : 0.0f);
#pragma unroll
      for (uint32_t p = 0; p < V / 2; ++p) {
        a[p] = add2(a[p], less);
        b[p] = add2(b[p], less);
      }
    }
    f32x2 sum = mul2(a[0], a[0]);
#pragma unroll
    for (uint32_t p = 0; p < V / 2; ++p) {
      if (p) sum = fma2(a[p], a[p], sum);
      sum = fma2(b[p], b[p], sum);
    }
    const f32x2 rstd = twice(rsqrtf(__fmaf_rn(team_sum<T>(sum2(sum)), part, g.eps)));
    f32x2 ya[V / 2], yb[V / 2];
#pragma unroll
    for (uint32_t p = 0; p < V / 2; ++p) {
      const f32x2 sa = mul2(a[p], rstd), sb = mul2(b[p], rstd);
      ya[p] = fma2(sa, ac[p], mul2(sb, bn[p]));
      yb[p] = fma2(sb, bc[p], mul2(sa, an[p]));
    }
    join<HALVES, V>(ya, yb, x);
    if (there[i] && at >= 0) {
      uint8_t* o = s.out + out_at<DT>(s, token, head0 + i);
      store_vec<DT>(o + slot.a * kEs<DT>, x);
      store_vec<DT>(o + slot.b * kEs<DT>, x + V);
    }
  }
}

// Backward.  CTAs are dealt out to queries and keys, and each adds up its rows' part of the weights' gradient: a lane for its slot, then teams, then warps,
// in a fixed order.  A team's next row is asked for while it works on one.  (16384 tokens of 32 + 8 heads of 128 in bf16: 108 us with registers for four CTAs
// an SM, 127 for three; in fp32 8192 of 16 + 16: 73 for five, 77 for four.  Before, in bf16: two rows of a team at once and none ahead 140; a ring in shared
// memory filled by asynchronous copies 156 to 204, as its addresses and second reads cost more than they hid.)
template <int DT>
constexpr uint32_t kBackCtas = DT == kF32 ? 5 : 4;
template <int DT, int T, bool HALVES>
__global__ void __launch_bounds__(kHeadThreads, kBackCtas<DT>) heads_backward_kernel(const HeadsArgs g) {
  constexpr uint32_t V = kV<DT>, kTeams = 32 / T;
  __shared__ float sums[kHeadWarps][T * 2 * V];
  dep_trigger();
  dep_wait();
  const uint32_t extra = g.status ? 1u : 0u;
  if (blockIdx.x < extra) {
    report_positions(g);
    return;
  }
  const uint32_t cta = blockIdx.x - extra, which = cta >= g.side[0].parts, part = which ? cta - g.side[0].parts : cta;
  const HeadsSide& s = g.side[which];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, team = lane / T;
  const Slot<DT> slot(lane % T, g.dim, g.rotary, HALVES);
  const float size = (float)g.dim, share = 1.0f / size;
  f32x2 wa[V / 2], wb[V / 2], sa[V / 2], sb[V / 2];
  {
    float w[2 * V] = {};
    if (slot.there) load_weights<DT>(s.gamma, g, slot.a, slot.b, w);
    split<HALVES, V>(w, wa, wb);
#pragma unroll
    for (uint32_t p = 0; p < V / 2; ++p) sa[p] = sb[p] = 0ull;
  }
  // Each team's rows are neighbours, so that a token's position, cosines and sines serve several heads.
  const uint64_t rows = (uint64_t)g.tokens * s.heads, teams = (uint64_t)s.parts * kHeadWarps * kTeams, me = ((uint64_t)part * kHeadWarps + warp) * kTeams + team;
  const uint64_t each = rows / teams, over = rows % teams, first = each * me + (me < over ? me : over);
  const uint32_t count = (uint32_t)each + (me < over ? 1u : 0u), most = (uint32_t)each + (over ? 1u : 0u);
  uint32_t token = (uint32_t)(first / s.heads), head = (uint32_t)(first % s.heads);
  RawSlot nx, ny;
  auto ask = [&](bool more) {
    nx.zero();
    ny.zero();
    if (slot.there && more) {
      nx.load<DT>(row_of<DT>(s, token, head), slot.a, slot.b);
      ny.load<DT>(s.dy + out_at<DT>(s, token, head), slot.a, slot.b);
    }
  };
  ask(count != 0u);
  int32_t at = count ? position_of(g, token) : -1, next_at = at;
  bool fresh = true;
  f32x2 c[V / 2], n[V / 2];
#pragma unroll
  for (uint32_t p = 0; p < V / 2; ++p) c[p] = n[p] = 0ull;
  for (uint32_t k = 0; k < most; ++k) {  // (all teams of a warp as often)
    const RawSlot rx = nx, ry = ny;
    const uint32_t now = token, row = head;
    if (fresh && at >= 0 && slot.there) {
      float fc[V], fn[V];
      load_turn<DT>(g, slot, at, fc, fn);
#pragma unroll
      for (uint32_t p = 0; p < V / 2; ++p) {
        c[p] = pack2(fc[2 * p], fc[2 * p + 1]);
        n[p] = pack2(fn[2 * p], fn[2 * p + 1]);
      }
    }
    const bool there = slot.there && k < count && at >= 0;
    fresh = false;
    if (++head == s.heads) {
      head = 0;
      ++token;
      fresh = true;
    }
    ask(k + 1u < count);
    if (fresh && k + 1u < count) next_at = position_of(g, token);
    at = next_at;
    f32x2 xa[V / 2], xb[V / 2], da[V / 2], db[V / 2];
    {
      float v[2 * V];
      rx.values<DT>(v);
      split<HALVES, V>(v, xa, xb);
      ry.values<DT>(v);
      split<HALVES, V>(v, da, db);
    }
    if (g.layer) {
      f32x2 sum = add2(xa[0], xb[0]);
#pragma unroll
      for (uint32_t p = 1; p < V / 2; ++p) sum = add2(sum, add2(xa[p], xb[p]));
      const float mean = __fdiv_rn(team_sum<T>(sum2(sum)), size);
      const f32x2 less = twice(there ? -mean : 0.0f);
#pragma unroll
      for (uint32_t p = 0; p < V / 2; ++p) {
        xa[p] = add2(xa[p], less);
        xb[p] = add2(xb[p], less);
      }
    }
    // dz in da and db, then the sums of x^2, g x and g (of a slot that is not there everything is zero)
    f32x2 xx = 0ull, gx = 0ull, gs = 0ull;
#pragma unroll
    for (uint32_t p = 0; p < V / 2; ++p) {
      const f32x2 ya = da[p], yb = db[p];
      da[p] = fma2(ya, c[p], mul2(yb, n[p]));
      db[p] = fma2(mul2(ya, n[p]), twice(-1.0f), mul2(yb, c[p]));
      const f32x2 ga = mul2(da[p], wa[p]), gb = mul2(db[p], wb[p]);
      xx = fma2(xb[p], xb[p], fma2(xa[p], xa[p], xx));
      gx = fma2(gb, xb[p], fma2(ga, xa[p], gx));
      if (g.layer) gs = add2(gs, add2(ga, gb));
    }
    const float sxx = team_sum<T>(sum2(xx)), sgx = team_sum<T>(sum2(gx)), sgs = g.layer ? team_sum<T>(sum2(gs)) : 0.0f;
    const float rstd = rsqrtf(__fmaf_rn(sxx, share, g.eps));
    // dx = rstd (g - x rstd mean(g xhat) - mean(g))
    const f32x2 r = twice(rstd), along = twice(-(sgx * rstd * share) * rstd), level = twice(-(sgs * share));
#pragma unroll
    for (uint32_t p = 0; p < V / 2; ++p) {
      if (there) {  // (a row without elements has no rstd where eps is 0)
        sa[p] = fma2(da[p], mul2(xa[p], r), sa[p]);
        sb[p] = fma2(db[p], mul2(xb[p], r), sb[p]);
      }
      da[p] = mul2(r, add2(fma2(xa[p], along, mul2(da[p], wa[p])), level));
      db[p] = mul2(r, add2(fma2(xb[p], along, mul2(db[p], wb[p])), level));
    }
    if (there && s.dx) {
      float v[2 * V];
      join<HALVES, V>(da, db, v);
      uint8_t* o = s.dx + ((uint64_t)now * s.token + (uint64_t)row * s.head) * kEs<DT>;
      store_vec<DT>(o + slot.a * kEs<DT>, v);
      store_vec<DT>(o + slot.b * kEs<DT>, v + V);
    }
  }
  if (!s.dgamma) return;
  float acc[2 * V];
  join<HALVES, V>(sa, sb, acc);
#pragma unroll
  for (uint32_t e = 0; e < 2 * V; ++e) {
#pragma unroll
    for (int o = T; o < 32; o *= 2) acc[e] += __shfl_xor_sync(0xFFFFFFFFu, acc[e], o);
    if (team == 0) sums[warp][(lane % T) * 2 * V + e] = acc[e];
  }
  __syncthreads();
  float* out = g.work + (uint64_t)((which ? g.side[0].parts : 0u) + part) * g.dim;
  for (uint32_t i = threadIdx.x; i < T * 2 * V; i += kHeadThreads) {
    const Slot<DT> of(i / (2 * V), g.dim, g.rotary, HALVES);
    const uint32_t e = i % (2 * V);
    float sum = 0.0f;
#pragma unroll
    for (uint32_t x = 0; x < kHeadWarps; ++x) sum += sums[x][i];
    if (of.there) out[(e < V ? of.a : of.b - V) + e] = sum;
  }
}

// ---- any size, stride and alignment: a warp to a row, a lane to pairs 32 apart.  What is not rotated is taken in pairs too (the last element of an odd
// number alone), whose angle is zero.  N pairs of a lane stay in registers; N = 0: the row is too long for that, and its elements are read again from L1.
struct LoosePair {
  uint32_t a, b;
  bool turned, two;  // whether the table has it, and whether it has a second element
};
template <bool HALVES>
__device__ __forceinline__ LoosePair loose_pair(const HeadsArgs& g, uint32_t i) {
  const uint32_t half = g.rotary / 2u;
  LoosePair p;
  p.turned = i < half;
  if (!HALVES) {
    p.a = 2u * i;
    p.b = p.a + 1u;
    p.two = p.b < g.dim;
  } else if (p.turned) {
    p.a = i;
    p.b = half + i;
    p.two = true;
  } else {
    const uint32_t rest = (g.dim - g.rotary) / 2u, at = i - half;
    p.two = at < rest;
    p.a = p.two ? g.rotary + at : g.dim - 1u;
    p.b = g.rotary + rest + at;
  }
  return p;
}
__device__ __forceinline__ uint32_t loose_pairs(const HeadsArgs& g) { return (g.dim + 1u) / 2u; }

// Where a lane's pairs are, with their weights: N of them.
template <int N, bool HALVES>
struct LooseLane {
  LoosePair p[N];
  bool there[N];
  float wa[N], wb[N];
  __device__ __forceinline__ LooseLane(const HeadsArgs& g, const uint8_t* gamma, uint32_t lane) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t i = lane + 32u * j;
      there[j] = i < loose_pairs(g);
      p[j] = loose_pair<HALVES>(g, i);
      p[j].two = p[j].two && there[j];
      wa[j] = there[j] ? weight_at(gamma, g.wdtype, p[j].a) : 0.0f;
      wb[j] = p[j].two ? weight_at(gamma, g.wdtype, p[j].b) : 0.0f;
    }
  }
  template <int DT>
  __device__ __forceinline__ void load(const uint8_t* x, float (&a)[N], float (&b)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      a[j] = there[j] ? elem_at<DT>(x, p[j].a) : 0.0f;
      b[j] = p[j].two ? elem_at<DT>(x, p[j].b) : 0.0f;
    }
  }
  __device__ __forceinline__ void less(float mean, float (&a)[N], float (&b)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      a[j] = there[j] ? a[j] - mean : 0.0f;
      b[j] = p[j].two ? b[j] - mean : 0.0f;
    }
  }
  __device__ __forceinline__ void turns(const HeadsArgs& g, int32_t at, uint32_t lane, float2 (&t)[N]) const {
#pragma unroll
    for (int j = 0; j < N; ++j) t[j] = there[j] && p[j].turned ? g.table[(uint64_t)at * (g.rotary / 2u) + lane + 32u * j] : make_float2(1.0f, 0.0f);
  }
};
template <int N>
__device__ __forceinline__ float sum_both(const float (&a)[N], const float (&b)[N]) {
  float s = 0.0f;
#pragma unroll
  for (int j = 0; j < N; ++j) s += a[j] + b[j];
  return s;
}

template <int DT>
__device__ __forceinline__ float loose_mean(const HeadsArgs& g, const uint8_t* p, uint32_t lane) {
  if (!g.layer) return 0.0f;
  float sum = 0.0f;
  for (uint32_t e = lane; e < g.dim; e += 32u) sum += elem_at<DT>(p, e);
  return __fdiv_rn(team_sum<32>(sum), (float)g.dim);
}

template <int DT, int N, bool HALVES>
__global__ void __launch_bounds__(kHeadThreads) heads_forward_loose_kernel(const HeadsArgs g) {
  dep_trigger();
  dep_wait();
  const uint32_t extra = g.status ? 1u : 0u;
  if (blockIdx.x < extra) {
    report_positions(g);
    return;
  }
  const uint32_t lane = threadIdx.x % 32;
  const uint64_t units = (uint64_t)g.tokens * (g.side[0].heads + g.side[1].heads);
  const uint64_t u = (uint64_t)(blockIdx.x - extra) * kHeadWarps + threadIdx.x / 32;
  if (u >= units) return;
  const HeadUnit unit(u, g);
  const HeadsSide& s = g.side[unit.side];
  const uint8_t* p = s.x + ((uint64_t)unit.token * s.token + (uint64_t)unit.head * s.head) * kEs<DT>;
  uint8_t* o = s.out + ((uint64_t)unit.token * s.out_token + (uint64_t)unit.head * s.out_head) * kEs<DT>;
  const float size = (float)g.dim;
  if constexpr (N > 0) {
    const LooseLane<N, HALVES> my(g, s.gamma, lane);
    float a[N], b[N];
    my.template load<DT>(p, a, b);
    const int32_t at = position_of(g, unit.token);
    if (at < 0) return;
    float2 t[N];
    my.turns(g, at, lane, t);
    if (g.layer) my.less(__fdiv_rn(team_sum<32>(sum_both(a, b)), size), a, b);
    float sum = 0.0f;
#pragma unroll
    for (int j = 0; j < N; ++j) sum = __fmaf_rn(b[j], b[j], __fmaf_rn(a[j], a[j], sum));
    const float rstd = 1.0f / sqrtf(__fdiv_rn(team_sum<32>(sum), size) + g.eps);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float za = a[j] * rstd * my.wa[j], zb = b[j] * rstd * my.wb[j];
      if (my.there[j]) put_elem<DT>(o, my.p[j].a, __fmaf_rn(za, t[j].x, -(zb * t[j].y)));
      if (my.p[j].two) put_elem<DT>(o, my.p[j].b, __fmaf_rn(zb, t[j].x, za * t[j].y));
    }
  } else {
    const int32_t at = position_of(g, unit.token);
    if (at < 0) return;
    const float2* turn = g.table + (uint64_t)at * (g.rotary / 2u);
    const float mean = loose_mean<DT>(g, p, lane);
    float sum = 0.0f;
    for (uint32_t e = lane; e < g.dim; e += 32u) {
      const float v = elem_at<DT>(p, e) - mean;
      sum = __fmaf_rn(v, v, sum);
    }
    const float rstd = 1.0f / sqrtf(__fdiv_rn(team_sum<32>(sum), size) + g.eps);
    __syncwarp();  // (in place, the row has been read by all lanes before one of them writes)
    for (uint32_t i = lane; i < loose_pairs(g); i += 32u) {
      const LoosePair q = loose_pair<HALVES>(g, i);
      const float za = (elem_at<DT>(p, q.a) - mean) * rstd * weight_at(s.gamma, g.wdtype, q.a);
      const float zb = q.two ? (elem_at<DT>(p, q.b) - mean) * rstd * weight_at(s.gamma, g.wdtype, q.b) : 0.0f;
      const float2 t = q.turned ? turn[i] : make_float2(1.0f, 0.0f);
      put_elem<DT>(o, q.a, __fmaf_rn(za, t.x, -(zb * t.y)));
      if (q.two) put_elem<DT>(o, q.b, __fmaf_rn(zb, t.x, za * t.y));
    }
  }
}

// Warps of a CTA each have sums of their own, `dim` floats in shared memory: while they work where N = 0, at the end otherwise.
template <int DT, int N, bool HALVES>
__global__ void __launch_bounds__(kHeadThreads) heads_backward_loose_kernel(const HeadsArgs g) {
  extern __shared__ float loose_sums[];
  dep_trigger();
  dep_wait();
  const uint32_t extra = g.status ? 1u : 0u;
  if (blockIdx.x < extra) {
    report_positions(g);
    return;
  }
  const uint32_t cta = blockIdx.x - extra, which = cta >= g.side[0].parts, part = which ? cta - g.side[0].parts : cta;
  const HeadsSide& s = g.side[which];
  const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
  float* acc = loose_sums + (uint64_t)warp * g.dim;
  const float size = (float)g.dim;
  const uint64_t units = (uint64_t)g.tokens * s.heads, first = (uint64_t)part * warps + warp, step = (uint64_t)s.parts * warps;
  if constexpr (N > 0) {
    const LooseLane<N, HALVES> my(g, s.gamma, lane);
    float sa[N] = {}, sb[N] = {};
#pragma unroll 2
    for (uint64_t u = first; u < units; u += step) {
      const uint32_t token = (uint32_t)(u / s.heads), head = (uint32_t)(u % s.heads);
      float a[N], b[N], ya[N], yb[N];
      my.template load<DT>(s.x + ((uint64_t)token * s.token + (uint64_t)head * s.head) * kEs<DT>, a, b);
      my.template load<DT>(s.dy + ((uint64_t)token * s.out_token + (uint64_t)head * s.out_head) * kEs<DT>, ya, yb);
      const int32_t at = position_of(g, token);
      if (at < 0) continue;
      float2 t[N];
      my.turns(g, at, lane, t);
      if (g.layer) my.less(__fdiv_rn(team_sum<32>(sum_both(a, b)), size), a, b);
      float xx = 0.0f, gx = 0.0f, gs = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float da = __fmaf_rn(ya[j], t[j].x, yb[j] * t[j].y), db = __fmaf_rn(yb[j], t[j].x, -(ya[j] * t[j].y));
        ya[j] = da;
        yb[j] = db;
        const float ga = da * my.wa[j], gb = db * my.wb[j];
        xx = __fmaf_rn(b[j], b[j], __fmaf_rn(a[j], a[j], xx));
        gx = __fmaf_rn(gb, b[j], __fmaf_rn(ga, a[j], gx));
        gs += ga + gb;
      }
      xx = team_sum<32>(xx);
      gx = team_sum<32>(gx);
      if (g.layer) gs = team_sum<32>(gs);
      const float rstd = 1.0f / sqrtf(__fdiv_rn(xx, size) + g.eps);
      const float along = gx * rstd / size, level = g.layer ? gs / size : 0.0f;
      uint8_t* o = s.dx + ((uint64_t)token * s.token + (uint64_t)head * s.head) * kEs<DT>;
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float xa = a[j] * rstd, xb = b[j] * rstd;
        sa[j] = __fmaf_rn(ya[j], xa, sa[j]);
        sb[j] = __fmaf_rn(yb[j], xb, sb[j]);
        if (s.dx && my.there[j]) put_elem<DT>(o, my.p[j].a, rstd * (__fmaf_rn(-xa, along, ya[j] * my.wa[j]) - level));
        if (s.dx && my.p[j].two) put_elem<DT>(o, my.p[j].b, rstd * (__fmaf_rn(-xb, along, yb[j] * my.wb[j]) - level));
      }
    }
    if (!s.dgamma) return;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (my.there[j]) acc[my.p[j].a] = sa[j];
      if (my.p[j].two) acc[my.p[j].b] = sb[j];
    }
  } else {
    if (s.dgamma)
      for (uint32_t e = lane; e < g.dim; e += 32u) acc[e] = 0.0f;
    __syncwarp();
    for (uint64_t u = first; u < units; u += step) {
      const uint32_t token = (uint32_t)(u / s.heads), head = (uint32_t)(u % s.heads);
      const int32_t at = position_of(g, token);
      if (at < 0) continue;
      const uint8_t* p = s.x + ((uint64_t)token * s.token + (uint64_t)head * s.head) * kEs<DT>;
      const uint8_t* q = s.dy + ((uint64_t)token * s.out_token + (uint64_t)head * s.out_head) * kEs<DT>;
      const float2* turn = g.table + (uint64_t)at * (g.rotary / 2u);
      const float mean = loose_mean<DT>(g, p, lane);
      // x less the mean, dz, and g of pair i
      struct Both {
        float xa, xb, da, db, ga, gb;
      };
      auto take = [&](uint32_t i, const LoosePair& e) {
        Both v;
        v.xa = elem_at<DT>(p, e.a) - mean;
        v.xb = e.two ? elem_at<DT>(p, e.b) - mean : 0.0f;
        const float ya = elem_at<DT>(q, e.a), yb = e.two ? elem_at<DT>(q, e.b) : 0.0f;
        const float2 t = e.turned ? turn[i] : make_float2(1.0f, 0.0f);
        v.da = __fmaf_rn(ya, t.x, yb * t.y);
        v.db = __fmaf_rn(yb, t.x, -(ya * t.y));
        v.ga = v.da * weight_at(s.gamma, g.wdtype, e.a);
        v.gb = e.two ? v.db * weight_at(s.gamma, g.wdtype, e.b) : 0.0f;
        return v;
      };
      float xx = 0.0f, gx = 0.0f, gs = 0.0f;
      for (uint32_t i = lane; i < loose_pairs(g); i += 32u) {
        const Both v = take(i, loose_pair<HALVES>(g, i));
        xx = __fmaf_rn(v.xb, v.xb, __fmaf_rn(v.xa, v.xa, xx));
        gx = __fmaf_rn(v.gb, v.xb, __fmaf_rn(v.ga, v.xa, gx));
        gs += v.ga + v.gb;
      }
      xx = team_sum<32>(xx);
      gx = team_sum<32>(gx);
      gs = team_sum<32>(gs);
      const float rstd = 1.0f / sqrtf(__fdiv_rn(xx, size) + g.eps);
      const float along = gx * rstd / size, level = g.layer ? gs / size : 0.0f;
      uint8_t* o = s.dx + ((uint64_t)token * s.token + (uint64_t)head * s.head) * kEs<DT>;
      for (uint32_t i = lane; i < loose_pairs(g); i += 32u) {
        const LoosePair e = loose_pair<HALVES>(g, i);
        const Both v = take(i, e);
        const float xa = v.xa * rstd, xb = v.xb * rstd;
        if (s.dgamma) {
          acc[e.a] = __fmaf_rn(v.da, xa, acc[e.a]);
          if (e.two) acc[e.b] = __fmaf_rn(v.db, xb, acc[e.b]);
        }
        if (s.dx) {
          put_elem<DT>(o, e.a, rstd * (__fmaf_rn(-xa, along, v.ga) - level));
          if (e.two) put_elem<DT>(o, e.b, rstd * (__fmaf_rn(-xb, along, v.gb) - level));
        }
      }
    }
    if (!s.dgamma) return;
  }
  __syncthreads();
  float* out = g.work + (uint64_t)((which ? g.side[0].parts : 0u) + part) * g.dim;
  for (uint32_t e = threadIdx.x; e < g.dim; e += blockDim.x) {
    float sum = 0.0f;
    for (uint32_t w = 0; w < warps; ++w) sum += loose_sums[(uint64_t)w * g.dim + e];
    out[e] = sum;
  }
}

// The weights' gradients: a warp's lanes have 32 columns, 32 warps share the parts, and are added up in their order.
__global__ void __launch_bounds__(1024) heads_columns_kernel(const HeadsArgs g) {
  __shared__ float sums[32][32];
  dep_trigger();
  dep_wait();
  const uint32_t groups = (g.dim + 31u) / 32u, which = blockIdx.x / groups, col = blockIdx.x % groups * 32u + threadIdx.x % 32, warp = threadIdx.x / 32;
  const HeadsSide& s = g.side[which];
  if (!s.dgamma) return;
  const float* p = g.work + (which ? (uint64_t)g.side[0].parts * g.dim : 0u) + col;
  float sum = 0.0f;
  if (col < g.dim) {
#pragma unroll 8
    for (uint32_t x = warp; x < s.parts; x += 32u) sum += p[(uint64_t)x * g.dim];
  }
  sums[warp][threadIdx.x % 32] = sum;
  __syncthreads();
  if (warp || col >= g.dim) return;
  sum = 0.0f;
#pragma unroll
  for (int w = 0; w < 32; ++w) sum += sums[w][threadIdx.x];
  if (g.wdtype == kF32)
    put_elem<kF32>(s.dgamma, col, sum);
  else
    put_elem<kBF16>(s.dgamma, col, sum);
}

struct TableArgs {
  float2* table;
  uint32_t positions, half;
  double step, scale;  // base^(-2 / rotary)'s logarithm to base 2
};
__global__ void __launch_bounds__(256) rotation_table_kernel(const TableArgs g) {
  dep_trigger();
  dep_wait();
  const uint64_t total = (uint64_t)g.positions * g.half;
  for (uint64_t i = (uint64_t)blockIdx.x * 256u + threadIdx.x; i < total; i += (uint64_t)gridDim.x * 256u) {
    const double angle = (double)(i / g.half) * exp2((double)(i % g.half) * g.step) * g.scale;
    double n, c;
    sincos(angle, &n, &c);
    g.table[i] = make_float2((float)c, (float)n);
  }
}

// Whether rows can be taken in slots: whole slots of what is rotated and of the rest, at most one to a lane, vectors on 16-byte boundaries.
template <int DT>
uint32_t heads_slots(const HeadsArgs& a) {
  const uint32_t two = 2u * kV<DT>;
  uint64_t all = a.dim % two || a.rotary % two || a.dim / two > 32u ? 1u : 0u;
  if (a.rotary) all |= (uintptr_t)a.table % 16u;
  for (const HeadsSide& s : a.side) {
    if (!s.heads) continue;
    all |= ((uintptr_t)s.x | (uintptr_t)s.out | (uintptr_t)s.dx | (uintptr_t)s.dy) % 16u;
    const uint64_t tokens = a.tokens > 1u ? s.token | s.out_token : 0u, heads = s.heads > 1u ? s.head | s.out_head : 0u;
    all |= ((tokens | heads) * kEs<DT>) % 16u;
  }
  return all ? 0u : a.dim / two;
}

// Pairs to a lane: 1, 2 or 4, or 0 where the row is longer.
template <typename L>
int loose_by_length(const HeadsArgs& a, L launch) {
  const uint32_t n = ((a.dim + 1u) / 2u + 31u) / 32u;
  auto with = [&](auto halves) {
    if (n <= 1u) return launch(std::integral_constant<int, 1>(), halves);
    if (n <= 2u) return launch(std::integral_constant<int, 2>(), halves);
    if (n <= 4u) return launch(std::integral_constant<int, 4>(), halves);
    return launch(std::integral_constant<int, 0>(), halves);
  };
  return a.halves ? with(std::true_type()) : with(std::false_type());
}

// `all` CTAs dealt out to queries and keys by the rows that they have, so that all end together.
void deal_out(HeadsArgs* a, uint64_t all) {
  const uint64_t q = a->side[0].heads, k = a->side[1].heads;
  a->side[0].parts = !q ? 0u : !k ? (uint32_t)all : (uint32_t)std::min<uint64_t>(all - 1, std::max<uint64_t>(1, all * q / (q + k)));
  a->side[1].parts = !k ? 0u : (uint32_t)(all - a->side[0].parts);
}

template <int DT, int T, int U, bool HALVES>
int forward_t(const HeadsArgs& a0, cudaStream_t stream) {
  HeadsArgs a = a0;
  constexpr uint32_t per_cta = kHeadWarps * (32 / T);
  uint64_t grid = a.status ? 1u : 0u;
  for (HeadsSide& s : a.side) {
    const uint64_t ctas = ((uint64_t)a.tokens * ((s.heads + U - 1u) / U) + per_cta - 1u) / per_cta;
    if (ctas > 0x3FFFFFFFull) return FH_ERR_UNSUPPORTED;
    s.parts = (uint32_t)ctas;
    grid += ctas;
  }
  return launch_plain<heads_forward_kernel<DT, T, U, HALVES>>((uint32_t)grid, kHeadThreads, 0, 1, stream, a);
}
template <int DT, int T>
int forward_n(const HeadsArgs& a, cudaStream_t stream) {
  // Heads to a team: four, or two where there are no more, if every SM then has eight warps; else one.  (16384 tokens of 32 + 8 heads of 128 in bf16: four 62 us,
  // two 73, one 93; 1024: 6.3, 7.2 and 8.1; 64: 3.0, 2.6 and 2.5.)
  const uint64_t rows = (uint64_t)a.tokens * (a.side[0].heads + a.side[1].heads), warps = rows / (32u / T), enough = 8ull * std::max(1, sm_count());
  const uint32_t heads = std::max(a.side[0].heads, a.side[1].heads);
  auto with = [&](auto halves) {
    if (heads > 2u && warps / 4u >= enough) return forward_t<DT, T, 4, halves.value>(a, stream);
    if (heads > 1u && warps / 2u >= enough) return forward_t<DT, T, 2, halves.value>(a, stream);
    return forward_t<DT, T, 1, halves.value>(a, stream);
  };
  return a.halves ? with(std::true_type()) : with(std::false_type());
}
template <int DT>
int forward_d(const HeadsArgs& a, cudaStream_t stream) {
  const uint32_t slots = heads_slots<DT>(a);
  if (!slots) {
    const uint64_t units = (uint64_t)a.tokens * (a.side[0].heads + a.side[1].heads), grid = (units + kHeadWarps - 1u) / kHeadWarps + (a.status ? 1u : 0u);
    if (grid > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
    return loose_by_length(a, [&](auto n, auto halves) {
      return launch_plain<heads_forward_loose_kernel<DT, n.value, halves.value>>((uint32_t)grid, kHeadThreads, 0, 1, stream, a);
    });
  }
  if (slots <= 4u) return forward_n<DT, 4>(a, stream);
  if (slots <= 8u) return forward_n<DT, 8>(a, stream);
  if (slots <= 16u) return forward_n<DT, 16>(a, stream);
  return forward_n<DT, 32>(a, stream);
}

// CTAs of the backward pass: a rule's most, and another for every so many rows.  The workspace is sized for kHeadMost and kHeadFewest, which no rule is
// beyond.  (148 SMs, whatever the device says: the workspace's size is asked for without one, and sums do not depend on it.)
constexpr uint32_t kHeadMost = 148 * 8, kHeadFewest = 4;

uint64_t heads_parts_of(const HeadsArgs& a, uint32_t most, uint32_t rows_per_cta) {
  const uint64_t rows = (uint64_t)a.tokens * (a.side[0].heads + a.side[1].heads);
  return std::min<uint64_t>(a.dim > 1024u ? 148u : most, std::max<uint64_t>(2, (rows + rows_per_cta - 1) / rows_per_cta));
}
void heads_parts(HeadsArgs* a, uint32_t most, uint32_t rows_per_cta) { deal_out(a, heads_parts_of(*a, most, rows_per_cta)); }

template <typename L>
int backward_launch(const HeadsArgs& a, cudaStream_t stream, L rows) {
  const int rc = rows(a.side[0].parts + a.side[1].parts + (a.status ? 1u : 0u));
  if (rc != FH_OK || (!a.side[0].dgamma && !a.side[1].dgamma)) return rc;
  return launch_plain<heads_columns_kernel>((a.dim + 31u) / 32u * 2u, 1024, 0, 1, stream, a);
}
template <int DT, int T, bool HALVES>
int backward_t(const HeadsArgs& a0, cudaStream_t stream) {
  HeadsArgs a = a0;
  constexpr uint32_t rows = kHeadWarps * (32u / T);
  static_assert(rows >= kHeadFewest, "the workspace's size");
  heads_parts(&a, 148u * kBackCtas<DT>, rows);
  return backward_launch(a, stream, [&](uint32_t grid) { return launch_plain<heads_backward_kernel<DT, T, HALVES>>(grid, kHeadThreads, 0, 1, stream, a); });
}
template <int DT, int T>
int backward_n(const HeadsArgs& a, cudaStream_t stream) {
  return a.halves ? backward_t<DT, T, true>(a, stream) : backward_t<DT, T, false>(a, stream);
}
template <int DT>
int backward_d(const HeadsArgs& a0, cudaStream_t stream) {
  const uint32_t slots = heads_slots<DT>(a0);
  if (!slots) {
    HeadsArgs a = a0;
    const uint32_t warps = std::max(1u, std::min(kHeadWarps, 8192u / a.dim));  // (32 KB of sums)
    heads_parts(&a, kHeadMost, kHeadFewest * warps);
    return backward_launch(a, stream, [&](uint32_t grid) {
      return loose_by_length(a, [&](auto n, auto halves) {
        return launch_plain<heads_backward_loose_kernel<DT, n.value, halves.value>>(grid, (int)warps * 32, (size_t)warps * a.dim * sizeof(float), 1, stream, a);
      });
    });
  }
  if (slots <= 4u) return backward_n<DT, 4>(a0, stream);
  if (slots <= 8u) return backward_n<DT, 8>(a0, stream);
  if (slots <= 16u) return backward_n<DT, 16>(a0, stream);
  return backward_n<DT, 32>(a0, stream);
}

}  // namespace

size_t heads_work_floats(const HeadsArgs& a) { return (size_t)heads_parts_of(a, kHeadMost, kHeadFewest) * a.dim; }

int launch_heads_forward(const HeadsArgs& a, int dtype, cudaStream_t stream) {
  return dtype == kF32 ? forward_d<kF32>(a, stream) : forward_d<kBF16>(a, stream);
}

int launch_heads_backward(const HeadsArgs& a, int dtype, cudaStream_t stream) {
  return dtype == kF32 ? backward_d<kF32>(a, stream) : backward_d<kBF16>(a, stream);
}

int launch_rotation_table(uint32_t positions, uint32_t rotary, double base, double scale, float2* table, cudaStream_t stream) {
  TableArgs a = {table, positions, rotary / 2u, -2.0 * std::log2(base) / rotary, scale};
  const uint64_t ctas = ((uint64_t)positions * a.half + 255u) / 256u;
  return launch_plain<rotation_table_kernel>((uint32_t)std::min<uint64_t>(ctas, (uint64_t)std::max(1, sm_count()) * 16u), 256, 0, 1, stream, a);
}

}  // namespace fh
