// The gated feed-forward block's backward pass up to the products: gradients of both projections' results, dense and in 8 bits.
#include <algorithm>

#include "fh_act.cuh"
#include "fh_i8.cuh"
#include "fh_i8_launch.cuh"
#include "fh_launch.cuh"

namespace fh {
namespace {

template <int DT>
constexpr uint32_t kEs = DT == kF32 ? 4u : 2u;

// dg = dh u act'(g), du = dh act(g); elementwise, so that memory bounds it, but for the row's scale, which needs the whole row.  A CTA takes a row, a lane
// chunks of 16 columns of g, u and dh.  A lane's I chunks of dg and du stay in registers, rounded to their type, from the row's maximum to its codes;
// I = 0: the row is too long for that, and they are read again where they were written, or made again.
//
// Where the width is no multiple of 16, du's chunks begin inside a chunk of the container.  The row's codes are then put together in shared memory (`room`
// bytes), or written byte by byte where there is no room.
//
// Registers for three CTAs an SM in bf16 (4096 x 8192 76 to 81 us; with earlier activations 83, for two 101, for four 92), for two in fp32 (4096 x 4096 78, three
// 82).  Four chunks to a lane, widths from 8193 to 16384, do not fit those: up to 124 bytes a thread are spilled there, and 4096 x 11008 takes 130 us.
struct GatedPlan {
  GatedArgs g;
  uint32_t room;
};

template <int DT, int ACT, int I, bool VEC>
__global__ void __launch_bounds__(256, DT == kF32 ? 2 : 3) gated_backward_kernel(const GatedPlan plan) {
  const GatedArgs& g = plan.g;
  using Loose = LooseRows<DT, 1>;
  extern __shared__ __align__(16) uint8_t joined[];
  __shared__ uint32_t tops[8];
  __shared__ __align__(16) uint8_t stages[VEC ? 16 : 8 * Loose::kBytes];
  const uint32_t width = g.width;
  const I8Layout l(g.rows, 2u * width);
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = blockDim.x / 32;
  const uint32_t row = blockIdx.x, chunks = (width + 15u) / 16u, first = tid, step = blockDim.x;
  const bool there = row < g.rows;
  const uint64_t at_h = (uint64_t)row * g.ldh * kEs<DT>, at_p = (uint64_t)row * g.ldp * kEs<DT>, behind = (uint64_t)width * kEs<DT>;
  uint8_t* stage = stages + (VEC ? 0u : warp * Loose::kBytes);
  dep_trigger();
  dep_wait();
  if (g.packed && blockIdx.x == 0 && tid < 32) i8_write_header(g.packed, l, tid);
  // Chunk j of a row of `width` elements at p.
  auto fetch = [&](Raw16<DT>& x, const uint8_t* p, uint64_t ld, uint32_t j) {
    if (VEC)
      x.template load<true>(p + (uint64_t)j * 16u * kEs<DT>, there && j < chunks ? (int)min(16u, width - j * 16u) : 0);
    else
      Loose::load(x, stage, p, ld, there ? 1u : 0u, (j - lane) * 16u, width, lane);
  };
  auto keep = [&](const Raw16<DT>& x, uint8_t* p, uint32_t j) {
    if (VEC)
      x.template store<true>(p + (uint64_t)j * 16u * kEs<DT>, there && j < chunks ? (int)min(16u, width - j * 16u) : 0);
    else
      Loose::store(x, stage, p, g.ldp, there ? 1u : 0u, (j - lane) * 16u, width, lane);
  };
  auto make = [&](uint32_t j, Raw16<DT>& dg, Raw16<DT>& du) {
    Raw16<DT> d;
    fetch(dg, g.pre + at_p, g.ldp, j);
    fetch(du, g.pre + at_p + behind, g.ldp, j);
    fetch(d, g.dh + at_h, g.ldh, j);
    float fg[16], fu[16], fd[16];
    dg.values(fg);
    du.values(fu);
    d.values(fd);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float act, slope;
      act_and_slope<ACT, DT>(fg[i], act, slope);
      fg[i] = fd[i] * (fu[i] * slope);  // (dh u may be beyond the largest number where the derivative is 0)
      fu[i] = fd[i] * act;
    }
    dg.take(fg);
    du.take(fu);
  };
  auto keep_both = [&](uint32_t j, const Raw16<DT>& dg, const Raw16<DT>& du) {
    keep(dg, g.dpre + at_p, j);
    keep(du, g.dpre + at_p + behind, j);
  };
  constexpr int N = I ? I : 1;
  Raw16<DT> dg[N], du[N];
  uint32_t top = 0;
  if (I) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      make(first + i * step, dg[i], du[i]);
      if (g.dpre) keep_both(first + i * step, dg[i], du[i]);
      top = max(top, max(dg[i].top(), du[i].top()));
    }
  } else {
    for (uint32_t j = first; j < chunks + lane; j += step) {  // (all lanes of a warp as often)
      make(j, dg[0], du[0]);
      if (g.dpre) keep_both(j, dg[0], du[0]);
      top = max(top, max(dg[0].top(), du[0].top()));
    }
  }
  if (!g.packed) return;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
  if (lane == 0) tops[warp] = top;
  __syncthreads();
  for (uint32_t w = 0; w < warps; ++w) top = max(top, tops[w]);
  const I8Coder<DT> coder(top);
  uint8_t* dst = g.packed + l.code_at(row, 0);
  const uint64_t pitch = 16ull * l.block_rows(row / 128u);
  // Codes of n elements from column c of dpre on.
  auto put = [&](const Raw16<DT>& v, uint32_t c, uint32_t n) {
    float f[16];
    v.values(f);
    const uint4 q = i8_codes16(f, coder);
    if (n == 16u && c % 16u == 0u && !plan.room) {
      *reinterpret_cast<uint4*>(dst + c / 16u * pitch) = q;
      return;
    }
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    if (plan.room && c % 4u == 0u && n == 16u) {
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i) reinterpret_cast<uint32_t*>(joined + c)[i] = w[i];
      return;
    }
#pragma unroll
    for (uint32_t i = 0; i < 16u; ++i)
      if (i < n) *(plan.room ? joined + c + i : dst + (c + i) / 16u * pitch + (c + i) % 16u) = (uint8_t)(w[i / 4u] >> (i % 4u * 8u));
  };
  auto put_both = [&](uint32_t j, const Raw16<DT>& a, const Raw16<DT>& b) {
    const uint32_t c = j * 16u, n = min(16u, width - c);
    put(a, c, n);
    put(b, width + c, n);
    if (j + 1u == chunks)
      for (uint32_t p = 2u * width; p < l.kp; ++p) *(plan.room ? joined + p : dst + p / 16u * pitch + p % 16u) = 0u;
  };
  if (I) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (first + i * step < chunks) put_both(first + i * step, dg[i], du[i]);
  } else {
    for (uint32_t j = first; j < chunks + lane; j += step) {
      if (g.dpre && VEC) {  // (this thread's own stores)
        fetch(dg[0], g.dpre + at_p, g.ldp, j);
        fetch(du[0], g.dpre + at_p + behind, g.ldp, j);
      } else if (g.dpre) {  // (this warp's)
        __syncwarp();
        fetch(dg[0], g.dpre + at_p, g.ldp, j);
        fetch(du[0], g.dpre + at_p + behind, g.ldp, j);
      } else {
        make(j, dg[0], du[0]);
      }
      if (j < chunks) put_both(j, dg[0], du[0]);
    }
  }
  if (tid == 0) *reinterpret_cast<uint32_t*>(g.packed + l.magnitude_at(row)) = i8_magnitude_bits(top);
  if (plan.room) {
    __syncthreads();
    for (uint32_t j = first; j < l.chunks(); j += step) *reinterpret_cast<uint4*>(dst + j * pitch) = *reinterpret_cast<const uint4*>(joined + j * 16u);
  }
}

template <int DT, int ACT, int I, bool VEC>
int gated_start(const GatedArgs& a, uint32_t warps, cudaStream_t stream) {
  const uint64_t grid = a.packed ? I8Layout(a.rows, 1u).r8 : a.rows;
  if (grid > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
  GatedPlan p = {a, 0u};
  const uint64_t room = I8Layout(1u, 2u * a.width).kp;
  // (with what the kernel declares, 17 KB at most, within the 48 KB that need no asking)
  if (a.packed && a.width % 16u && room <= 30 * 1024) p.room = (uint32_t)room;
  return launch_plain<gated_backward_kernel<DT, ACT, I, VEC>>((uint32_t)grid, (int)warps * 32, p.room, 1, stream, p);
}
// A row to a CTA (with two, whose codes are written in whole sectors, 4096 x 8192 bf16 took 6 % less, but 4096 x 2048 22.6 -> 27 us, 16384 x 1024 41 -> 46), of up
// to eight warps, and as few chunks to a lane as hold it; in fp32, whose chunks take twice the registers, two where there are two (4096 x 4096 90 us with one, 78).
template <int DT, int ACT, bool VEC>
int gated_by_length(const GatedArgs& a, cudaStream_t stream) {
  const uint32_t need = (a.width + 511u) / 512u;  // steps of a warp in all
  if (need <= (DT == kF32 ? 1u : 8u)) return gated_start<DT, ACT, 1, VEC>(a, need, stream);
  if (need <= 16u) return gated_start<DT, ACT, 2, VEC>(a, (need + 1u) / 2u, stream);
  if (DT == kBF16 && need <= 32u) return gated_start<DT, ACT, DT == kBF16 ? 4 : 2, VEC>(a, (need + 3u) / 4u, stream);
  return gated_start<DT, ACT, 0, VEC>(a, 8u, stream);
}
template <int DT, int ACT>
int gated_launch(const GatedArgs& a, cudaStream_t stream) {
  const uint64_t es = kEs<DT>;
  const bool vec = ((uintptr_t)a.dh | (uintptr_t)a.pre | (uintptr_t)a.dpre | a.ldh * es | a.ldp * es | a.width * es) % 16u == 0u;
  return vec ? gated_by_length<DT, ACT, true>(a, stream) : gated_by_length<DT, ACT, false>(a, stream);
}
template <int ACT>
int gated_by_type(const GatedArgs& a, int dtype, cudaStream_t stream) {
  return dtype == kF32 ? gated_launch<kF32, ACT>(a, stream) : gated_launch<kBF16, ACT>(a, stream);
}

}  // namespace

int launch_gated_backward(const GatedArgs& a, int dtype, int activation, cudaStream_t stream) {
  if (activation == FH_SILU) return gated_by_type<FH_SILU>(a, dtype, stream);
  if (activation == FH_GELU) return gated_by_type<FH_GELU>(a, dtype, stream);
  if (activation == FH_GELU_TANH) return gated_by_type<FH_GELU_TANH>(a, dtype, stream);
  return gated_by_type<FH_RELU>(a, dtype, stream);
}

}  // namespace fh
