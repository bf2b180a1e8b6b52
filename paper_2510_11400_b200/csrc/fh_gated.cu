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

// dg = dh u act'(g), du = dh act(g); elementwise, so that memory bounds it, but for the row's scale, which needs the whole row.  Lanes lie R rows by 32 / R
// chunks of 16 columns, as in the kernel that compresses a matrix by rows, each with the chunk of g, u and dh.  A lane's I chunks of dg and du stay in
// registers, rounded to their type, from the row's maximum to its codes; I = 0: the row is too long for that, and they are read again where they were
// written, or made again.
template <int DT, int ACT, int R, int I, bool VEC>
__global__ void __launch_bounds__(512) gated_backward_kernel(const GatedArgs g) {
  __shared__ uint32_t tops[16][R];
  constexpr uint32_t kLanes = 32 / R;
  const uint32_t width = g.width;
  const I8Layout l(g.rows, 2u * width);
  const uint32_t tid = threadIdx.x, warp = tid / 32, lane = tid % 32, warps = blockDim.x / 32;
  const uint32_t r = lane % R, row = blockIdx.x * R + r, chunks = (width + 15u) / 16u, first = warp * kLanes + lane / R, step = warps * kLanes;
  const bool there = row < g.rows;
  const uint8_t *dh = g.dh + (uint64_t)row * g.ldh * kEs<DT>, *pre = g.pre + (uint64_t)row * g.ldp * kEs<DT>;
  uint8_t* dpre = g.dpre + (uint64_t)row * g.ldp * kEs<DT>;
  dep_trigger();
  dep_wait();
  if (g.packed && blockIdx.x == 0 && tid < 32) i8_write_header(g.packed, l, tid);
  auto size = [&](uint32_t j) { return there && j < chunks ? (int)min(16u, width - j * 16u) : 0; };
  auto make = [&](uint32_t j, Raw16<DT>& dg, Raw16<DT>& du) {
    const int n = size(j);
    const uint64_t c = (uint64_t)j * 16u * kEs<DT>;
    Raw16<DT> a, b, d;
    a.template load<VEC>(pre + c, n);
    b.template load<VEC>(pre + c + (uint64_t)width * kEs<DT>, n);
    d.template load<VEC>(dh + c, n);
    float fg[16], fu[16], fd[16];
    a.values(fg);
    b.values(fu);
    d.values(fd);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float act, slope;
      act_and_slope<ACT>(fg[i], act, slope);
      fg[i] = fd[i] * fu[i] * slope;
      fu[i] = fd[i] * act;
    }
    dg.take(fg);
    du.take(fu);
  };
  auto keep = [&](uint32_t j, const Raw16<DT>& dg, const Raw16<DT>& du) {
    const int n = size(j);
    const uint64_t c = (uint64_t)j * 16u * kEs<DT>;
    dg.template store<VEC>(dpre + c, n);
    du.template store<VEC>(dpre + c + (uint64_t)width * kEs<DT>, n);
  };
  constexpr int N = I ? I : 1;
  Raw16<DT> dg[N], du[N];
  uint32_t top = 0;
  if (I) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      make(first + i * step, dg[i], du[i]);
      if (g.dpre) keep(first + i * step, dg[i], du[i]);
      top = max(top, max(dg[i].top(), du[i].top()));
    }
  } else {
    for (uint32_t j = first; j < chunks; j += step) {
      make(j, dg[0], du[0]);
      if (g.dpre) keep(j, dg[0], du[0]);
      top = max(top, max(dg[0].top(), du[0].top()));
    }
  }
  if (!g.packed) return;
#pragma unroll
  for (int s = R; s < 32; s *= 2) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
  if (lane < R) tops[warp][r] = top;
  __syncthreads();
  for (uint32_t w = 0; w < warps; ++w) top = max(top, tops[w][r]);
  if (row >= l.r8) return;
  const I8Coder<DT> coder(top);
  uint8_t* dst = g.packed + l.code_at(row, 0);
  const uint64_t pitch = 16ull * l.block_rows(row / 128u);
  // Codes of n elements from column c of dpre on, n < 16 or c off the chunks' boundaries where the width is no multiple of 16.
  auto put = [&](const Raw16<DT>& v, uint32_t c, uint32_t n) {
    float f[16];
    v.values(f);
    const uint4 q = i8_codes16(f, coder);
    if (n == 16u && c % 16u == 0u) {
      *reinterpret_cast<uint4*>(dst + c / 16u * pitch) = q;
      return;
    }
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (uint32_t i = 0; i < 16u; ++i)
      if (i < n) dst[(c + i) / 16u * pitch + (c + i) % 16u] = (uint8_t)(w[i / 4u] >> (i % 4u * 8u));
  };
  auto put_both = [&](uint32_t j, const Raw16<DT>& a, const Raw16<DT>& b) {
    const uint32_t c = j * 16u, n = min(16u, width - c);
    put(a, c, n);
    put(b, width + c, n);
    if (j + 1u == chunks)
      for (uint32_t p = 2u * width; p < l.kp; ++p) dst[p / 16u * pitch + p % 16u] = 0u;
  };
  if (I) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (first + i * step < chunks) put_both(first + i * step, dg[i], du[i]);
  } else {
    for (uint32_t j = first; j < chunks; j += step) {
      if (g.dpre) {  // (this thread's own stores)
        const int n = size(j);
        const uint64_t c = (uint64_t)j * 16u * kEs<DT>;
        dg[0].template load<VEC>(dpre + c, n);
        du[0].template load<VEC>(dpre + c + (uint64_t)width * kEs<DT>, n);
      } else {
        make(j, dg[0], du[0]);
      }
      put_both(j, dg[0], du[0]);
    }
  }
  if (warp == 0 && lane < R) *reinterpret_cast<uint32_t*>(g.packed + l.magnitude_at(row)) = i8_magnitude_bits(top);
}

template <int DT, int ACT, int R, bool VEC>
int gated_by_length(const GatedArgs& a, cudaStream_t stream) {
  constexpr uint32_t kLanes = 32 / R;
  const uint32_t need = ((a.width + 15u) / 16u + kLanes - 1u) / kLanes;  // steps of a warp in all
  const uint64_t rows = a.packed ? I8Layout(a.rows, 1u).r8 : a.rows, grid = (rows + R - 1u) / R;
  if (grid > 0x7FFFFFFFull) return FH_ERR_UNSUPPORTED;
  if (need <= 16u) return launch_plain<gated_backward_kernel<DT, ACT, R, 1, VEC>>((uint32_t)grid, (int)need * 32, 0, 1, stream, a);
  return launch_plain<gated_backward_kernel<DT, ACT, R, 0, VEC>>((uint32_t)grid, 512, 0, 1, stream, a);
}
template <int DT, int ACT>
int gated_launch(const GatedArgs& a, cudaStream_t stream) {
  const uint64_t es = kEs<DT>;
  const bool vec = ((uintptr_t)a.dh | (uintptr_t)a.pre | (uintptr_t)a.dpre | a.ldh * es | a.ldp * es | a.width * es) % 16u == 0u;
  const uint32_t sms = (uint32_t)std::max(1, sm_count());
  // Eight rows to a CTA write pieces of codes whole; fewer where there are not enough rows for every SM.
  const bool many = a.rows / 8u >= sms;
  if (many) return vec ? gated_by_length<DT, ACT, 8, true>(a, stream) : gated_by_length<DT, ACT, 8, false>(a, stream);
  return vec ? gated_by_length<DT, ACT, 1, true>(a, stream) : gated_by_length<DT, ACT, 1, false>(a, stream);
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
