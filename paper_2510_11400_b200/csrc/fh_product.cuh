// What the kernels of products of matrices held in few bits share (fh_mx_product.cu, fh_i8_product.cu): the rules of their waits, rings of stages,
// accesses to C, the order of tiles, tensor maps, and how many clusters there are.
#pragma once

#include <cuda.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fh_launch.cuh"
#include "fh_mx_launch.cuh"
#include "fh_tcgen05.cuh"

namespace fh {
namespace {

constexpr uint32_t kDrainPolls = 1u << 20;  // waits of up to 2 us each, for copies under way

// Waits.  Every wait of a role (loads, matrix instructions, scales, result) has a limit, `polls` (2^26, some seconds); the first one that runs
// out sets a flag, the CTA's or in a pair that of the whole cluster, which ends the others.  What is still under way then is waited for at the
// end, when no role runs any more and the flag no longer changes: nothing may be in flight, in this CTA's memory or the other one's, when a
// CTA ends.  Where no wait has run out, everything has been waited for on the way: copies by the thread that reads them (matrix instructions
// or scales), the instructions by the result's warps, and the word that a stage is free, given only where the stage is used again, by
// the loading thread.  The status is first written by CTA 0, one of the first to run, as it begins; a CTA that has given up writes
// FH_ERR_TIMEOUT as it ends, a wait and a drain later.

// An aligned place for a CTA's stages.  `zero` hides from the compiler that it has this address already: what only the end of the pair
// kernel needs would take registers from its result warps (168 instead of 165; 4096 x 4096 x 4096 42.4 us and 48, 8192 x 16384 x 8192 400 and 428).
__device__ __forceinline__ uint8_t* stages_at(uint8_t* raw, uint32_t zero = 0u) { return raw + ((128u - (smem_u32(raw) & 127u)) & 127u) + zero; }
__device__ __forceinline__ uint32_t hidden_zero() {
  uint32_t r;
  asm volatile("mov.u32 %0, 0;" : "=r"(r));
  return r;
}

// Stage of a ring and the parity of its round.
template <int STAGES>
struct Turn {
  uint32_t stage = 0, round = 0;
  __device__ __forceinline__ void next() {
    if (++stage == (uint32_t)STAGES) {
      stage = 0;
      round ^= 1u;
    }
  }
};

// NR rows of a column of C from row `row` on, those below `end`.  (Addresses step from row to row: a product with ldc for each of them
// made a tile of 128 x 256 take 4 us.)
template <int DT>
using CType = typename std::conditional<DT == kF32, float, __nv_bfloat16>::type;
template <int DT, int NR>
__device__ __forceinline__ void load_c(const uint8_t* c, uint64_t ldc, uint32_t row, uint32_t end, uint32_t col, float (&v)[NR]) {
  const CType<DT>* p = reinterpret_cast<const CType<DT>*>(c) + (uint64_t)row * ldc + col;
#pragma unroll
  for (int x = 0; x < NR; ++x, p += ldc) {
    v[x] = 0.0f;
    if (row + x < end) v[x] = (float)*p;
  }
}
template <int DT, int NR>
__device__ __forceinline__ void store_c(uint8_t* c, uint64_t ldc, uint32_t row, uint32_t end, uint32_t col, const float (&v)[NR]) {
  CType<DT>* p = reinterpret_cast<CType<DT>*>(c) + (uint64_t)row * ldc + col;
  if (row + NR <= end) {
#pragma unroll
    for (int x = 0; x < NR; ++x, p += ldc) *p = (CType<DT>)v[x];
    return;
  }
#pragma unroll
  for (int x = 0; x < NR; ++x, p += ldc)
    if (row + x < end) *p = (CType<DT>)v[x];
}

// Tile `t` of the pairs' order: eight rows of tiles at a time, column by column, so that the tiles under way together share rows of A and of B
// in L2 (row by row, 8192 x 16384 x 8192 took 595 us).
struct PairTile {
  uint32_t m, n;
  __device__ __forceinline__ PairTile(uint32_t t, uint32_t tiles_m, uint32_t tiles_n) {
    const uint32_t band = t / (8u * tiles_n), at = t % (8u * tiles_n), high = min(8u, tiles_m - 8u * band);
    m = 8u * band + at % high;
    n = at / high;
  }
};

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static std::atomic<void*> fn{nullptr};
  void* f = fn.load();
  if (!f) {
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) return nullptr;
    fn.store(f);
  }
  return (EncodeTiled)f;
}

// A map of `dims` boxes of 128 bytes, `strides` bytes apart, as bytes.
bool encode_map(CUtensorMap* map, const uint8_t* base, uint32_t rank, const cuuint64_t (&dims)[3], const cuuint64_t (&strides)[2], const cuuint32_t (&box)[3]) {
  const EncodeTiled f = encode_tiled();
  const cuuint32_t ones[3] = {1, 1, 1};
  return f && f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, rank, const_cast<uint8_t*>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Clusters of `size` CTAs of a kernel that the device holds at once (0: an error): fewer than CTAs divided by size, as a cluster stays within
// a part of the device (of 148 CTAs of the pair kernel, 33 clusters of four, 22 of six, 15 of eight).
template <auto Kernel>
int clusters_at_once(int size, int threads, size_t smem) {
  static std::atomic<int> known[64][9];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || size < 1 || size > 8) return 0;
  if (dev < 64 && known[dev][size].load()) return known[dev][size].load();
  if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMxSmemLimit) != cudaSuccess) return 0;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)size);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)size;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  int n = 0;
  if (cudaOccupancyMaxActiveClusters(&n, Kernel, &cfg) != cudaSuccess) {
    cudaGetLastError();
    return 0;
  }
  if (dev < 64) known[dev][size].store(n);
  return n;
}

// Into how many parts to split the common axis: what takes the fewest rounds of stages, where a round of clusters costs `fixed` stages besides and a
// split two more than that.  At least two stages to a part.
template <typename AtOnce>
uint32_t choose_split(uint64_t tiles, uint64_t steps, uint32_t most, uint64_t fixed, AtOnce at_once) {
  uint32_t best = 1;
  uint64_t least = ~0ull;
  for (uint32_t s = 1; s <= most && (s == 1 || 2 * s <= steps); ++s) {
    const int n = at_once(s);
    if (n < 1) continue;
    const uint64_t cost = (tiles + n - 1) / n * ((steps + s - 1) / s + fixed + (s > 1 ? fixed / 2 : 0));
    if (cost < least) {
      least = cost;
      best = s;
    }
  }
  return best;
}

}  // namespace
}  // namespace fh
