// Launching the kernels on microscaled 4-bit matrices and of the layer norm: their arguments, and what their host sides share.
#pragma once

#include "../../include/fh.h"

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace fh {

struct MxSaveArgs {
  const uint8_t* src;              // dense (compress) or container (decompress)
  uint64_t src_bytes;              // decompress: readable bytes of the container
  uint8_t *by_rows, *by_cols;      // compress: containers, either may be null
  uint8_t* dst;                    // decompress: dense
  unsigned long long* status;      // decompress: may be null
  uint32_t rows, cols;
  uint64_t ld;
  int32_t exponent;
  uint64_t tensor_id;
  uint32_t round_keys[20];         // compress, random rounding: the keys of Philox's ten rounds
};
// (Enqueues on `stream`; returns an fh_status.)
int launch_mx_save(const MxSaveArgs& a, int dtype, int format, bool compress, bool random, cudaStream_t stream);

struct MxProductArgs {
  const uint8_t *a, *b;            // containers
  uint64_t a_bytes, b_bytes;
  uint8_t* c;
  unsigned long long* status;      // may be null
  uint32_t m, n, k;
  uint64_t ldc;
  float alpha;
  bool accumulate;
  uint32_t polls, silent;          // limit of the kernels' waits, and a stage that is not loaded (fh_debug_set)
  uint32_t tiles_m, tiles_n, split;  // set where the kernel is launched
};
int launch_mx_product(const MxProductArgs& a, int dtype, int format, cudaStream_t stream);

struct NormArgs {
  const uint8_t *x, *gamma, *beta, *dy;  // x: dense, or a container of x_bytes bytes (backward, x_bytes > 0)
  uint64_t x_bytes;
  uint8_t *y, *dx, *dgamma, *dbeta;      // any may be null
  float *mean, *rstd;                    // forward: may be null
  uint8_t* packed;                       // forward: container of y, may be null
  float* work;                           // backward: sums of each CTA's rows, null when no weight's gradient is wanted
  unsigned long long* status;            // backward: may be null
  uint64_t ldx, ldy;                     // of x and dx, of y and dy
  uint64_t tensor_id;
  uint32_t rows, cols, format;
  int32_t exponent, wdtype;
  uint32_t parts;                        // backward: CTAs (set where the kernel is launched)
  float eps;
};
constexpr uint32_t kNormCols = 28672;    // longest row: two sums a column in an SM's shared memory
// CTAs among which the rows are dealt out in the backward pass.
uint32_t norm_parts(uint32_t rows, uint32_t cols, int dtype);
int launch_norm_forward(const NormArgs& a, int dtype, cudaStream_t stream);
int launch_norm_backward(const NormArgs& a, int dtype, cudaStream_t stream);

constexpr size_t kMxSmemLimit = 226 * 1024;  // dynamic shared memory a CTA may have, next to a little that a kernel declares

// What fh_debug_set has set, for the product's waits.
void debug_waits(uint32_t* polls, uint32_t* silent);

// Counts a kernel for fh_kernel_launches().
void count_launch(int kernels = 1);

// Launch of `grid` CTAs, in clusters of `cluster`, that may become resident as the previous kernel on the stream drains (its order
// is kept by dep_wait()).  A kernel that needs more than the usual 48 KB, with the little that it declares, gets it raised once for each device.
template <auto Kernel, typename A>
int launch_plain(uint32_t grid, int threads, size_t smem, int cluster, cudaStream_t stream, const A& a) {
  static std::atomic<uint64_t> raised{0};  // bit per device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return FH_ERR_CUDA;
  if (smem > 40 * 1024 && (dev > 63 || !(raised.load() >> dev & 1u))) {
    if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMxSmemLimit) != cudaSuccess) {
      cudaGetLastError();
      return FH_ERR_CUDA;
    }
    if (dev < 64) raised.fetch_or(1ull << dev);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (cluster > 1) {
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
  }
  if (cudaLaunchKernelEx(&cfg, Kernel, a) != cudaSuccess) {
    cudaGetLastError();
    return FH_ERR_CUDA;
  }
  count_launch();
  return FH_OK;
}

}  // namespace fh
