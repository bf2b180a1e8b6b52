// Launching the kernels on 8-bit matrices and on heads: their arguments.
#pragma once

#include "fh_mx_launch.cuh"

namespace fh {

struct I8SaveArgs {
  const uint8_t* src;          // dense (compress) or container (decompress)
  uint64_t src_bytes;          // decompress: readable bytes of the container
  uint8_t* dst;                // container (compress) or dense (decompress)
  unsigned long long* status;  // decompress: may be null
  uint32_t rows, cols;
  uint64_t ld;
  uint32_t parts;              // by columns: CTAs of a cluster (set where the kernel is launched)
};
// (All of these enqueue on `stream` and return an fh_status.)
int launch_i8_rows(const I8SaveArgs& a, int dtype, cudaStream_t stream);
int launch_i8_cols(const I8SaveArgs& a, int dtype, cudaStream_t stream);
int launch_i8_decompress(const I8SaveArgs& a, int dtype, cudaStream_t stream);

struct I8ProductArgs {
  const uint8_t *a, *b, *up;            // containers; up: the gated block's second weight
  uint64_t a_bytes, b_bytes, up_bytes;
  uint8_t *c, *pre;                     // product: C, null; gated: h and pre, either may be null
  unsigned long long* status;           // may be null
  uint32_t m, n, k;
  uint64_t ldc, ldp;
  float alpha;
  bool accumulate;
  uint32_t polls, silent;               // limit of the kernels' waits, and a stage that is not loaded (fh_debug_set)
  uint32_t tiles_m, tiles_n, split;     // set where the kernel is launched
};
int launch_i8_product(const I8ProductArgs& a, int dtype, cudaStream_t stream);
int launch_i8_gated(const I8ProductArgs& a, int dtype, int activation, cudaStream_t stream);

struct GatedArgs {
  const uint8_t *dh, *pre;
  uint8_t *dpre, *packed;  // either may be null
  uint32_t rows, width;
  uint64_t ldh, ldp;
};
int launch_gated_backward(const GatedArgs& a, int dtype, int activation, cudaStream_t stream);

struct HeadsSide {  // queries or keys
  const uint8_t *x, *gamma, *dy;
  uint8_t *out, *dx, *dgamma;
  uint64_t token, head, out_token, out_head;
  uint32_t heads;
  uint32_t parts;  // CTAs (set where the kernel is launched)
};
struct HeadsArgs {
  HeadsSide side[2];
  const float2* table;
  const int32_t* at;
  unsigned long long* status;
  float* work;
  uint32_t tokens, dim, rotary, positions;
  float eps;
  bool layer, halves;
  int wdtype;
};
constexpr uint32_t kHeadDim = 8192;
size_t heads_work_floats(const HeadsArgs& a);
int launch_heads_forward(const HeadsArgs& a, int dtype, cudaStream_t stream);
int launch_heads_backward(const HeadsArgs& a, int dtype, cudaStream_t stream);
int launch_rotation_table(uint32_t positions, uint32_t rotary, double base, double scale, float2* table, cudaStream_t stream);

}  // namespace fh
