// Host side of the C ABI's functions on microscaled 4-bit matrices: argument checks and launches.  None of them keeps anything between
// calls, so that they can be captured, replayed and called from several threads.
#include "../../include/fh.h"

#include <cuda_runtime.h>

#include "fh_checks.cuh"
#include "fh_launch.cuh"
#include "fh_mx.cuh"
#include "fh_mx_launch.cuh"

namespace {

using namespace fh;

bool is_format(int format) { return format == FH_MX_B32 || format == FH_MX_B16; }

int check_mx(const fh_mx_params* p) {
  if (!p || !is_format(p->format) || p->reserved != 0) return FH_ERR_ARG;
  if (p->rounding != 0 && p->rounding != 1) return FH_ERR_UNSUPPORTED;
  if (p->format == FH_MX_B32 ? p->exponent != 0 : (p->exponent < -64 || p->exponent > 64)) return FH_ERR_ARG;
  return FH_OK;
}

int check_norm(const fh_norm_desc* d) {
  if (!d || !is_dtype(d->dtype) || !is_dtype(d->wdtype) || d->rows < 1 || d->cols < 1 || d->reserved != 0) return FH_ERR_ARG;
  if (d->ldx < d->cols || d->ldy < d->cols || d->ldx > (INT64_MAX >> 3) / d->rows || d->ldy > (INT64_MAX >> 3) / d->rows) return FH_ERR_ARG;
  if (!(d->eps >= 0.0f && d->eps <= 3.4028235e38f)) return FH_ERR_ARG;
  return (uint32_t)d->cols > fh::kNormCols ? FH_ERR_UNSUPPORTED : FH_OK;
}

fh::NormArgs norm_args(const fh_norm_desc* d) {
  fh::NormArgs a = {};
  a.rows = (uint32_t)d->rows;
  a.cols = (uint32_t)d->cols;
  a.ldx = (uint64_t)d->ldx;
  a.ldy = (uint64_t)d->ldy;
  a.wdtype = d->wdtype;
  a.eps = d->eps;
  return a;
}

}  // namespace

extern "C" {

size_t fh_mx_bytes(int32_t rows, int32_t cols, int32_t format) {
  // (padded extents stay below 2^32)
  if (rows < 1 || cols < 1 || !is_format(format)) return 0;
  return (size_t)fh::MxLayout((uint32_t)rows, (uint32_t)cols, (uint32_t)format).total;
}

int fh_mx_compress(const fh_matrix* matrix, const fh_mx_params* params, const void* d_src, void* d_rows, size_t rows_capacity,
                   void* d_cols, size_t cols_capacity, void* stream) {
  int rc = check_matrix(matrix);
  if (rc != FH_OK) return rc;
  rc = check_mx(params);
  if (rc != FH_OK) return rc;
  if (!d_src || (!d_rows && !d_cols) || misaligned(d_src, esize_of(matrix->dtype)) || misaligned(d_rows, 16) || misaligned(d_cols, 16))
    return FH_ERR_ARG;
  if (d_rows && rows_capacity < fh_mx_bytes(matrix->rows, matrix->cols, params->format)) return FH_ERR_CAPACITY;
  if (d_cols && cols_capacity < fh_mx_bytes(matrix->cols, matrix->rows, params->format)) return FH_ERR_CAPACITY;
  const size_t in = extent(matrix->rows, matrix->cols, matrix->ld, matrix->dtype), by_rows = fh_mx_bytes(matrix->rows, matrix->cols, params->format),
               by_cols = fh_mx_bytes(matrix->cols, matrix->rows, params->format);
  if (overlap(d_rows, by_rows, d_cols, by_cols) || overlap(d_src, in, d_rows, by_rows) || overlap(d_src, in, d_cols, by_cols)) return FH_ERR_ARG;
  fh::MxSaveArgs a = {};
  a.src = (const uint8_t*)d_src;
  a.by_rows = (uint8_t*)d_rows;
  a.by_cols = (uint8_t*)d_cols;
  a.rows = (uint32_t)matrix->rows;
  a.cols = (uint32_t)matrix->cols;
  a.ld = (uint64_t)matrix->ld;
  a.exponent = params->exponent;
  for (uint32_t r = 0; r < 10; ++r) {
    a.round_keys[2 * r] = (uint32_t)params->seed + r * 0x9E3779B9u;
    a.round_keys[2 * r + 1] = (uint32_t)(params->seed >> 32) + r * 0xBB67AE85u;
  }
  a.tensor_id = params->tensor_id;
  return fh::launch_mx_save(a, matrix->dtype, params->format, true, params->rounding == 1, (cudaStream_t)stream);
}

int fh_mx_decompress(const void* d_src, size_t src_bytes, const fh_matrix* expect, int32_t format, void* d_dst, uint64_t* d_status,
                     void* stream) {
  const int rc = check_matrix(expect);
  if (rc != FH_OK) return rc;
  if (!is_format(format) || !d_src || !d_dst || misaligned(d_src, 16) || misaligned(d_dst, esize_of(expect->dtype)) || misaligned(d_status, 8))
    return FH_ERR_ARG;
  if (overlap(d_src, fh_mx_bytes(expect->rows, expect->cols, format), d_dst, extent(expect->rows, expect->cols, expect->ld, expect->dtype)))
    return FH_ERR_ARG;
  if (meets(Rows(d_status, 8), Rows(d_src, fh_mx_bytes(expect->rows, expect->cols, format)), Rows(d_dst, expect->rows, expect->cols, expect->ld, expect->dtype)))
    return FH_ERR_ARG;
  fh::MxSaveArgs a = {};
  a.src = (const uint8_t*)d_src;
  a.src_bytes = src_bytes;
  a.dst = (uint8_t*)d_dst;
  a.status = (unsigned long long*)d_status;
  a.rows = (uint32_t)expect->rows;
  a.cols = (uint32_t)expect->cols;
  a.ld = (uint64_t)expect->ld;
  return fh::launch_mx_save(a, expect->dtype, format, false, false, (cudaStream_t)stream);
}

int fh_mx_product(const fh_mx_product_desc* desc, const void* d_a, size_t a_bytes, const void* d_b, size_t b_bytes, void* d_c,
                  uint64_t* d_status, void* stream) {
  if (!desc || !is_format(desc->format) || !is_dtype(desc->dtype) || desc->m < 1 || desc->n < 1 || desc->k < 1) return FH_ERR_ARG;
  if ((desc->accumulate != 0 && desc->accumulate != 1) || desc->reserved != 0 || desc->ldc < desc->n ||
      desc->ldc > (INT64_MAX >> 3) / desc->m)
    return FH_ERR_ARG;
  if (!(desc->alpha >= -3.4028235e38f && desc->alpha <= 3.4028235e38f)) return FH_ERR_ARG;
  if (!d_a || !d_b || !d_c || misaligned(d_a, 16) || misaligned(d_b, 16) || misaligned(d_c, esize_of(desc->dtype)) || misaligned(d_status, 8))
    return FH_ERR_ARG;
  const size_t out = extent(desc->m, desc->n, desc->ldc, desc->dtype);
  if (overlap(d_c, out, d_a, fh_mx_bytes(desc->m, desc->k, desc->format)) || overlap(d_c, out, d_b, fh_mx_bytes(desc->n, desc->k, desc->format)))
    return FH_ERR_ARG;
  if (meets(Rows(d_status, 8), Rows(d_a, fh_mx_bytes(desc->m, desc->k, desc->format)), Rows(d_b, fh_mx_bytes(desc->n, desc->k, desc->format)),
            Rows(d_c, desc->m, desc->n, desc->ldc, desc->dtype)))
    return FH_ERR_ARG;
  fh::MxProductArgs a = {};
  a.a = (const uint8_t*)d_a;
  a.b = (const uint8_t*)d_b;
  a.a_bytes = a_bytes;
  a.b_bytes = b_bytes;
  a.c = (uint8_t*)d_c;
  a.status = (unsigned long long*)d_status;
  a.m = (uint32_t)desc->m;
  a.n = (uint32_t)desc->n;
  a.k = (uint32_t)desc->k;
  a.ldc = (uint64_t)desc->ldc;
  a.alpha = desc->alpha;
  a.accumulate = desc->accumulate == 1;
  fh::debug_waits(&a.polls, &a.silent);
  return fh::launch_mx_product(a, desc->dtype, desc->format, (cudaStream_t)stream);
}

int fh_layer_norm(const fh_norm_desc* desc, const void* d_x, const void* d_gamma, const void* d_beta, void* d_y, float* d_mean,
                  float* d_rstd, const fh_mx_params* params, void* d_packed, size_t packed_capacity, void* stream) {
  int rc = check_norm(desc);
  if (rc != FH_OK) return rc;
  const size_t es = esize_of(desc->dtype), ws = esize_of(desc->wdtype);
  if (!d_x || (!d_y && !d_packed) || misaligned(d_x, es) || misaligned(d_y, es) || misaligned(d_gamma, ws) || misaligned(d_beta, ws) ||
      misaligned(d_mean, 4) || misaligned(d_rstd, 4) || misaligned(d_packed, 16))
    return FH_ERR_ARG;
  fh::NormArgs a = norm_args(desc);
  if (d_packed) {
    rc = check_mx(params);
    if (rc != FH_OK) return rc;
    if (params->rounding != 0) return FH_ERR_UNSUPPORTED;
    const size_t n = fh_mx_bytes(desc->rows, desc->cols, params->format);
    if (packed_capacity < n) return FH_ERR_CAPACITY;
    if (overlap(d_packed, n, d_x, extent(desc->rows, desc->cols, desc->ldx, desc->dtype)) ||
        overlap(d_packed, n, d_y, extent(desc->rows, desc->cols, desc->ldy, desc->dtype)))
      return FH_ERR_ARG;
    a.packed = (uint8_t*)d_packed;
    a.format = (uint32_t)params->format;
    a.exponent = params->exponent;
    a.tensor_id = params->tensor_id;
  }
  const Rows x(d_x, desc->rows, desc->cols, desc->ldx, desc->dtype), y(d_y, desc->rows, desc->cols, desc->ldy, desc->dtype);
  const Rows gamma(d_gamma, desc->cols * ws), beta(d_beta, desc->cols * ws), mean(d_mean, desc->rows * sizeof(float)), rstd(d_rstd, desc->rows * sizeof(float));
  const Rows packed(d_packed, d_packed ? fh_mx_bytes(desc->rows, desc->cols, params->format) : 1);
  const bool in_place = d_y == d_x && (desc->ldx == desc->ldy || desc->rows == 1);
  if ((!in_place && meet(y, x)) || meets(y, gamma, beta) || meets(mean, x, gamma, beta, y) || meets(rstd, x, gamma, beta, y, mean) ||
      meets(packed, gamma, beta, mean, rstd))
    return FH_ERR_ARG;
  a.x = (const uint8_t*)d_x;
  a.gamma = (const uint8_t*)d_gamma;
  a.beta = (const uint8_t*)d_beta;
  a.y = (uint8_t*)d_y;
  a.mean = d_mean;
  a.rstd = d_rstd;
  return fh::launch_norm_forward(a, desc->dtype, (cudaStream_t)stream);
}

size_t fh_layer_norm_work_bytes(const fh_norm_desc* desc) {
  if (check_norm(desc) != FH_OK) return 0;
  return (size_t)fh::norm_parts((uint32_t)desc->rows, (uint32_t)desc->cols, desc->dtype) * 2 * (size_t)desc->cols * sizeof(float);
}

int fh_layer_norm_backward(const fh_norm_desc* desc, const void* d_dy, const void* d_x, size_t x_bytes, int32_t x_format, const void* d_gamma,
                           const float* d_mean, const float* d_rstd, void* d_dx, void* d_dgamma, void* d_dbeta, void* d_work,
                           size_t work_bytes, uint64_t* d_status, void* stream) {
  const int rc = check_norm(desc);
  if (rc != FH_OK) return rc;
  const size_t es = esize_of(desc->dtype), ws = esize_of(desc->wdtype);
  if (!d_dy || !d_x || !d_mean || !d_rstd || (!d_dx && !d_dgamma && !d_dbeta) || (x_bytes && !is_format(x_format))) return FH_ERR_ARG;
  if (misaligned(d_dy, es) || misaligned(d_x, x_bytes ? 16 : es) || misaligned(d_gamma, ws) || misaligned(d_mean, 4) || misaligned(d_rstd, 4) ||
      misaligned(d_dx, es) || misaligned(d_dgamma, ws) || misaligned(d_dbeta, ws) || misaligned(d_work, 16) || misaligned(d_status, 8))
    return FH_ERR_ARG;
  fh::NormArgs a = norm_args(desc);
  const size_t dx = extent(desc->rows, desc->cols, desc->ldx, desc->dtype), weights = (size_t)desc->cols * ws;
  if ((x_bytes && overlap(d_dx, dx, d_x, fh_mx_bytes(desc->rows, desc->cols, x_format))) || overlap(d_dgamma, weights, d_dbeta, weights)) return FH_ERR_ARG;
  if (d_dgamma || d_dbeta) {
    if (!d_work) return FH_ERR_ARG;
    if (work_bytes < fh_layer_norm_work_bytes(desc)) return FH_ERR_CAPACITY;
    a.work = (float*)d_work;
  }
  {
    const Rows dy(d_dy, desc->rows, desc->cols, desc->ldy, desc->dtype), dx(d_dx, desc->rows, desc->cols, desc->ldx, desc->dtype);
    const Rows x = x_bytes ? Rows(d_x, fh_mx_bytes(desc->rows, desc->cols, x_format)) : Rows(d_x, desc->rows, desc->cols, desc->ldx, desc->dtype);
    const Rows gamma(d_gamma, weights), dgamma(d_dgamma, weights), dbeta(d_dbeta, weights), work(a.work, a.work ? fh_layer_norm_work_bytes(desc) : 1);
    const Rows mean(d_mean, desc->rows * sizeof(float)), rstd(d_rstd, desc->rows * sizeof(float)), status(d_status, 8);
    const bool over_dy = d_dx == d_dy && (desc->ldx == desc->ldy || desc->rows == 1), over_x = d_dx == d_x && !x_bytes;
    if ((!over_dy && meet(dx, dy)) || (!over_x && meet(dx, x)) || meets(dx, gamma, mean, rstd, dgamma, dbeta)) return FH_ERR_ARG;
    if (meets(work, dy, x, gamma, mean, rstd, dx, dgamma, dbeta) || meets(status, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, work)) return FH_ERR_ARG;
    // (the weights' gradients may lie over dense inputs: the second kernel writes them; a container's header it reads)
    if (x_bytes && (meet(x, dgamma) || meet(x, dbeta))) return FH_ERR_ARG;
  }
  a.dy = (const uint8_t*)d_dy;
  a.x = (const uint8_t*)d_x;
  a.x_bytes = x_bytes;
  a.format = x_bytes ? (uint32_t)x_format : 0u;
  a.gamma = (const uint8_t*)d_gamma;
  a.mean = const_cast<float*>(d_mean);
  a.rstd = const_cast<float*>(d_rstd);
  a.dx = (uint8_t*)d_dx;
  a.dgamma = (uint8_t*)d_dgamma;
  a.dbeta = (uint8_t*)d_dbeta;
  a.status = (unsigned long long*)d_status;
  return fh::launch_norm_backward(a, desc->dtype, (cudaStream_t)stream);
}

}  // extern "C"
