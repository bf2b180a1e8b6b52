// Host side of the C ABI's functions on 8-bit matrices, of the gated feed-forward block and of norms of heads: argument checks and launches.  None of them keeps anything
// between calls, so that they can be captured, replayed and called from several threads.
#include "../../include/fh.h"

#include <cuda_runtime.h>

#include "fh_checks.cuh"
#include "fh_i8.cuh"
#include "fh_i8_launch.cuh"

namespace {

using namespace fh;

bool finite(float f) { return f >= -3.4028235e38f && f <= 3.4028235e38f; }

int check_gated(const fh_gated_desc* d) {
  if (!d || !is_dtype(d->dtype) || d->rows < 1 || d->width < 1 || d->width > INT32_MAX / 2 || d->reserved != 0) return FH_ERR_ARG;
  if (d->activation < FH_SILU || d->activation > FH_RELU) return FH_ERR_ARG;
  if (d->ldh < d->width || d->ldp < 2ll * d->width || d->ldh > (INT64_MAX >> 3) / d->rows || d->ldp > (INT64_MAX >> 3) / d->rows) return FH_ERR_ARG;
  return FH_OK;
}

// ---- heads: rows of `dim` elements, token by token and head by head ----
struct HeadRows {
  const uint8_t* p;
  int64_t tokens, heads, token, head, dim;  // strides in elements
  int dtype;
  // All rows of a head.
  Rows of_head(int64_t h) const { return Rows(p + h * head * (int64_t)esize_of(dtype), tokens, dim, std::max(token, dim), dtype); }
  // Whether rows keep apart: all heads of a token within its stride, or all tokens of a head within its.
  bool apart() const {
    if (tokens > 1 && token < dim) return false;
    if (heads > 1 && head < dim) return false;
    return tokens == 1 || heads == 1 || token >= (heads - 1) * head + dim || head >= (tokens - 1) * token + dim;
  }
  // The rows with what lies between the heads of a token, or the tokens of a head.
  Rows coarse() const {
    if (tokens == 1) return Rows(p, heads, dim, std::max(head, dim), dtype);
    if (heads == 1 || token >= (heads - 1) * head + dim) return Rows(p, tokens, (heads - 1) * head + dim, token, dtype);
    return Rows(p, heads, (tokens - 1) * token + dim, head, dtype);
  }
};
// Whether rows of heads have a byte in common.  (Between the heads of one lie those of the other where queries, keys and values alternate.)
bool meet(const HeadRows& a, const HeadRows& b) {
  if (!a.p || !b.p || !a.heads || !b.heads || !meet(a.coarse(), b.coarse())) return false;
  for (int64_t i = 0; i < a.heads; ++i)
    for (int64_t j = 0; j < b.heads; ++j)
      if (meet(a.of_head(i), b.of_head(j))) return true;
  return false;
}
bool meet(const Rows& a, const HeadRows& b) {
  if (!a.at || !b.p || !b.heads || !meet(a, b.coarse())) return false;
  for (int64_t j = 0; j < b.heads; ++j)
    if (meet(a, b.of_head(j))) return true;
  return false;
}
bool same_strides(const HeadRows& a, const HeadRows& b) { return (a.tokens == 1 || a.token == b.token) && (a.heads == 1 || a.head == b.head); }

struct Heads {
  HeadRows q, k, q_out, k_out;  // (without addresses)
  explicit Heads(const fh_heads_desc* d)
      : q{nullptr, d->tokens, d->q_heads, d->q_token, d->q_head, d->dim, d->dtype},
        k{nullptr, d->tokens, d->k_heads, d->k_token, d->k_head, d->dim, d->dtype},
        q_out{nullptr, d->tokens, d->q_heads, d->q_out_token, d->q_out_head, d->dim, d->dtype},
        k_out{nullptr, d->tokens, d->k_heads, d->k_out_token, d->k_out_head, d->dim, d->dtype} {}
};
HeadRows at(HeadRows r, const void* p) {
  r.p = (const uint8_t*)p;
  return r;
}

int check_heads(const fh_heads_desc* d) {
  if (!d || !is_dtype(d->dtype) || !is_dtype(d->wdtype) || d->reserved != 0) return FH_ERR_ARG;
  if ((d->kind != FH_HEADS_RMS && d->kind != FH_HEADS_LAYER) || (d->pairs != FH_PAIRS_HALVES && d->pairs != FH_PAIRS_NEIGHBOURS)) return FH_ERR_ARG;
  if (d->tokens < 1 || d->dim < 1 || d->q_heads < 0 || d->k_heads < 0 || (!d->q_heads && !d->k_heads)) return FH_ERR_ARG;
  if (d->rotary < 0 || d->rotary > d->dim || d->rotary % 2 || (d->rotary && d->positions < 1)) return FH_ERR_ARG;
  if (!(d->eps >= 0.0f && d->eps <= 3.4028235e38f)) return FH_ERR_ARG;
  const Heads h(d);
  for (const HeadRows* r : {&h.q, &h.k, &h.q_out, &h.k_out}) {
    if (!r->heads) continue;
    // (addresses are formed in 64 bits of bytes)
    if (r->token < 0 || r->head < 0 || r->token > (INT64_MAX >> 4) / r->tokens || r->head > (INT64_MAX >> 4) / r->heads || !r->apart()) return FH_ERR_ARG;
  }
  return (uint32_t)d->dim > kHeadDim ? FH_ERR_UNSUPPORTED : FH_OK;
}

HeadsArgs heads_args(const fh_heads_desc* d) {
  HeadsArgs a = {};
  a.side[0].heads = (uint32_t)d->q_heads;
  a.side[0].token = (uint64_t)d->q_token;
  a.side[0].head = (uint64_t)d->q_head;
  a.side[0].out_token = (uint64_t)d->q_out_token;
  a.side[0].out_head = (uint64_t)d->q_out_head;
  a.side[1].heads = (uint32_t)d->k_heads;
  a.side[1].token = (uint64_t)d->k_token;
  a.side[1].head = (uint64_t)d->k_head;
  a.side[1].out_token = (uint64_t)d->k_out_token;
  a.side[1].out_head = (uint64_t)d->k_out_head;
  a.tokens = (uint32_t)d->tokens;
  a.dim = (uint32_t)d->dim;
  a.rotary = (uint32_t)d->rotary;
  a.positions = (uint32_t)d->positions;
  a.eps = d->eps;
  a.layer = d->kind == FH_HEADS_LAYER;
  a.halves = d->pairs == FH_PAIRS_HALVES;
  a.wdtype = d->wdtype;
  return a;
}

// What both passes are given besides rows of heads.
int check_turn(const fh_heads_desc* d, const float* table, const int32_t* positions, const uint64_t* status) {
  if (d->rotary && (!table || misaligned(table, 8) || misaligned(positions, 4) || (!positions && d->tokens > d->positions))) return FH_ERR_ARG;
  return misaligned(status, 8) ? FH_ERR_ARG : FH_OK;
}
size_t table_bytes(const fh_heads_desc* d) { return (size_t)d->positions * (size_t)(d->rotary / 2) * 8; }

}  // namespace

extern "C" {

size_t fh_i8_bytes(int32_t rows, int32_t cols) {
  // (padded extents stay below 2^32)
  if (rows < 1 || cols < 1) return 0;
  return (size_t)I8Layout((uint32_t)rows, (uint32_t)cols).total;
}

int fh_i8_compress(const fh_matrix* matrix, const void* d_src, void* d_rows, size_t rows_capacity, void* d_cols, size_t cols_capacity, void* stream) {
  int rc = check_matrix(matrix);
  if (rc != FH_OK) return rc;
  if (!d_src || (!d_rows && !d_cols) || misaligned(d_src, esize_of(matrix->dtype)) || misaligned(d_rows, 16) || misaligned(d_cols, 16)) return FH_ERR_ARG;
  const size_t by_rows = fh_i8_bytes(matrix->rows, matrix->cols), by_cols = fh_i8_bytes(matrix->cols, matrix->rows);
  if ((d_rows && rows_capacity < by_rows) || (d_cols && cols_capacity < by_cols)) return FH_ERR_CAPACITY;
  const Rows in(d_src, matrix->rows, matrix->cols, matrix->ld, matrix->dtype);
  if (overlap(d_rows, by_rows, d_cols, by_cols) || meets(in, Rows(d_rows, by_rows), Rows(d_cols, by_cols))) return FH_ERR_ARG;
  I8SaveArgs a = {};
  a.src = (const uint8_t*)d_src;
  a.rows = (uint32_t)matrix->rows;
  a.cols = (uint32_t)matrix->cols;
  a.ld = (uint64_t)matrix->ld;
  if (d_rows) {
    a.dst = (uint8_t*)d_rows;
    rc = launch_i8_rows(a, matrix->dtype, (cudaStream_t)stream);
  }
  if (d_cols && rc == FH_OK) {
    a.dst = (uint8_t*)d_cols;
    rc = launch_i8_cols(a, matrix->dtype, (cudaStream_t)stream);
  }
  return rc;
}

int fh_i8_decompress(const void* d_src, size_t src_bytes, const fh_matrix* expect, void* d_dst, uint64_t* d_status, void* stream) {
  const int rc = check_matrix(expect);
  if (rc != FH_OK) return rc;
  if (!d_src || !d_dst || misaligned(d_src, 16) || misaligned(d_dst, esize_of(expect->dtype)) || misaligned(d_status, 8)) return FH_ERR_ARG;
  const Rows in(d_src, fh_i8_bytes(expect->rows, expect->cols)), out(d_dst, expect->rows, expect->cols, expect->ld, expect->dtype);
  if (meet(in, out) || meets(Rows(d_status, 8), in, out)) return FH_ERR_ARG;
  I8SaveArgs a = {};
  a.src = (const uint8_t*)d_src;
  a.src_bytes = src_bytes;
  a.dst = (uint8_t*)d_dst;
  a.status = (unsigned long long*)d_status;
  a.rows = (uint32_t)expect->rows;
  a.cols = (uint32_t)expect->cols;
  a.ld = (uint64_t)expect->ld;
  return launch_i8_decompress(a, expect->dtype, (cudaStream_t)stream);
}

int fh_i8_product(const fh_i8_product_desc* desc, const void* d_a, size_t a_bytes, const void* d_b, size_t b_bytes, void* d_c, uint64_t* d_status,
                  void* stream) {
  if (!desc || !is_dtype(desc->dtype) || desc->m < 1 || desc->n < 1 || desc->k < 1) return FH_ERR_ARG;
  if ((desc->accumulate != 0 && desc->accumulate != 1) || desc->ldc < desc->n || desc->ldc > (INT64_MAX >> 3) / desc->m || !finite(desc->alpha)) return FH_ERR_ARG;
  if (desc->k > FH_I8_MAX_K) return FH_ERR_UNSUPPORTED;
  if (!d_a || !d_b || !d_c || misaligned(d_a, 16) || misaligned(d_b, 16) || misaligned(d_c, esize_of(desc->dtype)) || misaligned(d_status, 8))
    return FH_ERR_ARG;
  const Rows a_in(d_a, fh_i8_bytes(desc->m, desc->k)), b_in(d_b, fh_i8_bytes(desc->n, desc->k)), out(d_c, desc->m, desc->n, desc->ldc, desc->dtype);
  if (meets(out, a_in, b_in) || meets(Rows(d_status, 8), a_in, b_in, out)) return FH_ERR_ARG;
  I8ProductArgs a = {};
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
  debug_waits(&a.polls, &a.silent);
  return launch_i8_product(a, desc->dtype, (cudaStream_t)stream);
}

int fh_i8_gated(const fh_gated_desc* desc, const void* d_x, size_t x_bytes, const void* d_gate, size_t gate_bytes, const void* d_up, size_t up_bytes,
                void* d_h, void* d_pre, uint64_t* d_status, void* stream) {
  const int rc = check_gated(desc);
  if (rc != FH_OK) return rc;
  if (desc->k < 1) return FH_ERR_ARG;
  if (desc->k > FH_I8_MAX_K) return FH_ERR_UNSUPPORTED;
  const size_t es = esize_of(desc->dtype);
  if (!d_x || !d_gate || !d_up || (!d_h && !d_pre) || misaligned(d_x, 16) || misaligned(d_gate, 16) || misaligned(d_up, 16) || misaligned(d_h, es) ||
      misaligned(d_pre, es) || misaligned(d_status, 8))
    return FH_ERR_ARG;
  const size_t weight = fh_i8_bytes(desc->width, desc->k);
  const Rows x(d_x, fh_i8_bytes(desc->rows, desc->k)), gate(d_gate, weight), up(d_up, weight);
  const Rows h(d_h, desc->rows, desc->width, desc->ldh, desc->dtype), pre(d_pre, desc->rows, 2ll * desc->width, desc->ldp, desc->dtype);
  if (meets(h, x, gate, up, pre) || meets(pre, x, gate, up) || meets(Rows(d_status, 8), x, gate, up, h, pre)) return FH_ERR_ARG;
  I8ProductArgs a = {};
  a.a = (const uint8_t*)d_x;
  a.b = (const uint8_t*)d_gate;
  a.up = (const uint8_t*)d_up;
  a.a_bytes = x_bytes;
  a.b_bytes = gate_bytes;
  a.up_bytes = up_bytes;
  a.c = (uint8_t*)d_h;
  a.pre = (uint8_t*)d_pre;
  a.status = (unsigned long long*)d_status;
  a.m = (uint32_t)desc->rows;
  a.n = (uint32_t)desc->width;
  a.k = (uint32_t)desc->k;
  a.ldc = (uint64_t)desc->ldh;
  a.ldp = (uint64_t)desc->ldp;
  a.alpha = 1.0f;
  debug_waits(&a.polls, &a.silent);
  return launch_i8_gated(a, desc->dtype, desc->activation, (cudaStream_t)stream);
}

int fh_gated_backward(const fh_gated_desc* desc, const void* d_dh, const void* d_pre, void* d_dpre, void* d_packed, size_t packed_capacity, void* stream) {
  const int rc = check_gated(desc);
  if (rc != FH_OK) return rc;
  const size_t es = esize_of(desc->dtype), packed_bytes = fh_i8_bytes(desc->rows, 2 * desc->width);
  if (!d_dh || !d_pre || (!d_dpre && !d_packed) || misaligned(d_dh, es) || misaligned(d_pre, es) || misaligned(d_dpre, es) || misaligned(d_packed, 16))
    return FH_ERR_ARG;
  if (d_packed && packed_capacity < packed_bytes) return FH_ERR_CAPACITY;
  const Rows dh(d_dh, desc->rows, desc->width, desc->ldh, desc->dtype), pre(d_pre, desc->rows, 2ll * desc->width, desc->ldp, desc->dtype);
  const Rows dpre(d_dpre, desc->rows, 2ll * desc->width, desc->ldp, desc->dtype), packed(d_packed, packed_bytes);
  if (meet(dpre, dh) || (d_dpre != d_pre && meet(dpre, pre)) || meets(packed, dh, pre, dpre)) return FH_ERR_ARG;
  GatedArgs a = {};
  a.dh = (const uint8_t*)d_dh;
  a.pre = (const uint8_t*)d_pre;
  a.dpre = (uint8_t*)d_dpre;
  a.packed = (uint8_t*)d_packed;
  a.rows = (uint32_t)desc->rows;
  a.width = (uint32_t)desc->width;
  a.ldh = (uint64_t)desc->ldh;
  a.ldp = (uint64_t)desc->ldp;
  return launch_gated_backward(a, desc->dtype, desc->activation, (cudaStream_t)stream);
}

int fh_rotation_table(int32_t positions, int32_t rotary, double base, double scale, float* d_table, void* stream) {
  if (positions < 1 || rotary < 2 || rotary % 2 || !(base > 0.0 && base <= 1.7976931348623157e308) || !(scale >= -1.7976931348623157e308 && scale <= 1.7976931348623157e308) ||
      !d_table || misaligned(d_table, 8))
    return FH_ERR_ARG;
  return launch_rotation_table((uint32_t)positions, (uint32_t)rotary, base, scale, (float2*)d_table, (cudaStream_t)stream);
}

int fh_head_norm(const fh_heads_desc* desc, const void* d_q, const void* d_k, const void* d_gamma_q, const void* d_gamma_k, const float* d_table,
                 const int32_t* d_positions, void* d_q_out, void* d_k_out, uint64_t* d_status, void* stream) {
  int rc = check_heads(desc);
  if (rc != FH_OK) return rc;
  rc = check_turn(desc, d_table, d_positions, d_status);
  if (rc != FH_OK) return rc;
  const size_t es = esize_of(desc->dtype), ws = esize_of(desc->wdtype);
  if ((desc->q_heads && (!d_q || !d_q_out)) || (desc->k_heads && (!d_k || !d_k_out)) || misaligned(d_q, es) || misaligned(d_k, es) || misaligned(d_q_out, es) ||
      misaligned(d_k_out, es) || misaligned(d_gamma_q, ws) || misaligned(d_gamma_k, ws))
    return FH_ERR_ARG;
  {
    const Heads h(desc);
    const HeadRows q = at(h.q, d_q), k = at(h.k, d_k), qo = at(h.q_out, d_q_out), ko = at(h.k_out, d_k_out);
    const Rows gq(d_gamma_q, desc->dim * ws), gk(d_gamma_k, desc->dim * ws), table(desc->rotary ? d_table : nullptr, table_bytes(desc)),
        places(desc->rotary ? d_positions : nullptr, desc->tokens * 4ull), status(d_status, 8);
    const bool over_q = d_q_out == d_q && same_strides(h.q, h.q_out), over_k = d_k_out == d_k && same_strides(h.k, h.k_out);
    if ((!over_q && meet(qo, q)) || (!over_k && meet(ko, k)) || meet(qo, k) || meet(ko, q) || meet(qo, ko)) return FH_ERR_ARG;
    for (const Rows* r : {&gq, &gk, &table, &places, &status})
      if (meet(*r, qo) || meet(*r, ko) || (r != &status && fh::meet(*r, status))) return FH_ERR_ARG;
    if (meet(status, q) || meet(status, k)) return FH_ERR_ARG;
  }
  HeadsArgs a = heads_args(desc);
  a.side[0].x = (const uint8_t*)d_q;
  a.side[1].x = (const uint8_t*)d_k;
  a.side[0].gamma = (const uint8_t*)d_gamma_q;
  a.side[1].gamma = (const uint8_t*)d_gamma_k;
  a.side[0].out = (uint8_t*)d_q_out;
  a.side[1].out = (uint8_t*)d_k_out;
  a.table = (const float2*)d_table;
  a.at = d_positions;
  a.status = (unsigned long long*)d_status;
  return launch_heads_forward(a, desc->dtype, (cudaStream_t)stream);
}

size_t fh_head_norm_work_bytes(const fh_heads_desc* desc) {
  if (check_heads(desc) != FH_OK) return 0;
  return heads_work_floats(heads_args(desc)) * sizeof(float);
}

int fh_head_norm_backward(const fh_heads_desc* desc, const void* d_dq_out, const void* d_dk_out, const void* d_q, const void* d_k, const void* d_gamma_q,
                          const void* d_gamma_k, const float* d_table, const int32_t* d_positions, void* d_dq, void* d_dk, void* d_dgamma_q,
                          void* d_dgamma_k, void* d_work, size_t work_bytes, uint64_t* d_status, void* stream) {
  int rc = check_heads(desc);
  if (rc != FH_OK) return rc;
  rc = check_turn(desc, d_table, d_positions, d_status);
  if (rc != FH_OK) return rc;
  const size_t es = esize_of(desc->dtype), ws = esize_of(desc->wdtype);
  if ((desc->q_heads && (!d_q || !d_dq_out)) || (desc->k_heads && (!d_k || !d_dk_out)) || (!d_dq && !d_dk && !d_dgamma_q && !d_dgamma_k)) return FH_ERR_ARG;
  if ((!desc->q_heads && (d_dq || d_dgamma_q)) || (!desc->k_heads && (d_dk || d_dgamma_k))) return FH_ERR_ARG;
  for (const void* p : {d_dq_out, d_dk_out, d_q, d_k, (const void*)d_dq, (const void*)d_dk})
    if (misaligned(p, es)) return FH_ERR_ARG;
  for (const void* p : {d_gamma_q, d_gamma_k, (const void*)d_dgamma_q, (const void*)d_dgamma_k})
    if (misaligned(p, ws)) return FH_ERR_ARG;
  const bool weights = d_dgamma_q || d_dgamma_k;
  const size_t room = fh_head_norm_work_bytes(desc);
  if (weights) {
    if (!d_work || misaligned(d_work, 16)) return FH_ERR_ARG;
    if (work_bytes < room) return FH_ERR_CAPACITY;
  }
  {
    const Heads h(desc);
    const HeadRows q = at(h.q, d_q), k = at(h.k, d_k), yq = at(h.q_out, d_dq_out), yk = at(h.k_out, d_dk_out), dq = at(h.q, d_dq), dk = at(h.k, d_dk);
    const Rows gq(d_gamma_q, desc->dim * ws), gk(d_gamma_k, desc->dim * ws), table(desc->rotary ? d_table : nullptr, table_bytes(desc)),
        places(desc->rotary ? d_positions : nullptr, desc->tokens * 4ull), status(d_status, 8), work(weights ? d_work : nullptr, room),
        wq(d_dgamma_q, desc->dim * ws), wk(d_dgamma_k, desc->dim * ws);
    // (in place of one of its side's inputs; the other one is still another's)
    const bool on_q = d_dq == d_q, on_yq = d_dq == d_dq_out && same_strides(h.q, h.q_out), on_k = d_dk == d_k, on_yk = d_dk == d_dk_out && same_strides(h.k, h.k_out);
    if ((!on_q && meet(dq, q)) || (!on_yq && meet(dq, yq)) || (!on_k && meet(dk, k)) || (!on_yk && meet(dk, yk))) return FH_ERR_ARG;
    if (meet(dq, k) || meet(dq, yk) || meet(dk, q) || meet(dk, yq) || meet(dq, dk)) return FH_ERR_ARG;
    const Rows* small[] = {&gq, &gk, &table, &places, &status, &work, &wq, &wk};
    for (const Rows* r : small) {
      if (meet(*r, dq) || meet(*r, dk)) return FH_ERR_ARG;
      const bool written = r == &status || r == &work || r == &wq || r == &wk;
      if (!written) continue;
      if (meet(*r, q) || meet(*r, k) || meet(*r, yq) || meet(*r, yk)) return FH_ERR_ARG;
      for (const Rows* o : small)
        if (o != r && fh::meet(*r, *o)) return FH_ERR_ARG;
    }
  }
  HeadsArgs a = heads_args(desc);
  a.side[0].x = (const uint8_t*)d_q;
  a.side[1].x = (const uint8_t*)d_k;
  a.side[0].gamma = (const uint8_t*)d_gamma_q;
  a.side[1].gamma = (const uint8_t*)d_gamma_k;
  a.side[0].dy = (const uint8_t*)d_dq_out;
  a.side[1].dy = (const uint8_t*)d_dk_out;
  a.side[0].dx = (uint8_t*)d_dq;
  a.side[1].dx = (uint8_t*)d_dk;
  a.side[0].dgamma = (uint8_t*)d_dgamma_q;
  a.side[1].dgamma = (uint8_t*)d_dgamma_k;
  a.table = (const float2*)d_table;
  a.at = d_positions;
  a.status = (unsigned long long*)d_status;
  a.work = weights ? (float*)d_work : nullptr;
  return launch_heads_backward(a, desc->dtype, (cudaStream_t)stream);
}

}  // extern "C"
