// Argument checks that the C entry points of the cache share.
#pragma once
#include "ts_kernels.h"
#include <math.h>

namespace ts {

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
inline bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + bn && y < x + an;
}

inline int32_t check_quant(const ts_problem* p, const ts_quant* c, QuantPools* pools) {
  const int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  if (c == nullptr || (c->code != TS_INT8 && c->code != TS_E4M3)) return TS_ERR_INVALID_ARG;
  for (const void* x : {(const void*)c->k_codes, (const void*)c->v_codes, (const void*)c->k_scale, (const void*)c->v_scale})
    if (x == nullptr || !aligned16(x)) return TS_ERR_INVALID_ARG;
  *pools = QuantPools{(uint8_t*)c->k_codes, (uint8_t*)c->v_codes, c->k_scale, c->v_scale, c->code};
  return TS_OK;
}

// rows of new tokens: without q_indptr every sequence has `chunk` of them
inline int32_t check_rows(const ts_problem* p, const int32_t* q_indptr, int32_t num_rows) {
  if (num_rows < 0) return TS_ERR_INVALID_ARG;
  if (q_indptr == nullptr && (int64_t)num_rows != (int64_t)p->batch * p->chunk && num_rows != 0) return TS_ERR_INVALID_ARG;
  return TS_OK;
}

inline int32_t check_rope(const ts_rope* r, int D) {
  if (r == nullptr) return TS_OK;
  if (r->rotary_dim < 0 || r->rotary_dim > D || (r->rotary_dim & 1) != 0) return TS_ERR_INVALID_ARG;
  if (r->num_axes < 1 || r->num_axes > TS_ROPE_MAX_AXES || (r->adjacent != 0 && r->adjacent != 1)) return TS_ERR_INVALID_ARG;
  if (!(fabsf(r->scale) < INFINITY) || (r->rotary_dim > 0 && r->inv_freq == nullptr)) return TS_ERR_INVALID_ARG;
  for (int i = 0; i < r->rotary_dim / 2; ++i)
    if (r->pair_axis[i] >= r->num_axes) return TS_ERR_INVALID_ARG;
  return TS_OK;
}

// rows q (null: none), k, v in and q_out: alignment, strides (0 = packed, filled in) and what may not overlap
inline int32_t check_append_rows(const ts_problem* p, const void* q, int64_t* q_stride, const void* k, int64_t* k_stride, const void* v, int64_t* v_stride,
                                 int32_t num_rows, const void* q_out) {
  const int64_t es = p->dtype == TS_BF16 ? 2 : 4;
  const int64_t qrow = (int64_t)p->num_q_heads * p->head_dim, krow = (int64_t)p->num_kv_heads * p->head_dim;
  if (*q_stride == 0) *q_stride = qrow;
  if (*k_stride == 0) *k_stride = krow;
  if (*v_stride == 0) *v_stride = krow;
  if (q != nullptr) {
    if (!aligned16(q) || !aligned16(q_out) || *q_stride < qrow || (*q_stride * es) % 16 != 0) return TS_ERR_INVALID_ARG;
    const size_t in = (size_t)((num_rows - 1) * *q_stride + qrow) * es, out = (size_t)num_rows * qrow * es;
    if (!(q == q_out && *q_stride == qrow) && overlap(q, in, q_out, out)) return TS_ERR_INVALID_ARG;
    if (k != nullptr) {
      // k and v are read while q_out is written: parts of one projection next to q are refused with it, q_out = q needs them apart
      if (overlap(k, (size_t)((num_rows - 1) * *k_stride + krow) * es, q_out, out) ||
          overlap(v, (size_t)((num_rows - 1) * *v_stride + krow) * es, q_out, out)) return TS_ERR_INVALID_ARG;
    }
  }
  if (k != nullptr) {
    if (!aligned16(k) || !aligned16(v)) return TS_ERR_INVALID_ARG;
    if (*k_stride < krow || *v_stride < krow || (*k_stride * es) % 16 != 0 || (*v_stride * es) % 16 != 0) return TS_ERR_INVALID_ARG;
  }
  return TS_OK;
}

}  // namespace ts
