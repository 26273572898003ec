// C ABI of the cache in 8 bits.  Argument checks and launches.
#include "api_checks.h"

using namespace ts;

extern "C" {

int32_t ts_quant_append(const ts_problem* p, const ts_quant* c, const ts_rope* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const void* v, int64_t v_stride, const int32_t* q_indptr, int32_t num_rows, const int32_t* positions, void* q_out, void* stream) {
  QuantPools pools;
  int32_t st = check_quant(p, c, &pools);
  if (st != TS_OK) return st;
  if ((st = check_rows(p, q_indptr, num_rows)) != TS_OK) return st;
  if ((st = check_rope(r, p->head_dim)) != TS_OK) return st;
  if (num_rows == 0) return TS_OK;
  if ((q == nullptr) != (q_out == nullptr) || k == nullptr || v == nullptr) return TS_ERR_INVALID_ARG;
  if ((st = check_append_rows(p, q, &q_stride, k, &k_stride, v, &v_stride, num_rows, q_out)) != TS_OK) return st;
  const int64_t es = p->dtype == TS_BF16 ? 2 : 4;
  RopeAppendArgs a{};
  a.q = (const uint8_t*)q; a.k = (const uint8_t*)k; a.v = (const uint8_t*)v; a.q_out = (uint8_t*)q_out;
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens; a.q_indptr = q_indptr;
  a.positions = positions;
  a.q_stride = q_stride * es; a.k_stride = k_stride * es; a.v_stride = v_stride * es;
  a.B = p->batch; a.C = p->chunk; a.T = num_rows; a.H = p->num_q_heads; a.H_kv = p->num_kv_heads; a.D = p->head_dim;
  a.P = p->page_size; a.p_shift = ilog2(p->page_size); a.max_seq_len = p->max_seq_len;
  if (r != nullptr) {
    a.inv_freq = r->inv_freq; a.rotary = r->rotary_dim; a.adjacent = r->adjacent; a.scale = r->scale;
    for (int i = 0; i < r->rotary_dim / 2; ++i) a.pair_axis[i] = r->pair_axis[i];
  }
  return launch_quant_append(p->dtype, a, pools, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int32_t ts_quant_read(const ts_problem* p, const ts_quant* c, const int32_t* q_indptr, int32_t num_rows, void* k_out, void* v_out, void* stream) {
  QuantPools pools;
  int32_t st = check_quant(p, c, &pools);
  if (st != TS_OK) return st;
  if ((st = check_rows(p, q_indptr, num_rows)) != TS_OK) return st;
  if (num_rows == 0) return TS_OK;
  if ((k_out == nullptr && v_out == nullptr) || !aligned16(k_out) || !aligned16(v_out)) return TS_ERR_INVALID_ARG;
  const size_t bytes = (size_t)num_rows * p->num_kv_heads * p->head_dim * (p->dtype == TS_BF16 ? 2 : 4);
  if (k_out != nullptr && v_out != nullptr && overlap(k_out, bytes, v_out, bytes)) return TS_ERR_INVALID_ARG;
  QuantReadArgs a{};
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens; a.q_indptr = q_indptr;
  a.k_out = (uint8_t*)k_out; a.v_out = (uint8_t*)v_out;
  a.B = p->batch; a.C = p->chunk; a.T = num_rows; a.H_kv = p->num_kv_heads; a.D = p->head_dim;
  a.P = p->page_size; a.p_shift = ilog2(p->page_size); a.max_seq_len = p->max_seq_len;
  return launch_quant_read(p->dtype, a, pools, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int32_t ts_quant_pages_copy(const ts_problem* p, const ts_quant* c, const int32_t* src, const int32_t* dst, int32_t n, int32_t num_pages, void* stream) {
  QuantPools pools;
  const int32_t st = check_quant(p, c, &pools);
  if (st != TS_OK) return st;
  if (n < 0 || num_pages < 1) return TS_ERR_INVALID_ARG;
  if (n == 0) return TS_OK;
  if (src == nullptr || dst == nullptr) return TS_ERR_INVALID_ARG;
  return launch_quant_pages_copy(pools, src, dst, n, num_pages, p->page_size, p->num_kv_heads, p->head_dim, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

}  // extern "C"
