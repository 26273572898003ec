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

int32_t ts_quant_attn_workspace_bytes(const ts_problem* p, int32_t num_rows, size_t* bytes) {
  if (bytes == nullptr || num_rows < 0) return TS_ERR_INVALID_ARG;
  const int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  *bytes = quant_attn_workspace(p->dtype, p->head_dim, p->num_q_heads / p->num_kv_heads, p->num_kv_heads, p->chunk);
  return TS_OK;
}

int32_t ts_quant_attn(const ts_problem* p, const ts_quant* c, const void* q, const int32_t* q_indptr, int32_t num_rows, int32_t window, const uint32_t* mask,
                      int32_t mask_words, float sm_scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  QuantPools pools;
  int32_t st = check_quant(p, c, &pools);
  if (st != TS_OK) return st;
  if ((st = check_rows(p, q_indptr, num_rows)) != TS_OK) return st;
  if (window < 0 || !(fabsf(sm_scale) < INFINITY)) return TS_ERR_INVALID_ARG;
  if (mask != nullptr && (mask_words < 1 || ((uintptr_t)mask & 3) != 0)) return TS_ERR_INVALID_ARG;
  if (num_rows == 0) return TS_OK;
  if (q == nullptr || out == nullptr || !aligned16(q) || !aligned16(out)) return TS_ERR_INVALID_ARG;
  const size_t es = p->dtype == TS_BF16 ? 2 : 4, bytes = (size_t)num_rows * p->num_q_heads * p->head_dim * es;
  if (overlap(q, bytes, out, bytes)) return TS_ERR_INVALID_ARG;
  const size_t need = quant_attn_workspace(p->dtype, p->head_dim, p->num_q_heads / p->num_kv_heads, p->num_kv_heads, p->chunk);
  if (ws == nullptr || ((uintptr_t)ws & 255) != 0 || ws_bytes < need) return TS_ERR_WORKSPACE;
  PagedAttnArgs a{};
  a.q = (const uint8_t*)q;
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens; a.q_indptr = q_indptr;
  a.out = (uint8_t*)out; a.lse = lse;
  a.B = p->batch; a.C = p->chunk; a.T = num_rows; a.H = p->num_q_heads; a.H_kv = p->num_kv_heads;
  a.P = p->page_size; a.p_shift = ilog2(p->page_size); a.max_seq_len = p->max_seq_len; a.window = window < p->max_seq_len ? window : 0;   // one that reaches every token is none
  a.sm_scale = sm_scale; a.mask = mask; a.mask_words = mask_words;
  return launch_quant_attn(p->dtype, p->head_dim, a, pools, ws, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
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
