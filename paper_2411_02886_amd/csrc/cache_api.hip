// C ABI of the cache's own calls: filling, attending and moving it.  Argument checks and launches.
#include "ts_kernels.h"
#include <math.h>

using namespace ts;

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }
static bool overlap(const void* a, size_t an, const void* b, size_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + bn && y < x + an;
}

// rows of new tokens: without q_indptr every sequence has `chunk` of them
static int32_t check_rows(const ts_problem* p, const int32_t* q_indptr, int32_t num_rows) {
  if (num_rows < 0) return TS_ERR_INVALID_ARG;
  if (q_indptr == nullptr && (int64_t)num_rows != (int64_t)p->batch * p->chunk && num_rows != 0) return TS_ERR_INVALID_ARG;
  return TS_OK;
}

static int32_t attend(const ts_problem* p, const void* q, const int32_t* q_indptr, int32_t num_rows, int32_t window, float sm_scale, void* out, float* lse,
                      void* ws, size_t ws_bytes, bool round_weights, void* stream) {
  int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  if ((st = check_rows(p, q_indptr, num_rows)) != TS_OK) return st;
  if (window < 0 || !(fabsf(sm_scale) < INFINITY)) return TS_ERR_INVALID_ARG;
  if (p->k_pool == nullptr || p->v_pool == nullptr) return TS_ERR_INVALID_ARG;
  if (num_rows == 0) return TS_OK;
  if (q == nullptr || out == nullptr) return TS_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(out) || !aligned16(p->k_pool) || !aligned16(p->v_pool)) return TS_ERR_INVALID_ARG;
  const size_t es = p->dtype == TS_BF16 ? 2 : 4, bytes = (size_t)num_rows * p->num_q_heads * p->head_dim * es;
  if (overlap(q, bytes, out, bytes)) return TS_ERR_INVALID_ARG;
  const size_t need = paged_attn_workspace(p->dtype, p->head_dim, p->num_q_heads / p->num_kv_heads, p->chunk);
  if (ws == nullptr || ((uintptr_t)ws & 255) != 0 || ws_bytes < need) return TS_ERR_WORKSPACE;
  PagedAttnArgs a{};
  a.q = (const uint8_t*)q; a.k_pool = (const uint8_t*)p->k_pool; a.v_pool = (const uint8_t*)p->v_pool;
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens; a.q_indptr = q_indptr;
  a.out = (uint8_t*)out; a.lse = lse;
  a.B = p->batch; a.C = p->chunk; a.T = num_rows; a.H = p->num_q_heads; a.H_kv = p->num_kv_heads;
  a.P = p->page_size; a.p_shift = ilog2(p->page_size); a.max_seq_len = p->max_seq_len; a.window = window < p->max_seq_len ? window : 0;   // one that reaches every token is none
  a.sm_scale = sm_scale; a.round_weights = round_weights ? 1 : 0;
  return launch_paged_attn(p->dtype, p->head_dim, a, ws, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

extern "C" {

int32_t ts_paged_attn_workspace_bytes(const ts_problem* p, int32_t num_rows, size_t* bytes) {
  if (bytes == nullptr || num_rows < 0) return TS_ERR_INVALID_ARG;
  const int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  *bytes = paged_attn_workspace(p->dtype, p->head_dim, p->num_q_heads / p->num_kv_heads, p->chunk);
  return TS_OK;
}

int32_t ts_paged_attn(const ts_problem* p, const void* q, const int32_t* q_indptr, int32_t num_rows, int32_t window,
                      float sm_scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return attend(p, q, q_indptr, num_rows, window, sm_scale, out, lse, ws, ws_bytes, false, stream);
}

int32_t ts_paged_attn_rounded(const ts_problem* p, const void* q, const int32_t* q_indptr, int32_t num_rows, int32_t window,
                              float sm_scale, void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  return attend(p, q, q_indptr, num_rows, window, sm_scale, out, lse, ws, ws_bytes, true, stream);
}

int32_t ts_rope_append(const ts_problem* p, const ts_rope* r, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                       const void* v, int64_t v_stride, const int32_t* q_indptr, int32_t num_rows, const int32_t* positions,
                       void* q_out, void* stream) {
  int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  if ((st = check_rows(p, q_indptr, num_rows)) != TS_OK) return st;
  const int D = p->head_dim;
  if (r != nullptr) {
    if (r->rotary_dim < 0 || r->rotary_dim > D || (r->rotary_dim & 1) != 0) return TS_ERR_INVALID_ARG;
    if (r->num_axes < 1 || r->num_axes > TS_ROPE_MAX_AXES || (r->adjacent != 0 && r->adjacent != 1)) return TS_ERR_INVALID_ARG;
    if (!(fabsf(r->scale) < INFINITY) || (r->rotary_dim > 0 && r->inv_freq == nullptr)) return TS_ERR_INVALID_ARG;
    for (int i = 0; i < r->rotary_dim / 2; ++i)
      if (r->pair_axis[i] >= r->num_axes) return TS_ERR_INVALID_ARG;
  }
  if (num_rows == 0) return TS_OK;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (v == nullptr) || (q == nullptr && k == nullptr)) return TS_ERR_INVALID_ARG;
  const int64_t es = p->dtype == TS_BF16 ? 2 : 4;
  const int64_t qrow = (int64_t)p->num_q_heads * D, krow = (int64_t)p->num_kv_heads * D;
  if (q_stride == 0) q_stride = qrow;
  if (k_stride == 0) k_stride = krow;
  if (v_stride == 0) v_stride = krow;
  if (q != nullptr) {
    if (!aligned16(q) || !aligned16(q_out) || q_stride < qrow || (q_stride * es) % 16 != 0) return TS_ERR_INVALID_ARG;
    const size_t in = (size_t)((num_rows - 1) * q_stride + qrow) * es, out = (size_t)num_rows * qrow * es;
    if (!(q == q_out && q_stride == qrow) && overlap(q, in, q_out, out)) return TS_ERR_INVALID_ARG;
    if (k != nullptr) {
      // k and v are read while q_out is written: parts of one projection next to q are refused with it, q_out = q needs them apart
      if (overlap(k, (size_t)((num_rows - 1) * k_stride + krow) * es, q_out, out) ||
          overlap(v, (size_t)((num_rows - 1) * v_stride + krow) * es, q_out, out)) return TS_ERR_INVALID_ARG;
    }
  }
  if (k != nullptr) {
    if (p->k_pool == nullptr || p->v_pool == nullptr) return TS_ERR_INVALID_ARG;
    if (!aligned16(k) || !aligned16(v) || !aligned16(p->k_pool) || !aligned16(p->v_pool)) return TS_ERR_INVALID_ARG;
    if (k_stride < krow || v_stride < krow || (k_stride * es) % 16 != 0 || (v_stride * es) % 16 != 0) return TS_ERR_INVALID_ARG;
  }
  RopeAppendArgs a{};
  a.q = (const uint8_t*)q; a.k = (const uint8_t*)k; a.v = (const uint8_t*)v; a.q_out = (uint8_t*)q_out;
  a.k_pool = (uint8_t*)const_cast<void*>(p->k_pool); a.v_pool = (uint8_t*)const_cast<void*>(p->v_pool);
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens; a.q_indptr = q_indptr;
  a.positions = positions;
  a.q_stride = q_stride * es; a.k_stride = k_stride * es; a.v_stride = v_stride * es;
  a.B = p->batch; a.C = p->chunk; a.T = num_rows; a.H = p->num_q_heads; a.H_kv = p->num_kv_heads; a.D = D;
  a.P = p->page_size; a.p_shift = ilog2(p->page_size); a.max_seq_len = p->max_seq_len;
  if (r != nullptr) {
    a.inv_freq = r->inv_freq; a.rotary = r->rotary_dim; a.adjacent = r->adjacent; a.scale = r->scale;
    for (int i = 0; i < r->rotary_dim / 2; ++i) a.pair_axis[i] = r->pair_axis[i];
  }
  return launch_rope_append(p->dtype, a, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int32_t ts_pages_copy(const ts_problem* p, const int32_t* src, const int32_t* dst, int32_t n, int32_t num_pages, void* stream) {
  const int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  if (n < 0 || num_pages < 1 || p->k_pool == nullptr) return TS_ERR_INVALID_ARG;
  if (!aligned16(p->k_pool) || !aligned16(p->v_pool)) return TS_ERR_INVALID_ARG;
  if (n == 0) return TS_OK;
  if (src == nullptr || dst == nullptr) return TS_ERR_INVALID_ARG;
  PagesCopyArgs a{};
  a.src = src; a.dst = dst; a.n = n; a.num_pages = num_pages;
  a.k_pool = (uint8_t*)const_cast<void*>(p->k_pool); a.v_pool = (uint8_t*)const_cast<void*>(p->v_pool);
  a.page_bytes = (int64_t)p->page_size * p->num_kv_heads * p->head_dim * (p->dtype == TS_BF16 ? 2 : 4);
  return launch_pages_copy(a, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int32_t ts_cache_compact(const ts_problem* p, const int32_t* idx, int32_t idx_stride, const int32_t* count, const uint8_t* skip,
                         const int32_t* to_indptr, const int32_t* to_indices, int32_t* to_lens, void* stream) {
  const int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  if (idx == nullptr || count == nullptr || idx_stride < 1 || to_indptr == nullptr || to_indices == nullptr || to_lens == nullptr)
    return TS_ERR_INVALID_ARG;
  if (p->k_pool == nullptr || p->v_pool == nullptr || !aligned16(p->k_pool) || !aligned16(p->v_pool)) return TS_ERR_INVALID_ARG;
  if (p->chunk != 1) return TS_ERR_UNSUPPORTED;
  // a sequence's first workgroup writes its new length while others still read the rest
  const size_t B = (size_t)p->batch, lens = B * 4;
  if (overlap(to_lens, lens, p->seq_lens, lens) || overlap(to_lens, lens, count, lens) || overlap(to_lens, lens, idx, B * (size_t)idx_stride * 4) ||
      overlap(to_lens, lens, p->page_indptr, lens + 4) || overlap(to_lens, lens, to_indptr, lens + 4) || (skip != nullptr && overlap(to_lens, lens, skip, B)))
    return TS_ERR_INVALID_ARG;
  CompactArgs a{};
  a.k_pool = (uint8_t*)const_cast<void*>(p->k_pool); a.v_pool = (uint8_t*)const_cast<void*>(p->v_pool);
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens;
  a.idx = idx; a.count = count; a.skip = skip; a.to_indptr = to_indptr; a.to_indices = to_indices; a.to_lens = to_lens;
  a.idx_stride = idx_stride; a.n_init = p->num_initial; a.n_local = p->num_local; a.max_seq_len = p->max_seq_len;
  a.p_shift = ilog2(p->page_size);
  a.row_bytes = p->num_kv_heads * p->head_dim * (p->dtype == TS_BF16 ? 2 : 4);
  return launch_cache_compact(a, p->batch, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

}  // extern "C"
