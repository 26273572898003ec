// C ABI of drafted trees: their masks and accepted paths (their attention: cache_api.hip, quant_api.hip).  Argument checks and launches.
#include "api_checks.h"

using namespace ts;

extern "C" {

int32_t ts_tree_mask(const ts_problem* p, const int32_t* parents, const int32_t* q_indptr, int32_t num_rows, uint32_t* mask, int32_t mask_words,
                     int32_t* positions, void* stream) {
  int32_t st = check_problem(p);
  if (st != TS_OK) return st;
  if ((st = check_rows(p, q_indptr, num_rows)) != TS_OK) return st;
  if (mask_words < 1) return TS_ERR_INVALID_ARG;
  if (num_rows == 0) return TS_OK;
  if (parents == nullptr || mask == nullptr) return TS_ERR_INVALID_ARG;
  const size_t rows = (size_t)num_rows * 4, words = rows * mask_words;
  // a sequence's workgroups write while others still read what tells them their rows
  const size_t lens = (size_t)p->batch * 4;
  auto taken = [&](const void* x, size_t n) {
    return overlap(x, n, parents, rows) || overlap(x, n, p->seq_lens, lens) || (q_indptr != nullptr && overlap(x, n, q_indptr, lens + 4));
  };
  if (taken(mask, words) || (positions != nullptr && (taken(positions, rows) || overlap(positions, rows, mask, words)))) return TS_ERR_INVALID_ARG;
  TreeMaskArgs a{};
  a.parents = parents; a.q_indptr = q_indptr; a.seq_lens = p->seq_lens; a.mask = mask; a.positions = positions;
  a.C = p->chunk; a.T = num_rows; a.words = mask_words;
  return launch_tree_mask(a, p->batch, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

int32_t ts_tree_keep(const ts_problem* p, const ts_quant* c, const int32_t* path, int32_t path_stride, const int32_t* count, const int32_t* q_indptr,
                     int32_t* to_lens, void* stream) {
  TreeKeepArgs a{};
  if (c != nullptr) {
    QuantPools pools;
    const int32_t st = check_quant(p, c, &pools);
    if (st != TS_OK) return st;
    a.k = pools.k_codes; a.v = pools.v_codes; a.k_scale = pools.k_scale; a.v_scale = pools.v_scale;
    a.row_bytes = p->num_kv_heads * p->head_dim;
  } else {
    const int32_t st = check_problem(p);
    if (st != TS_OK) return st;
    if (p->k_pool == nullptr || p->v_pool == nullptr || !aligned16(p->k_pool) || !aligned16(p->v_pool)) return TS_ERR_INVALID_ARG;
    a.k = (uint8_t*)const_cast<void*>(p->k_pool); a.v = (uint8_t*)const_cast<void*>(p->v_pool);
    a.row_bytes = p->num_kv_heads * p->head_dim * (p->dtype == TS_BF16 ? 2 : 4);
  }
  if (path == nullptr || path_stride < 1 || count == nullptr || to_lens == nullptr) return TS_ERR_INVALID_ARG;
  // a sequence's first workgroup writes its new length while others still read the rest
  const size_t B = (size_t)p->batch, lens = B * 4;
  if (overlap(to_lens, lens, p->seq_lens, lens) || overlap(to_lens, lens, count, lens) || overlap(to_lens, lens, path, B * (size_t)path_stride * 4) ||
      overlap(to_lens, lens, p->page_indptr, lens + 4) || (q_indptr != nullptr && overlap(to_lens, lens, q_indptr, lens + 4)))
    return TS_ERR_INVALID_ARG;
  a.page_indptr = p->page_indptr; a.page_indices = p->page_indices; a.seq_lens = p->seq_lens; a.q_indptr = q_indptr;
  a.path = path; a.count = count; a.to_lens = to_lens;
  a.path_stride = path_stride; a.C = p->chunk; a.H_kv = p->num_kv_heads; a.p_shift = ilog2(p->page_size); a.max_seq_len = p->max_seq_len;
  return launch_tree_keep(a, p->batch, (hipStream_t)stream) == hipSuccess ? TS_OK : TS_ERR_HIP;
}

}  // extern "C"
