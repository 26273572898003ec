// Rows of new tokens: which sequence a row belongs to, and where in it.
#pragma once
#include "ts_common.h"

#ifdef __HIPCC__
namespace ts {

struct RowPlace { int b, left; };              // sequence (-1: none) and rows of it from this one to its end, this one included

// first row of sequence b (b = B: the end of the last), whatever the caller left there
__device__ __forceinline__ int row_begin(const int32_t* q_indptr, int C, int T, int b) {
  return q_indptr != nullptr ? min(max(q_indptr[b], 0), T) : b * C;
}

// Binary search for the last sequence that begins at or before `row`: log2(B) dependent loads, the same for all lanes of a row.
__device__ __forceinline__ RowPlace row_place(const int32_t* q_indptr, int B, int C, int T, int row) {
  if (q_indptr == nullptr) { const int b = row / C; return RowPlace{b, (b + 1) * C - row}; }
  int lo = 0, hi = B + 1;                      // sequences below lo begin at or before the row, from hi on after it
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (row_begin(q_indptr, C, T, mid) <= row) lo = mid + 1; else hi = mid;
  }
  if (lo == 0 || lo == B + 1) return RowPlace{-1, 0};
  return RowPlace{lo - 1, row_begin(q_indptr, C, T, lo) - row};
}

}  // namespace ts
#endif
