// Rows of new tokens: which sequence a row belongs to, and where in it.
#pragma once
#include "ts_common.h"

#ifdef __HIPCC__
namespace ts {

struct RowPlace { int b, left; };              // sequence (-1: none) and rows of it from this one to its end, this one included

// first row of sequence b (b = B: the end of the last), whatever the caller left there
__device__ __forceinline__ int row_begin(const int32_t* q_indptr, int T, int b) { return min(max(q_indptr[b], 0), T); }

// The last sequence that begins at or before `row`, by all lanes of a wave together: 64 places at a time, so one load for up to 63
// sequences, two for up to 4095.
__device__ __forceinline__ RowPlace row_place(const int32_t* q_indptr, int B, int C, int T, int row) {
  if (q_indptr == nullptr) { const int b = row / C; return RowPlace{b, (b + 1) * C - row}; }
  const int lane = threadIdx.x & 63;
  int lo = 0, n = B + 1;                       // of the places lo .. lo + n - 1 those that begin at or before the row come first
  for (;;) {
    const int step = (n + 63) >> 6, i = lane * step;
    const int begin = i < n ? row_begin(q_indptr, T, lo + i) : 0;
    const uint64_t at_or_before = __builtin_amdgcn_ballot_w64(i < n && begin <= row);
    const int k = __builtin_popcountll(at_or_before);                  // places lo, lo + step, ... that do
    if (step == 1) {
      const int b = lo + k - 1;                                        // -1: none does (only with a first entry above 0)
      if (k == 0 || b >= B) return RowPlace{-1, 0};
      const int next = k < 64 && k < n ? __builtin_amdgcn_readlane(begin, k) : row_begin(q_indptr, T, b + 1);
      return RowPlace{b, next - row};
    }
    if (k == 0) return RowPlace{-1, 0};
    lo += (k - 1) * step;
    n = min(step, n - (k - 1) * step);
  }
}

}  // namespace ts
#endif
