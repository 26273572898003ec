// Drafted trees: which new tokens a row sees, from the tree's parents, and the rows of an accepted path moved up behind the cached tokens.  Both
// are a few kilobytes and bound by latency: a launch, and one memory round trip after the other.
#include "ts_kernels.h"
#include <algorithm>

namespace ts {

constexpr int kTreeStaged = 4096;              // parents of a sequence in LDS

// A workgroup per sequence and 256 new tokens, a thread per token: it walks from the token to its root through parents in LDS.  A parent lies before
// its child, so that the words of the row are written from the last to the first, once each.
__global__ __launch_bounds__(256) void tree_mask_kernel(TreeMaskArgs a) {
  __shared__ int32_t s_parent[kTreeStaged];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int r0 = a.q_indptr != nullptr ? min(max(a.q_indptr[b], 0), a.T) : b * a.C;
  const int n = max((a.q_indptr != nullptr ? min(max(a.q_indptr[b + 1], 0), a.T) : r0 + a.C) - r0, 0);
  const int32_t* parents = a.parents + r0;
  const int base = max(a.seq_lens[b], 0) - n;
  for (int c0 = blockIdx.x * 256; c0 < n; c0 += gridDim.x * 256) {
    const int staged = min(min(c0 + 256, n), kTreeStaged);
    __syncthreads();                           // the turn before is done with it
    for (int i = tid; i < staged; i += 256) s_parent[i] = parents[i];
    __syncthreads();
    const int c = c0 + tid;
    if (c < n) {
      uint32_t* row = a.mask + (size_t)(r0 + c) * a.words;
      auto put = [&](int w, uint32_t bits, int down_to) {              // word w, and zeros below it down to that one
        if (w < a.words) row[w] = bits;
        for (int x = min(w, a.words) - 1; x >= down_to; --x) row[x] = 0u;
      };
      int at = c, word = c >> 5, seen = 1;
      uint32_t bits = 1u << (c & 31);
      for (int x = a.words - 1; x > word; --x) row[x] = 0u;
      for (;;) {
        const int up = at < kTreeStaged ? s_parent[at] : parents[at];
        if ((uint32_t)up >= (uint32_t)at) break;                       // a root, or what cannot be a parent
        if (up >> 5 != word) { put(word, bits, (up >> 5) + 1); word = up >> 5; bits = 0u; }
        bits |= 1u << (up & 31);
        ++seen;
        at = up;
      }
      put(word, bits, 0);
      if (a.positions != nullptr) a.positions[r0 + c] = base + seen - 1;
    }
  }
}

hipError_t launch_tree_mask(const TreeMaskArgs& a, int B, hipStream_t s) {
  hipLaunchKernelGGL(tree_mask_kernel, dim3((unsigned)std::min((a.C + 255) / 256, 1024), B), dim3(256), 0, s, a);
  return hipGetLastError();
}

constexpr int kKeepSlots = 64;                 // path entries whose places are in LDS at a time
constexpr int kKeepBatch = 8;                  // rows in flight

// A thread has one 16-byte column of K or V (or one head's scale) and moves it for the whole path in order: an entry's place lies at or behind the
// place it goes to, and places that have been written are in front of all that are still read, so that a batch may be read before it is written.
__global__ __launch_bounds__(256) void tree_keep_kernel(TreeKeepArgs a) {
  __shared__ int64_t s_from[kKeepSlots], s_to[kKeepSlots];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int n = a.q_indptr != nullptr ? max(a.q_indptr[b + 1] - a.q_indptr[b], 0) : a.C;
  const int count = min(max(a.count[b], 0), min(a.path_stride, n));
  const int64_t base = (int64_t)max(a.seq_lens[b], 0) - n;
  if (blockIdx.x == 0 && tid == 0) a.to_lens[b] = (int)max(base + count, (int64_t)0);
  const int32_t* pages = a.page_indices + a.page_indptr[b];
  const int mask = (1 << a.p_shift) - 1, pieces = a.row_bytes / 16, j = blockIdx.x * 256 + tid;
  const bool is_row = j < 2 * pieces, is_scale = !is_row && a.k_scale != nullptr && j - 2 * pieces < 2 * a.H_kv;
  uint8_t* rows = (j < pieces ? a.k : a.v) + (int64_t)(j < pieces ? j : j - pieces) * 16;
  const int h = j - 2 * pieces;                // scales: K's heads, then V's
  float* scales = (h < a.H_kv ? a.k_scale : a.v_scale);
  const int head = h < a.H_kv ? h : h - a.H_kv;
  for (int i0 = 0; i0 < count; i0 += kKeepSlots) {
    const int many = min(count - i0, kKeepSlots);
    __syncthreads();
    if (tid < many) {
      const int i = i0 + tid;
      const int64_t to = base + i, from = base + min(max(a.path[(size_t)b * a.path_stride + i], i), n - 1);
      const bool moves = to >= 0 && from < a.max_seq_len && from != to;
      s_from[tid] = moves ? ((int64_t)pages[from >> a.p_shift] << a.p_shift) + (from & mask) : -1;
      s_to[tid] = moves ? ((int64_t)pages[to >> a.p_shift] << a.p_shift) + (to & mask) : -1;
    }
    __syncthreads();
    if (is_row) {
      for (int i = 0; i < many; i += kKeepBatch) {
        u32x4_t x[kKeepBatch];
#pragma unroll
        for (int u = 0; u < kKeepBatch; ++u)
          if (i + u < many && s_from[i + u] >= 0) x[u] = *reinterpret_cast<const u32x4_t*>(rows + s_from[i + u] * a.row_bytes);
#pragma unroll
        for (int u = 0; u < kKeepBatch; ++u)
          if (i + u < many && s_from[i + u] >= 0) *reinterpret_cast<u32x4_t*>(rows + s_to[i + u] * a.row_bytes) = x[u];
      }
    } else if (is_scale) {
      auto at = [&](int64_t slot) -> float* { return scales + ((((slot >> a.p_shift) * a.H_kv + head) << a.p_shift) + (slot & mask)); };
      for (int i = 0; i < many; ++i)
        if (s_from[i] >= 0) *at(s_to[i]) = *at(s_from[i]);
    }
  }
}

hipError_t launch_tree_keep(const TreeKeepArgs& a, int B, hipStream_t s) {
  const int columns = 2 * (a.row_bytes / 16) + (a.k_scale != nullptr ? 2 * a.H_kv : 0);
  hipLaunchKernelGGL(tree_keep_kernel, dim3((unsigned)((columns + 255) / 256), B), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ts
