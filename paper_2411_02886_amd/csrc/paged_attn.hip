// Dense attention of new tokens over their whole sequence through the page table.
//
// A wave per (row, query head): lane l holds the D / 64 elements 64 i + l of the query and the output; a key's score is a sum over
// the lanes, and the softmax runs along with a running maximum and sum.
#include "ts_kernels.h"
#include "ts_rows.h"

namespace ts {

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_attn_rows_kernel(PagedAttnArgs a) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, h = blockIdx.y * 4 + (threadIdx.x >> 6), row = blockIdx.x;
  if (h >= a.H) return;
  const RowPlace at = row_place(a.q_indptr, a.B, a.C, a.T, row);
  if (at.b < 0) return;
  const int n = min(max(a.seq_lens[at.b], 0), a.max_seq_len), x = n - at.left;
  const int t0 = a.window > 0 ? max(0, x - a.window + 1) : 0;
  const int kvh = h / (a.H / a.H_kv);
  const int32_t* pages = a.page_indices + a.page_indptr[at.b];
  auto el = [](const uint8_t* p, int64_t i) -> float {
    if (sizeof(T) == 4) return reinterpret_cast<const float*>(p)[i];
    return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16);
  };
  float q[E], o[E], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) { q[e] = el(a.q, ((int64_t)row * a.H + h) * D + e * 64 + lane); o[e] = 0.f; }
  for (int t = t0; t <= x; ++t) {
    const int64_t r = ((((int64_t)pages[t >> a.p_shift] << a.p_shift) + (t & (a.P - 1))) * a.H_kv + kvh) * D;
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) s = fmaf(q[e], el(a.k_pool, r + e * 64 + lane), s);
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
    s *= a.sm_scale;
    const float top = fmaxf(m, s), f = expf(m - top), w = expf(s - top);
    m = top; l = l * f + w;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(w, el(a.v_pool, r + e * 64 + lane), o[e] * f);
  }
  const int64_t hb = (int64_t)row * a.H + h;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const float v = l > 0.f ? o[e] / l : 0.f;
    if (sizeof(T) == 4) reinterpret_cast<float*>(a.out)[hb * D + e * 64 + lane] = v;
    else reinterpret_cast<uint16_t*>(a.out)[hb * D + e * 64 + lane] = (uint16_t)f32_to_bf16_bits(v);
  }
  if (lane == 0 && a.lse != nullptr) a.lse[hb] = l > 0.f ? m + logf(l) : -INFINITY;
}

hipError_t launch_paged_attn(int dtype, int D, const PagedAttnArgs& a, hipStream_t s) {
  const dim3 grid(a.T, (a.H + 3) / 4);
  if (dtype == TS_BF16) {
    if (D == 64) hipLaunchKernelGGL((paged_attn_rows_kernel<uint16_t, 64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_attn_rows_kernel<uint16_t, 128>), grid, dim3(256), 0, s, a);
  } else {
    if (D == 64) hipLaunchKernelGGL((paged_attn_rows_kernel<float, 64>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_attn_rows_kernel<float, 128>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}

}  // namespace ts
