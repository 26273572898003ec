// Rotary positions with several axes, and the new tokens' K and V rows into their pages.
//
// A workgroup takes one token.  Its angles are the same for all heads: a lane per pair forms the angle in double (an exact int32
// times a float has 55 bits), takes whole turns off in double and leaves cosine and sine in LDS; then every lane turns pieces of
// heads.  Whoever writes an element is the only one who read it, so q may be turned in place.
#include "ts_kernels.h"
#include "ts_rows.h"

namespace ts {

template <typename T> __device__ __forceinline__ float load_el(const uint8_t* p, int i);
template <> __device__ __forceinline__ float load_el<float>(const uint8_t* p, int i) { return reinterpret_cast<const float*>(p)[i]; }
template <> __device__ __forceinline__ float load_el<uint16_t>(const uint8_t* p, int i) { return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << 16); }
template <typename T> __device__ __forceinline__ void store_el(uint8_t* p, int i, float x);
template <> __device__ __forceinline__ void store_el<float>(uint8_t* p, int i, float x) { reinterpret_cast<float*>(p)[i] = x; }
template <> __device__ __forceinline__ void store_el<uint16_t>(uint8_t* p, int i, float x) { reinterpret_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_bits(x); }

template <typename T>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeAppendArgs a) {
  constexpr int VE = 16 / sizeof(T);
  __shared__ float s_cos[64], s_sin[64];
  const int row = blockIdx.x, tid = threadIdx.x;
  const RowPlace at = row_place(a.q_indptr, a.B, a.C, a.T, row);
  if (at.b < 0) return;
  const int n = min(max(a.seq_lens[at.b], 0), a.max_seq_len);
  const int place = n - at.left, half = a.rotary >> 1;
  if (tid < half) {
    const int pos = a.positions != nullptr ? a.positions[(size_t)a.pair_axis[tid] * a.T + row] : place;
    const double turns = (double)pos * (double)a.inv_freq[tid] * 0.15915494309189533577;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    s_cos[tid] = c * a.scale; s_sin[tid] = s * a.scale;
  }
  __syncthreads();
  const int D = a.D, row_elems = D;
  const bool append = a.k != nullptr && place >= 0;
  const int64_t slot = append ? ((int64_t)a.page_indices[a.page_indptr[at.b] + (place >> a.p_shift)] << a.p_shift) + (place & (a.P - 1)) : 0;
  const int heads_q = a.q != nullptr ? a.H : 0, heads_k = append ? a.H_kv : 0;
  // elements one by one: pairs, then what passes through
  const int units = half + (D - a.rotary);
  for (int u = tid; u < (heads_q + heads_k) * units; u += 256) {
    const int h = u / units, i = u % units;
    const uint8_t* from; uint8_t* to;
    if (h < heads_q) {
      from = a.q + row * a.q_stride + (int64_t)h * row_elems * sizeof(T);
      to = a.q_out + ((int64_t)row * a.H + h) * row_elems * sizeof(T);
    } else {
      from = a.k + row * a.k_stride + (int64_t)(h - heads_q) * row_elems * sizeof(T);
      to = a.k_pool + (slot * a.H_kv + (h - heads_q)) * row_elems * sizeof(T);
    }
    if (i >= half) { const int e = a.rotary + i - half; reinterpret_cast<T*>(to)[e] = reinterpret_cast<const T*>(from)[e]; continue; }
    const int e0 = a.adjacent ? 2 * i : i, e1 = a.adjacent ? 2 * i + 1 : i + half;
    const float x = load_el<T>(from, e0), y = load_el<T>(from, e1), c = s_cos[i], s = s_sin[i];
    store_el<T>(to, e0, x * c - y * s);
    store_el<T>(to, e1, x * s + y * c);
  }
  if (append)
    for (int u = tid; u < a.H_kv * D / VE; u += 256)
      reinterpret_cast<uint4*>(a.v_pool + slot * a.H_kv * D * sizeof(T))[u] = reinterpret_cast<const uint4*>(a.v + row * a.v_stride)[u];
}

hipError_t launch_rope_append(int dtype, const RopeAppendArgs& a, hipStream_t s) {
  if (dtype == TS_BF16) hipLaunchKernelGGL(rope_append_kernel<uint16_t>, dim3(a.T), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rope_append_kernel<float>, dim3(a.T), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace ts
