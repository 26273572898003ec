// A cache in 8 bits: new tokens turned, quantised and written into their pages, tokens read back, pages copied.  Bound by memory: every
// row is read and written once.
//
// Writing: up to sixteen waves take a token.  D / 8 lanes hold a row of eight elements each, so that
// a row's largest absolute value is three or four steps of the lanes' network away.  Rows are
// requested a turn ahead, the first before the token's place is known; cosines and sines stay in LDS (in registers they leave a SIMD four or five waves instead of seven): 16661 bf16 tokens of
// 32/8 heads of 128, all of it turned, into e4m3 102 us instead of 116, into int8 100 instead of 106 (97 and 89 on another card); nothing turned 78 and 76 (4.8 TB/s); fp32 153 us (4.7 TB/s).  All arithmetic is in double: a
// turned key next to the middle of two stored values, or a quotient next to the middle of two codes, falls as the definition says.  A quotient x Q / m is
// formed by the row's reciprocal and one correction with the exact remainder (Markstein's division): a quotient that is a double -- every tie
// between two codes is -- comes out exactly.
#include "ts_kernels.h"
#include "ts_rows.h"
#include "ts_codes.h"
#include <algorithm>

namespace ts {

template <typename T> struct Eight;                                    // eight stored elements
template <> struct Eight<uint16_t> {
  u32x4_t w;
  __device__ __forceinline__ void load(const uint8_t* at) { w = *reinterpret_cast<const u32x4_t*>(at); }
  __device__ __forceinline__ float get(int i) const { return (i & 1) != 0 ? bf16_hi(w[i >> 1]) : bf16_lo(w[i >> 1]); }
};
template <> struct Eight<float> {
  u32x4_t w[2];
  __device__ __forceinline__ void load(const uint8_t* at) { w[0] = reinterpret_cast<const u32x4_t*>(at)[0]; w[1] = reinterpret_cast<const u32x4_t*>(at)[1]; }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(w[i >> 2][i & 3]); }
};
template <typename T> __device__ __forceinline__ float load_one(const uint8_t* at);
template <> __device__ __forceinline__ float load_one<float>(const uint8_t* at) { return *reinterpret_cast<const float*>(at); }
template <> __device__ __forceinline__ float load_one<uint16_t>(const uint8_t* at) { return __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(at) << 16); }

__device__ __forceinline__ uint32_t round_bf16(float x) {              // bits; NaN stays NaN
  return __builtin_bit_cast(uint16_t, (__bf16)x);
}
__device__ __forceinline__ void store_eight(uint16_t*, uint8_t* at, const float (&x)[8]) {
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = round_bf16(x[2 * i]) | (round_bf16(x[2 * i + 1]) << 16);
  *reinterpret_cast<u32x4_t*>(at) = w;
}
__device__ __forceinline__ void store_eight(float*, uint8_t* at, const float (&x)[8]) {
  reinterpret_cast<u32x4_t*>(at)[0] = u32x4_t{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  reinterpret_cast<u32x4_t*>(at)[1] = u32x4_t{__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7])};
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}

// e4m3 of a double of at most 448, to nearest even: rounded to the code's step here (a float next to the middle of two codes would lose
// on which side it lies), so that the conversion is exact; with the sign of x, which the quotient of a zero has lost
__device__ __forceinline__ float e4m3_value(double z, float x) {
  const int behind = 4 - max(__builtin_amdgcn_frexp_exp(z), -5);       // |z| < 2^exponent; three bits behind the leading one, 2^-9 the smallest
  return __builtin_copysignf((float)__builtin_amdgcn_ldexp(rint(__builtin_amdgcn_ldexp(z, behind)), -behind), x);
}

template <typename T, int CODE, int D>
__global__ __launch_bounds__(256) void quant_append_kernel(RopeAppendArgs a, QuantPools c) {
  constexpr int LPR = D / 8, RPW = 64 / LPR, ES = sizeof(T), RB = D * ES;   // lanes of a row, rows side by side in a wave, bytes of a row
  __shared__ __attribute__((aligned(16))) double s_turn[4][8 * 9][2];       // pair p at p + p / 8: lanes read eight pairs each, 144 bytes apart
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t turn = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave;
  const int part = (int)turn & ((1 << a.share_shift) - 1), row = (int)(turn >> a.share_shift);
  if (row >= a.T) return;
  const int half = a.rotary >> 1, nq = a.q != nullptr ? a.H : 0, nk = a.H_kv;
  const uint8_t* q_row = a.q + row * a.q_stride;
  const uint8_t* k_row = a.k + row * a.k_stride;
  const uint8_t* v_row = a.v + row * a.v_stride;
  const int u = lane % LPR, e0 = u * 8;
  const bool any = e0 < a.rotary, in_piece = a.adjacent != 0, whole = (half & 7) == 0;
  const int all = nq + 2 * nk, step = RPW << a.share_shift;
  // this lane's elements of row h, and their partners where these are a piece of their own; requested a turn ahead, the first ones before the token's place is known
  Eight<T> own, other;
  auto row_at = [&](int h) -> const uint8_t* {
    return h < nq ? q_row + (int64_t)h * RB : h < nq + nk ? k_row + (int64_t)(h - nq) * RB : v_row + (int64_t)(h - nq - nk) * RB;
  };
  auto request = [&](int h) __attribute__((always_inline)) {
    if (h >= all) return;
    const uint8_t* from = row_at(h);
    own.load(from + e0 * ES);
    if (any && h < nq + nk && !in_piece && whole) other.load(from + (e0 < half ? e0 + half : e0 - half) * ES);   // (then the turned part is whole pieces too)
  };
  const int h0 = part * RPW + lane / LPR;
  request(h0);
  double freq = 0.;
  int pos = 0;
  if (lane < half) {
    freq = a.inv_freq[lane];
    if (a.positions != nullptr) pos = a.positions[(size_t)a.pair_axis[lane] * a.T + row];
  }
  const RowPlace at = row_place(a.q_indptr, a.B, a.C, a.T, row);
  if (at.b < 0) return;
  const int place = max(a.seq_lens[at.b], 0) - at.left, page0 = a.page_indptr[at.b];
  const bool append = place >= 0 && place < a.max_seq_len;             // (a step whose lengths have grown past the bound must not write over cached tokens)
  int64_t page = 0;
  if (append) page = a.page_indices[page0 + (place >> a.p_shift)];
  if (lane < half) {
    if (a.positions == nullptr) pos = place;
    const double turns = (double)pos * freq * 0.15915494309189533577;
    double s, co;
    sincospi(2.0 * (turns - rint(turns)), &s, &co);
    s_turn[wave][lane + (lane >> 3)][0] = co * a.scale; s_turn[wave][lane + (lane >> 3)][1] = s * a.scale;
  }
  __builtin_amdgcn_wave_barrier();                                     // (a wave's LDS accesses keep their order)

  const int64_t slot = (page << a.p_shift) + (place & (a.P - 1));
  auto turn_and_store = [&](int h, const Eight<T>& mine, const Eight<T>& partner) __attribute__((always_inline)) {
    const bool is_q = h < nq, is_v = h >= nq + nk;
    const int kv = is_v ? h - nq - nk : h - nq;                        // its KV head
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = mine.get(i);
    if (any && !is_v) {
      float y[8];
      if (in_piece) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[i ^ 1];
      } else if (whole) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = partner.get(i);
      } else {
        const uint8_t* from = row_at(h);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = e0 + i;
          y[i] = e < a.rotary ? load_one<T>(from + (e < half ? e + half : e - half) * ES) : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (e0 + i < a.rotary) {                                       // x cos - y sin for the first of a pair, x cos + y sin for the second
          const int e = e0 + i, pair = in_piece ? e >> 1 : e < half ? e : e - half;
          const double2 t = *reinterpret_cast<const double2*>(s_turn[wave][pair + (pair >> 3)]);
          const bool first = in_piece ? (i & 1) == 0 : e < half;
          x[i] = (float)fma((double)x[i], t.x, (double)y[i] * (first ? -t.y : t.y));
        }
    }
    if (is_q) { store_eight((T*)nullptr, a.q_out + ((int64_t)row * a.H + h) * RB + e0 * ES, x); return; }
    if (sizeof(T) == 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(round_bf16(x[i]) << 16);
    }
    uint32_t m = 0;                                                    // bits of the largest absolute value; those of infinities and NaN are larger still
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
    m = dpp_max_u32<0xB1>(m);     // quad_perm [1,0,3,2]
    m = dpp_max_u32<0x4E>(m);     // quad_perm [2,3,0,1]
    m = dpp_max_u32<0x141>(m);    // row_half_mirror
    if (LPR == 16) m = dpp_max_u32<0x140>(m);                          // row_mirror
    if (!append) return;
    const bool finite = m < 0x7f800000u;
    const double most = __uint_as_float(m), inv = 1. / most;
    uint32_t w[2] = {0u, 0u};
    if (finite && m != 0u) {
      double z[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const double n = (double)x[i] * kCodeTop<CODE>, q0 = n * inv;
        z[i] = fma(fma(-q0, most, n), inv, q0);
      }
      if constexpr (CODE == TS_INT8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= ((uint32_t)(int)rint(z[i]) & 0xffu) << (8 * (i & 3));
      } else {
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
          int v = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_value(z[i], x[i]), e4m3_value(z[i + 1], x[i + 1]), 0, false);
          w[i >> 2] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_value(z[i + 2], x[i + 2]), e4m3_value(z[i + 3], x[i + 3]), v, true);
        }
      }
    }
    *reinterpret_cast<uint2*>((is_v ? c.v_codes : c.k_codes) + (slot * nk + kv) * D + e0) = make_uint2(w[0], w[1]);
    if (u == 0)
      (is_v ? c.v_scale : c.k_scale)[(page * nk + kv) * a.P + (place & (a.P - 1))] = finite ? (float)(most / kCodeTop<CODE>) : __uint_as_float(0x7fc00000u);
  };
  for (int h = h0; h < all; h += step) {
    const Eight<T> mine = own, partner = other;
    request(h + step);
    turn_and_store(h, mine, partner);
  }
}

// log2 of the waves that share a token (a row that is read): no more than have a turn.  Few tokens are bound by one turn after the other, many by what each wave does before its first one.
// Times of a call in a captured graph of twenty (alone, with its start and end, a microsecond more), appending with 2, 4, 8 and 16 waves a token, int8 and 32/8 heads of 128: 64 tokens 8.1, 5.9, 5.2, 4.4 us; 256 8.3, 6.3, 6.1, 6.6; 512 8.8, 7.4, 8.2, 10.2; 4096 26, 29, 41, 62.  Reading
// with 1, 2, 4 and 8: 64 3.6, 3.0, 2.8, 2.8; 1024 4.2, 3.7, 3.8, 5.0; 4096 7.7, 7.3, 9.5, 16.
static int most_shared(int turns) { return turns <= 1 ? 0 : turns <= 2 ? 1 : turns <= 4 ? 2 : turns <= 8 ? 3 : 4; }
static int append_share(const RopeAppendArgs& a) {
  const int heads = (a.q != nullptr ? a.H : 0) + 2 * a.H_kv, side = 512 / a.D;      // rows side by side in a wave
  return std::min(most_shared((heads + side - 1) / side), a.T <= 128 ? 4 : a.T <= 256 ? 3 : a.T <= 1024 ? 2 : 1);
}
static int read_share(const QuantReadArgs& a) {
  return std::min(most_shared(2 * a.H_kv * a.D / 512), a.T <= 1024 ? 2 : a.T <= 8192 ? 1 : 0);
}

template <typename T, int CODE>
static hipError_t append_one(const RopeAppendArgs& b, const QuantPools& c, hipStream_t s) {
  RopeAppendArgs a = b;
  a.share_shift = append_share(a);
  const long wgs = (((long)a.T << a.share_shift) + 3) / 4, wide = 1 << 20;      // (a grid has less than 2^32 threads in a dimension)
  const dim3 grid((unsigned)std::min(wgs, wide), (unsigned)((wgs + wide - 1) / wide));
  if (a.D == 64) hipLaunchKernelGGL((quant_append_kernel<T, CODE, 64>), grid, dim3(256), 0, s, a, c);
  else hipLaunchKernelGGL((quant_append_kernel<T, CODE, 128>), grid, dim3(256), 0, s, a, c);
  return hipGetLastError();
}

hipError_t launch_quant_append(int dtype, const RopeAppendArgs& a, const QuantPools& c, hipStream_t s) {
  if (dtype == TS_BF16) return c.code == TS_INT8 ? append_one<uint16_t, TS_INT8>(a, c, s) : append_one<uint16_t, TS_E4M3>(a, c, s);
  return c.code == TS_INT8 ? append_one<float, TS_INT8>(a, c, s) : append_one<float, TS_E4M3>(a, c, s);
}

// One, two or four waves per row: pieces of eight codes, K's, then V's.
template <typename T, int CODE>
__global__ __launch_bounds__(256) void quant_read_kernel(QuantReadArgs a, QuantPools c) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t turn = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave;
  const int part = (int)turn & ((1 << a.share_shift) - 1), row = (int)(turn >> a.share_shift);
  if (row >= a.T) return;
  const RowPlace at = row_place(a.q_indptr, a.B, a.C, a.T, row);
  if (at.b < 0) return;
  const int place = max(a.seq_lens[at.b], 0) - at.left;
  const bool there = place >= 0 && place < a.max_seq_len;
  int64_t page = 0;
  if (there) page = a.page_indices[a.page_indptr[at.b] + (place >> a.p_shift)];
  const int in_page = place & (a.P - 1), d_shift = a.D == 64 ? 3 : 4, each = a.H_kv << d_shift;   // pieces of K, and of V
  const int64_t slot = (page << a.p_shift) + in_page;
  for (int i = part * 64 + lane; i < 2 * each; i += 64 << a.share_shift) {
    const bool is_v = i >= each;
    const int j = is_v ? i - each : i, kv = j >> d_shift;
    uint8_t* out = is_v ? a.v_out : a.k_out;
    if (out == nullptr) continue;
    float x[8] = {};
    if (there) {
      const uint2 w = *reinterpret_cast<const uint2*>((is_v ? c.v_codes : c.k_codes) + slot * a.H_kv * a.D + j * 8);
      const float scale = (is_v ? c.v_scale : c.k_scale)[(page * a.H_kv + kv) * a.P + in_page];
      float y[2][4];
      codes_to_f32<CODE>(w.x, y[0]);
      codes_to_f32<CODE>(w.y, y[1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = y[e >> 2][e & 3] * scale;
    }
    store_eight((T*)nullptr, out + ((int64_t)row * a.H_kv * a.D + j * 8) * sizeof(T), x);
  }
}

hipError_t launch_quant_read(int dtype, const QuantReadArgs& b, const QuantPools& c, hipStream_t s) {
  QuantReadArgs a = b;
  a.share_shift = read_share(a);
  const long wgs = (((long)a.T << a.share_shift) + 3) / 4, wide = 1 << 20;
  const dim3 grid((unsigned)std::min(wgs, wide), (unsigned)((wgs + wide - 1) / wide));
  if (dtype == TS_BF16) {
    if (c.code == TS_INT8) hipLaunchKernelGGL((quant_read_kernel<uint16_t, TS_INT8>), grid, dim3(256), 0, s, a, c);
    else hipLaunchKernelGGL((quant_read_kernel<uint16_t, TS_E4M3>), grid, dim3(256), 0, s, a, c);
  } else {
    if (c.code == TS_INT8) hipLaunchKernelGGL((quant_read_kernel<float, TS_INT8>), grid, dim3(256), 0, s, a, c);
    else hipLaunchKernelGGL((quant_read_kernel<float, TS_E4M3>), grid, dim3(256), 0, s, a, c);
  }
  return hipGetLastError();
}

// The scales of copied pages (P * H_kv floats, as few as one: no wider pieces).  blockIdx.y: K or V; pairs are dealt to gridDim.x.
__global__ __launch_bounds__(256) void quant_scales_copy_kernel(QuantPools c, const int32_t* src, const int32_t* dst, int n, int num_pages, int each) {
  float* pool = blockIdx.y == 0 ? c.k_scale : c.v_scale;
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int from = src[i], to = dst[i];
    if ((uint32_t)from >= (uint32_t)num_pages || (uint32_t)to >= (uint32_t)num_pages || from == to) continue;
    for (int e = threadIdx.x; e < each; e += 256) pool[(int64_t)to * each + e] = pool[(int64_t)from * each + e];
  }
}

hipError_t launch_quant_pages_copy(const QuantPools& c, const int32_t* src, const int32_t* dst, int n, int num_pages, int P, int H_kv, int D, hipStream_t s) {
  PagesCopyArgs a{};
  a.src = src; a.dst = dst; a.n = n; a.num_pages = num_pages;
  a.k_pool = c.k_codes; a.v_pool = c.v_codes;
  a.page_bytes = (int64_t)P * H_kv * D;
  const hipError_t e = launch_pages_copy(a, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(quant_scales_copy_kernel, dim3((unsigned)std::min(n, 16384), 2), dim3(256), 0, s, c, src, dst, n, num_pages, P * H_kv);
  return hipGetLastError();
}

}  // namespace ts
