// Rotary positions with several axes, and the new tokens' K and V rows into their pages.  Bound by memory: every row is read and written once.
//
// One, two or four waves take one token.  Its angles are the same for all heads: a lane per pair forms the angle in double (an exact int32 times
// a float has 55 bits), takes whole turns off, and leaves cosine and sine, formed in double and rounded once, in LDS (in float they cost 0.1 us less a call, and fp32
// results were off by 4.1e-8 instead of 3.0e-8).  Then a lane has the same piece of every
// head it works on, so that it reads its cosines once: 64 / (pieces of a head, rounded up to a power of two) heads side by side, several in flight.  A
// piece is 16 bytes and its partner (halves) or 16 bytes that hold whole pairs (neighbours); where the rotated part does not divide so, 8 bytes (3000 tokens of
// H 40/8, 24 of 128 elements turned, 20 us), and where it does not divide at all, single pairs (42).  Whoever writes an element is the only one who read it, so q may be turned in place.
// Measured (H 32/8, D 128): 15243 tokens, three axes, parts of a fused projection 155 us by a workgroup per token and single pairs, 75 so (5.0 TB/s, what a
// large copy reaches); 64 single tokens 4.5 us in a captured graph.
#include "ts_kernels.h"
#include "ts_rows.h"
#include <algorithm>

namespace ts {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

template <typename T> __device__ __forceinline__ float to_f32(T x) { return x; }
template <> __device__ __forceinline__ float to_f32<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
template <typename T> __device__ __forceinline__ T from_f32(float x) { return x; }
template <> __device__ __forceinline__ uint16_t from_f32<uint16_t>(float x) { return (uint16_t)f32_to_bf16_bits(x); }

typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
template <int BYTES> struct PieceWords { typedef u32x4_t type; };
template <> struct PieceWords<8> { typedef u32x2_t type; };

template <typename T, int BYTES> struct Piece {                        // 16 or 8 bytes as floats
  static constexpr int N = BYTES / sizeof(T);
  typedef typename PieceWords<BYTES>::type words_t;
  float x[N];
  __device__ __forceinline__ void load(words_t v) {
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) {
      if constexpr (sizeof(T) == 2) { x[2 * i] = bf16_lo(v[i]); x[2 * i + 1] = bf16_hi(v[i]); }
      else x[i] = __uint_as_float(v[i]);
    }
  }
  __device__ __forceinline__ words_t store() const {
    words_t w;
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) {
      if constexpr (sizeof(T) == 2) w[i] = __builtin_bit_cast(uint32_t, bf16x2_t{(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});   // one instruction, to nearest even
      else w[i] = __float_as_uint(x[i]);
    }
    return w;
  }
};

// Up to so many tokens four waves share each; beyond that two, and one where a wave has the heads in two steps.  (us by one, two, four waves, bf16: 64 tokens of
// H 32/8, D 128 6.2, 5.1, 4.5; 2048 11.4, 11.1, 11.1; 4096 17.7, 16.8, 19.4; 2000 of H 6/2, D 64 4.5, 5.1, 6.6, 30000 21.6, 33.0, 55.8; of H 16/4, D 128, three steps,
// 7.0, 6.9, 8.2 and 72.1, 70.4, 81.0.  Single pairs: always four, 5000 tokens of H 40/8 with 26 of 128 elements turned 79, 72, 62.)
constexpr int kRopeFew = 1024;

enum { kPairs = 0, kHalves = 1, kNeighbours = 2 };

template <typename T, int MODE, int BYTES>
__global__ __launch_bounds__(256) void rope_append_kernel(RopeAppendArgs a) {
  constexpr int VE = BYTES / sizeof(T), UN = 2;                        // elements of a piece; pieces per lane in flight
  typedef Piece<T, BYTES> piece_t;
  typedef typename piece_t::words_t words_t;
  __shared__ __attribute__((aligned(16))) float s_turn[4][2][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = 1 << a.share_shift;
  const int part = wave & (share - 1), row = (int)((((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * 4 + wave) >> a.share_shift);   // `share` waves to a token
  if (row >= a.T) return;
  // What does not wait for the row's place is requested first: frequencies, positions, the first pieces of the heads and of V.  (A load after the
  // stores would wait for them: 1300 fp32 tokens 18.7 us instead of 9.0.)
  const int D = a.D, row_bytes = D * (int)sizeof(T), half = a.rotary >> 1;
  const int nq = a.q != nullptr ? a.H : 0, nk = a.k != nullptr ? a.H_kv : 0;
  const uint8_t* q_row = a.q + row * a.q_stride;
  const uint8_t* k_row = a.k + row * a.k_stride;
  double freq = 0.;
  int pos = 0;
  if (lane < half) {
    freq = a.inv_freq[lane];
    if (a.positions != nullptr) pos = a.positions[(size_t)a.pair_axis[lane] * a.T + row];
  }
  // pieces of a head: those that turn, then those that pass through; this lane's, in every step-th head from side on
  const int turn = (MODE == kHalves ? half : a.rotary) / VE, units = turn + (D - a.rotary) / VE;
  const int shift = units > 1 ? 32 - __builtin_clz((uint32_t)(units - 1)) : 0;
  const int u = lane & ((1 << shift) - 1), lanes = 64 >> shift, side = part * lanes + (lane >> shift), step = lanes << a.share_shift;
  const bool turns = u < turn;
  const uint32_t e0 = (uint32_t)(turns || MODE == kNeighbours ? u * VE : a.rotary + (u - turn) * VE) * sizeof(T), e1 = e0 + half * sizeof(T);
  words_t v[UN], w[UN];
  auto load = [&](int h0) {
#pragma unroll
    for (int k = 0; k < UN; ++k) {
      const int h = h0 + k * step;
      if (h >= nq + nk || u >= units) continue;
      const uint8_t* from = h < nq ? q_row + h * row_bytes : k_row + (h - nq) * row_bytes;
      v[k] = *reinterpret_cast<const words_t*>(from + e0);
      if (MODE == kHalves && turns) w[k] = *reinterpret_cast<const words_t*>(from + e1);
    }
  };
  if constexpr (MODE != kPairs) load(side);
  const int v_pieces = nk * D * (int)sizeof(T) / 16, v_lane = part * 64 + lane, v_step = 64 << a.share_shift;
  const u32x4_t* v_row = reinterpret_cast<const u32x4_t*>(a.v + row * a.v_stride);
  u32x4_t x[UN];
  auto load_v = [&](int i0) {
#pragma unroll
    for (int k = 0; k < UN; ++k) if (i0 + k * v_step < v_pieces) x[k] = v_row[i0 + k * v_step];
  };
  load_v(v_lane);

  const RowPlace at = row_place(a.q_indptr, a.B, a.C, a.T, row);
  if (at.b < 0) return;
  const int place = max(a.seq_lens[at.b], 0) - at.left, page0 = a.page_indptr[at.b];
  const bool append = nk != 0 && place >= 0 && place < a.max_seq_len;  // (a step whose lengths have grown past the bound must not write over cached tokens)
  int64_t slot = 0;
  if (append) slot = ((int64_t)a.page_indices[page0 + (place >> a.p_shift)] << a.p_shift) + (place & (a.P - 1));
  float* s_cos = s_turn[wave][0];
  float* s_sin = s_turn[wave][1];
  if (lane < half) {
    if (a.positions == nullptr) pos = place;
    const double turns = (double)pos * freq * 0.15915494309189533577;
    double s, c;
    sincospi(2.0 * (turns - rint(turns)), &s, &c);
    s_cos[lane] = (float)(c * a.scale); s_sin[lane] = (float)(s * a.scale);
  }
  __builtin_amdgcn_wave_barrier();                                     // (a wave's LDS accesses keep their order)
  uint8_t* q_to = a.q_out + (int64_t)row * a.H * row_bytes;
  uint8_t* k_to = a.k_pool + slot * a.H_kv * row_bytes;
  if constexpr (MODE == kPairs) {
    const int each = half + (D - a.rotary), all = (nq + (append ? nk : 0)) * each;   // pairs, then elements that pass through
    for (int j = v_lane; j < all; j += v_step) {
      const int h = j / each, i = j - h * each;
      const T* from = reinterpret_cast<const T*>(h < nq ? q_row + h * row_bytes : k_row + (h - nq) * row_bytes);
      T* to = reinterpret_cast<T*>(h < nq ? q_to + h * row_bytes : k_to + (h - nq) * row_bytes);
      if (i >= half) { to[half + i] = from[half + i]; continue; }      // element rotary + i - half
      const int p0 = a.adjacent ? 2 * i : i, p1 = a.adjacent ? 2 * i + 1 : i + half;
      const float x = to_f32<T>(from[p0]), y = to_f32<T>(from[p1]), c = s_cos[i], s = s_sin[i];
      to[p0] = from_f32<T>(x * c - y * s);
      to[p1] = from_f32<T>(x * s + y * c);
    }
  } else {
    constexpr int NP = MODE == kHalves ? VE : VE / 2;                  // pairs of a piece
    float c[NP], s[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) { c[i] = turns ? s_cos[u * NP + i] : 1.f; s[i] = turns ? s_sin[u * NP + i] : 0.f; }
    const int nh = nq + (append ? nk : 0);
    for (int h0 = side; h0 < nq + nk; h0 += step * UN) {
      if (h0 != side) load(h0);
#pragma unroll
      for (int k = 0; k < UN; ++k) {
        const int h = h0 + k * step;
        if (h >= nh || u >= units) continue;
        uint8_t* to = h < nq ? q_to + h * row_bytes : k_to + (h - nq) * row_bytes;
        if (turns) {
          piece_t x;
          x.load(v[k]);
          if constexpr (MODE == kHalves) {
            piece_t y;
            y.load(w[k]);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              const float f = x.x[i], g = y.x[i];
              x.x[i] = f * c[i] - g * s[i];
              y.x[i] = f * s[i] + g * c[i];
            }
            *reinterpret_cast<words_t*>(to + e1) = y.store();
          } else {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
              const float f = x.x[2 * i], g = x.x[2 * i + 1];
              x.x[2 * i] = f * c[i] - g * s[i];
              x.x[2 * i + 1] = f * s[i] + g * c[i];
            }
          }
          v[k] = x.store();
        }
        *reinterpret_cast<words_t*>(to + e0) = v[k];
      }
    }
  }
  if (append) {
    u32x4_t* to = reinterpret_cast<u32x4_t*>(a.v_pool + slot * a.H_kv * row_bytes);
    for (int i0 = v_lane; i0 < v_pieces; i0 += v_step * UN) {
      if (i0 != v_lane) load_v(i0);
#pragma unroll
      for (int k = 0; k < UN; ++k) if (i0 + k * v_step < v_pieces) to[i0 + k * v_step] = x[k];
    }
  }
}

template <typename T, int BYTES>
static void rope_launch(bool pairs, const RopeAppendArgs& a, dim3 grid, hipStream_t s) {
  if (pairs) hipLaunchKernelGGL((rope_append_kernel<T, kPairs, 16>), grid, dim3(256), 0, s, a);
  else if (a.adjacent) hipLaunchKernelGGL((rope_append_kernel<T, kNeighbours, BYTES>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((rope_append_kernel<T, kHalves, BYTES>), grid, dim3(256), 0, s, a);
}

template <typename T>
static hipError_t rope_one(const RopeAppendArgs& b, hipStream_t s) {
  RopeAppendArgs a = b;
  // pieces of 16 bytes, or of 8, whichever divide the rotated part (its halves), or single pairs
  auto divides = [&](int bytes) -> bool { return a.rotary % ((a.adjacent ? 1 : 2) * bytes / (int)sizeof(T)) == 0; };
  const bool pairs = !divides(8);
  const int ve = (divides(16) ? 16 : 8) / (int)sizeof(T), units = (a.adjacent ? a.rotary : a.rotary / 2) / ve + (a.D - a.rotary) / ve;
  int lanes = 64;                                // heads side by side
  while (lanes * units > 64) lanes >>= 1;
  const int heads = (a.q != nullptr ? a.H : 0) + (a.k != nullptr ? a.H_kv : 0);
  a.share_shift = a.T <= kRopeFew || pairs ? 2 : heads <= 2 * lanes ? 0 : 1;
  const long wgs = (((long)a.T << a.share_shift) + 3) / 4, wide = 1 << 20;      // (a grid has less than 2^32 threads in a dimension)
  const dim3 grid((unsigned)std::min(wgs, wide), (unsigned)((wgs + wide - 1) / wide));
  if (divides(16)) rope_launch<T, 16>(false, a, grid, s);
  else rope_launch<T, 8>(pairs, a, grid, s);
  return hipGetLastError();
}

hipError_t launch_rope_append(int dtype, const RopeAppendArgs& a, hipStream_t s) {
  return dtype == TS_BF16 ? rope_one<uint16_t>(a, s) : rope_one<float>(a, s);
}

}  // namespace ts
