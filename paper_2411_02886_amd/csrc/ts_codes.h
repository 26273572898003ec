// The 8-bit codes of a quantised cache: whole numbers and e4m3.
#pragma once
#include "ts_common.h"

#ifdef __HIPCC__
namespace ts {

template <int CODE> constexpr double kCodeTop = CODE == TS_INT8 ? 127. : 448.;

// four codes as floats
template <int CODE>
__device__ __forceinline__ void codes_to_f32(uint32_t w, float (&x)[4]) {
  if constexpr (CODE == TS_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
  }
}

// four codes as two pairs of bf16 numbers
template <int CODE>
__device__ __forceinline__ uint2 widen(uint32_t w) {
  if constexpr (CODE == TS_E4M3) {
    return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, true)));
  } else {                                     // a whole number of seven bits is the high half of its float
    float x[4];
    codes_to_f32<CODE>(w, x);
    return make_uint2(__builtin_amdgcn_perm(__float_as_uint(x[1]), __float_as_uint(x[0]), 0x07060302u),
                      __builtin_amdgcn_perm(__float_as_uint(x[3]), __float_as_uint(x[2]), 0x07060302u));
  }
}
}  // namespace ts
#endif
