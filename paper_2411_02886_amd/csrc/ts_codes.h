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

}  // namespace ts
#endif
