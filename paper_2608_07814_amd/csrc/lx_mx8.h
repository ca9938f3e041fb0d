// Microscaled 8-bit values on the device: a block of 32 under one power of two,
// elements e4m3 (layout and rule in lorex_block.h).
#pragma once

#include "lx_vec.h"

namespace lx {

// 8 values of a lane to codes; 4 consecutive lanes (all active) share a block. The
// block's largest magnitude goes over the lanes as bits: as unsigned integers
// magnitudes keep their order, and infinities and NaNs come out above every finite
// one. s: the scale's byte, the smallest for which that magnitude is at most 448
// (1.75 2^8): eight below its exponent, one more where it is past 1.75. The product
// with the scale's inverse is exact (2^(127 - s), a normal number for every s that
// occurs), the conversion rounds to nearest even and never saturates.
__device__ __forceinline__ uint2 mx8_round(const F8& x, int& s) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x.v[e]) & 0x7FFFFFFFu);
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));
  top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
  const int e = (int)(top >> 23);  // biased; 255: infinity or NaN
  s = max(e - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0), 0);
  const float f = __uint_as_float((uint32_t)(254 - s) << 23);
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x.v[0] * f, x.v[1] * f, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(x.v[2] * f, x.v[3] * f, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x.v[4] * f, x.v[5] * f, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(x.v[6] * f, x.v[7] * f, hi, true);
  if (e == 255) {
    s = 255;
    lo = hi = 0;
  }
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

// What a scale's byte stands for (255: NaN; 2^-127 is not a normal number).
__device__ __forceinline__ float mx_scale(uint32_t s) {
  return __uint_as_float(s == 255 ? 0x7FC00000u : s ? s << 23 : 0x00400000u);
}

}  // namespace lx
