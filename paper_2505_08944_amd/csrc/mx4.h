// Values in 4 bits (OCP MXFP4): blocks of 32 consecutive values share a power of
// two, held as its exponent + 127 in a byte; a value is a code of 4 bits, sign and
// one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, two codes to a byte, the earlier one in its
// low half.  gfx950 converts both ways: checked on the card for all codes and all
// scales, the values that come back are exact bf16 from 0.5 2^-127 on (of 2^128 and more, under
// the bytes 253 and 254, infinity), scale byte 255 gives NaN, and f32 values go to the
// nearest code, in the middle to the even one, at most 6.
#pragma once

#include "aep_device.h"
#include "aep_internal.h"

namespace aep {

constexpr uint32_t kMx4NaN = 255;  // scale of a block that holds a NaN or an infinity

__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// One byte of codes, number B of w, to two bf16 (the earlier value in the low half).
template <int B>
__device__ __forceinline__ uint32_t mx4_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B));
}
// Eight values.
__device__ __forceinline__ uint4 mx4_bf16x8(uint32_t w, float scale) {
  return make_uint4(mx4_pair<0>(w, scale), mx4_pair<1>(w, scale), mx4_pair<2>(w, scale), mx4_pair<3>(w, scale));
}
// Eight f32 values to codes.
__device__ __forceinline__ uint32_t mx4_codes(const float* v, float scale) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}
// The largest of a quad of lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, true));         // lanes 1 0 3 2
  return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, true));      // lanes 2 3 0 1
}

// The scale byte of a block whose largest magnitude has these bits: the smallest
// power of two, from 2^-126 on, at which it is at most 7 (1.75 * 4): no value is then
// off by more than the power, and for normally distributed values the mean square of
// what is lost is least (1.25% of the values' own; a limit of 6 loses 1.34%, of 8
// 1.32%).  At most 2^125, so that what is finite stays so.  A block of zeros has 2^0.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits) {
  const uint32_t e = amax_bits >> 23;
  if (e == 255) return kMx4NaN;
  if (amax_bits == 0) return 127;
  return (uint32_t)min(max(1, (int)e - 2 + (int)((amax_bits & 0x7fffffu) > 0x600000u)), 252);
}

}  // namespace aep
