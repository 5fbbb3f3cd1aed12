// MX8: the microscaled 8-bit format of activations that are kept for the
// backward pass.  A row is cut into blocks of 32 entries; a block has one scale
// 2^(s - 127), s a byte (255: the block held a NaN or an infinity, and stands for
// NaN), and each entry is an E4M3 float (sign, four exponent bits, three of the
// fraction; largest 448).
//
// The scale is the smallest power of two at which the block's largest magnitude
// does not pass 448, so no entry is cut off: each is off by 2^-4 of itself at
// most, or by 2^-10 scales where it is below 2^-6 of them.
#pragma once

#include "mx4.hpp"

namespace bitsmoe {

constexpr int kMx8Block = 32;

// Scale byte of a block whose largest magnitude has these bits (a NaN's and an
// infinity's lie above every number's): 448 = 1.75 2^8.
__device__ __forceinline__ uint32_t mx8_scale_byte(uint32_t top) {
  const int e = static_cast<int>(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return top >= 0x7F800000u ? 255u : e > 0 ? static_cast<uint32_t>(e) : 0u;
}

// Eight entries of a block that lies on four neighbouring lanes to codes and the
// block's scale byte.  All four lanes are active.
__device__ __forceinline__ uint2 mx8_codes(const float (&v)[8], uint32_t* scale_byte) {
  uint32_t top = 0;
#pragma unroll
  for (int q = 0; q < 8; ++q) top = max(top, __float_as_uint(v[q]) & 0x7FFFFFFFu);
  top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), 0xB1, 0xF, 0xF, false)));
  top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(top), 0x4E, 0xF, 0xF, false)));
  const uint32_t s = mx8_scale_byte(top);
  const float scale = mx4_scale(s);  // (the conversions read a scale alike)
  typedef __attribute__((ext_vector_type(2))) short s16x2;
  s16x2 a = {0, 0}, b = {0, 0};
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[0], v[1], scale, false);
  a = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(a, v[2], v[3], scale, true);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[4], v[5], scale, false);
  b = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(b, v[6], v[7], scale, true);
  *scale_byte = s;
  const bool lost = s == 255u;
  return make_uint2(lost ? 0u : __builtin_bit_cast(uint32_t, a), lost ? 0u : __builtin_bit_cast(uint32_t, b));
}

// What eight codes stand for, in fp32 (exact).
__device__ __forceinline__ void mx8_values(uint2 c, uint32_t scale_byte, float (&v)[8]) {
  const float scale = mx4_scale(scale_byte);
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, scale, false);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, scale, true);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, scale, false);
  const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, scale, true);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
  v[4] = d[0], v[5] = d[1], v[6] = e[0], v[7] = e[1];
}

}  // namespace bitsmoe
