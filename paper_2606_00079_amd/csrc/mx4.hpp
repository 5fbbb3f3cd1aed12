// MX4: the microscaled 4-bit format of the experts' products.  A row is cut
// into blocks of 32 entries; a block has one scale 2^(s - 127), s a byte (255:
// the block held a NaN or an infinity, and stands for NaN), and each entry is
// a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 in four bits, entry 2i in the
// low half of byte i.
#pragma once

#include "common.hpp"

namespace bitsmoe {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int kMx4Block = 32;

// The scale as the conversion instructions take it: they read the exponent
// bits of a float alone, so 0 stands for 2^-127 and 255 gives NaN.
__device__ __forceinline__ float mx4_scale(uint32_t s) { return __uint_as_float(s << 23); }

// The eight entries of a word of codes as bf16.  Exact: a value has two
// significant bits and lies in bf16's range (down to its subnormals).
__device__ __forceinline__ uint4 mx4_bf16_words(uint32_t w, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
}
__device__ __forceinline__ bf16x8 mx4_bf16(uint32_t w, float scale) {
  return __builtin_bit_cast(bf16x8, mx4_bf16_words(w, scale));
}

}  // namespace bitsmoe
