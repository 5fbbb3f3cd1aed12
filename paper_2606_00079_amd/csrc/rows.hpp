// Eight consecutive entries of a row of bf16 or fp32 as fp32 values.
#pragma once

#include "common.hpp"

namespace bitsmoe {

template <bool BF16>
struct Eight {
  static constexpr int kBytes = BF16 ? 2 : 4;  // of an entry
  float v[8];
  // piece i (entries 8 i .. 8 i + 7) of a row; 16-byte aligned
  __device__ __forceinline__ void load(const void* row, int64_t i) {
    if constexpr (BF16) {
      const uint4 u = static_cast<const uint4*>(row)[i];
      const uint32_t d[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[2 * q] = __uint_as_float(d[q] << 16);
        v[2 * q + 1] = __uint_as_float(d[q] & 0xFFFF0000u);
      }
    } else {
      const f32x4 a = static_cast<const f32x4*>(row)[2 * i], b = static_cast<const f32x4*>(row)[2 * i + 1];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] = a[q];
        v[4 + q] = b[q];
      }
    }
  }
  __device__ __forceinline__ void store(void* row, int64_t i) const {
    if constexpr (BF16) {
      bf16x8 u;
#pragma unroll
      for (int q = 0; q < 8; ++q) u[q] = static_cast<__bf16>(v[q]);
      static_cast<bf16x8*>(row)[i] = u;
    } else {
      static_cast<f32x4*>(row)[2 * i] = f32x4{v[0], v[1], v[2], v[3]};
      static_cast<f32x4*>(row)[2 * i + 1] = f32x4{v[4], v[5], v[6], v[7]};
    }
  }
  // the values as the type holds them
  __device__ __forceinline__ void round() {
    if constexpr (BF16) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = static_cast<float>(static_cast<__bf16>(v[q]));
    }
  }
};

// The same as they lie in memory: what is on its way for the next row takes half the
// registers in bf16.
template <bool BF16>
struct RawEight {
  uint4 u[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* row, int64_t i) {
#pragma unroll
    for (int q = 0; q < (BF16 ? 1 : 2); ++q) u[q] = static_cast<const uint4*>(row)[i * (BF16 ? 1 : 2) + q];
  }
  __device__ __forceinline__ float value(int q) const {
    if constexpr (BF16) {
      const uint32_t d = q < 2 ? u[0].x : q < 4 ? u[0].y : q < 6 ? u[0].z : u[0].w;
      return __uint_as_float(q & 1 ? d & 0xFFFF0000u : d << 16);
    } else {
      const uint4 w = u[q >> 2];
      return __uint_as_float((q & 3) == 0 ? w.x : (q & 3) == 1 ? w.y : (q & 3) == 2 ? w.z : w.w);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < (BF16 ? 1 : 2); ++q) u[q] = make_uint4(0, 0, 0, 0);
  }
};

}  // namespace bitsmoe
