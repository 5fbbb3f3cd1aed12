// The experts' outputs joined per token, and the gradient of that.
//
//     y_t = sum_j w_tj z_{slots(t,j)},
//     dz_{slots(t,j)} = w_tj dy_t,   dw_tj = <dy_t, z_{slots(t,j)}>.
//
// Every row of z is read once and every result written once: the kernels are
// bound by memory.  Sums run over j (and over d, for dw) in a fixed order in
// fp32.
#include <cstdint>
#include <string>

#include "common.hpp"
#include "internal.hpp"

namespace bitsmoe {
namespace {

constexpr int kThreads = 256;

// 16 bytes of a row as fp32.
template <bool BF16>
struct Piece {
  static constexpr int kLen = BF16 ? 8 : 4;
  float v[kLen];
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
      const f32x4 u = static_cast<const f32x4*>(row)[i];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = u[q];
    }
  }
  __device__ __forceinline__ void store(void* row, int64_t i) const {
    if constexpr (BF16) {
      bf16x8 u;
#pragma unroll
      for (int q = 0; q < 8; ++q) u[q] = static_cast<__bf16>(v[q]);
      static_cast<bf16x8*>(row)[i] = u;
    } else {
      f32x4 u;
#pragma unroll
      for (int q = 0; q < 4; ++q) u[q] = v[q];
      static_cast<f32x4*>(row)[i] = u;
    }
  }
};

struct CombineArgs {
  const void* z;
  const int32_t* slots;
  const float* weights;
  const void* dy;
  void* y;  // or dz
  float* dweights;
  int64_t S, T;
  int k, pieces;  // 16-byte pieces of a row
};

// 16 bytes of a result a thread: neighbours read neighbours of the same k rows.
// 1003 tokens, k = 8, 2048 bf16 (37 MB): 8.5 us; 8192 tokens, k = 2, 4096 (201 MB):
// 34 us, 5.9 TB/s.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void combine_kernel(CombineArgs a) {
  using P = Piece<BF16>;
  const int64_t n = a.T * a.pieces, rowb = int64_t(a.pieces) * 16;
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    const int64_t t = i / a.pieces;
    const int c = static_cast<int>(i - t * a.pieces);
    P acc;
#pragma unroll
    for (int q = 0; q < P::kLen; ++q) acc.v[q] = 0.0f;
    for (int j = 0; j < a.k; ++j) {
      const int s = a.slots[t * a.k + j];
      if (s < 0 || s >= a.S) continue;
      const float w = a.weights ? a.weights[t * a.k + j] : 1.0f;
      P z;
      z.load(static_cast<const char*>(a.z) + s * rowb, c);
#pragma unroll
      for (int q = 0; q < P::kLen; ++q) acc.v[q] = fmaf(w, z.v[q], acc.v[q]);
    }
    acc.store(static_cast<char*>(a.y) + t * rowb, c);
  }
}

// One workgroup per token: dy's row stays in its caches for the k slots, and dw is
// a sum over the workgroup.  8192 tokens, k = 2, 4096 bf16 (0.34 GB): 65 us, 5.2 TB/s.
template <bool BF16>
__global__ __launch_bounds__(kThreads) void combine_grad_kernel(CombineArgs a) {
  using P = Piece<BF16>;
  __shared__ float part[BITSMOE_ROUTE_MAX_K][kThreads / 64];
  const int64_t t = blockIdx.x, rowb = int64_t(a.pieces) * 16;
  const int tid = threadIdx.x;
  const char* dy = static_cast<const char*>(a.dy) + t * rowb;
  for (int j = 0; j < a.k; ++j) {
    const int s = a.slots[t * a.k + j];
    const bool in = s >= 0 && s < a.S;
    const float w = a.weights ? a.weights[t * a.k + j] : 1.0f;
    float dot = 0.0f;
    if (in)
      for (int c = tid; c < a.pieces; c += kThreads) {
        P g, z;
        g.load(dy, c);
        if (a.dweights) {
          z.load(static_cast<const char*>(a.z) + s * rowb, c);
#pragma unroll
          for (int q = 0; q < P::kLen; ++q) dot = fmaf(g.v[q], z.v[q], dot);
        }
#pragma unroll
        for (int q = 0; q < P::kLen; ++q) g.v[q] *= w;
        g.store(static_cast<char*>(a.y) + s * rowb, c);
      }
    if (a.dweights) {
      dot = wave_sum(dot);
      if ((tid & 63) == 0) part[j][tid >> 6] = dot;
    }
  }
  if (!a.dweights) return;
  __syncthreads();
  if (tid < a.k) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += part[tid][w];
    a.dweights[t * a.k + tid] = s;
  }
}

bitsmoe_status check(const char* who, bitsmoe_dtype zt, int64_t S, int64_t T, int64_t k, int64_t d) {
  if (S < 0 || T < 0 || k <= 0 || d <= 0)
    return fail(BITSMOE_ERR_ARG, std::string(who) + ": non-positive size");
  if (zt != BITSMOE_F32 && zt != BITSMOE_BF16)
    return fail(BITSMOE_ERR_DTYPE, std::string(who) + ": rows must be fp32 or bf16");
  if (d % 8 != 0 || d > (int64_t(1) << 24) || k > BITSMOE_ROUTE_MAX_K || S > 0x7FFFFFFF || T > 0x7FFFFFFF)
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": needs d % 8 == 0, d <= 2^24, k <= 64, S and T < 2^31");
  return BITSMOE_OK;
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" bitsmoe_status bitsmoe_combine(const void* Z_dev, bitsmoe_dtype zt, int64_t S, const int32_t* slots_dev,
                                          const float* weights_dev, int64_t T, int64_t k, int64_t d, void* Y_dev,
                                          void* stream) {
  if (bitsmoe_status st = check("combine", zt, S, T, k, d)) return st;
  if (T == 0) return ok();
  if ((S > 0 && !Z_dev) || !slots_dev || !Y_dev) return fail(BITSMOE_ERR_ARG, "combine: null pointer");
  if (!aligned16({Z_dev, slots_dev, weights_dev, Y_dev}))
    return fail(BITSMOE_ERR_ARG, "combine: device pointers must be 16-byte aligned");
  CombineArgs a{Z_dev, slots_dev, weights_dev, nullptr, Y_dev, nullptr, S, T, static_cast<int>(k),
                static_cast<int>(d / (zt == BITSMOE_BF16 ? 8 : 4))};
  const int64_t blocks = (T * a.pieces + kThreads - 1) / kThreads;
  const unsigned grid = static_cast<unsigned>(blocks < (1 << 20) ? blocks : (1 << 20));
  auto* fn = zt == BITSMOE_BF16 ? combine_kernel<true> : combine_kernel<false>;
  fn<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("combine_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_combine_grad(const void* Z_dev, bitsmoe_dtype zt, int64_t S,
                                               const int32_t* slots_dev, const float* weights_dev,
                                               const void* dY_dev, int64_t T, int64_t k, int64_t d, void* dZ_dev,
                                               float* dweights_dev, void* stream) {
  if (bitsmoe_status st = check("combine_grad", zt, S, T, k, d)) return st;
  if (T == 0) return ok();
  if (!slots_dev || !dY_dev || (S > 0 && !dZ_dev) || (dweights_dev && S > 0 && !Z_dev))
    return fail(BITSMOE_ERR_ARG, "combine_grad: null pointer");
  if (!aligned16({Z_dev, slots_dev, weights_dev, dY_dev, dZ_dev, dweights_dev}))
    return fail(BITSMOE_ERR_ARG, "combine_grad: device pointers must be 16-byte aligned");
  CombineArgs a{Z_dev, slots_dev, weights_dev, dY_dev, dZ_dev, dweights_dev, S, T, static_cast<int>(k),
                static_cast<int>(d / (zt == BITSMOE_BF16 ? 8 : 4))};
  auto* fn = zt == BITSMOE_BF16 ? combine_grad_kernel<true> : combine_grad_kernel<false>;
  if (T >= (int64_t(1) << 24))
    return fail(BITSMOE_ERR_SHAPE, "combine_grad: needs T < 2^24");
  fn<<<static_cast<unsigned>(T), kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("combine_grad_kernel");
  return ok();
}
