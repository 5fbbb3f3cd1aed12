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
  // where rows that no slot names are cleared
  int clear;             // the first workgroups of the launch, which do that
  const int32_t* names;  // [S]: a slot (its place in slots) that names the row, if one does; else anything
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

// Which rows of dz no slot names, and so get 0: kLeave, they are the caller's;
// kScan, a clearing workgroup looks through all slots for those that name one of
// its rows; kMarks, combine_names_kernel has written down a slot for each named row.
enum Rest { kLeave, kScan, kMarks };

// 0 to the rows of dz that no slot names, a row a thread.
template <bool BF16, Rest REST>
__device__ __forceinline__ void clear_unnamed(const CombineArgs& a) {
  using P = Piece<BF16>;
  __shared__ uint32_t named[kThreads / 32];
  const int64_t n = a.T * a.k, rowb = int64_t(a.pieces) * 16;
  const int tid = threadIdx.x;
  for (int64_t row0 = int64_t(blockIdx.x) * kThreads; row0 < a.S; row0 += int64_t(a.clear) * kThreads) {
    const int64_t s = row0 + tid;
    bool unnamed = s < a.S;
    if constexpr (REST == kScan) {
      __syncthreads();
      if (tid < kThreads / 32) named[tid] = 0;
      __syncthreads();
      auto look = [&](int slot) {
        const int64_t r = slot - row0;
        if (r >= 0 && r < kThreads) atomicOr(&named[r >> 5], 1u << (r & 31));
      };
      const int4* four = reinterpret_cast<const int4*>(a.slots);
      const int pieces = static_cast<int>(n / 4);  // (n <= BITSMOE_COMBINE_SCAN)
      for (int i = tid; i < pieces; i += 8 * kThreads) {  // eight loads under way
        int4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u)
          v[u] = i + u * kThreads < pieces ? four[i + u * kThreads] : make_int4(-1, -1, -1, -1);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          look(v[u].x);
          look(v[u].y);
          look(v[u].z);
          look(v[u].w);
        }
      }
      if (tid < (n & 3)) look(a.slots[(n & ~int64_t(3)) + tid]);
      __syncthreads();
      unnamed = unnamed && !(named[tid >> 5] >> (tid & 31) & 1);
    } else if (unnamed) {
      const int64_t i = a.names[s];
      unnamed = i < 0 || i >= n || a.slots[i] != s;
    }
    for (uint64_t m = __ballot(unnamed); m; m &= m - 1) {  // a wave a row
      P zero;
#pragma unroll
      for (int q = 0; q < P::kLen; ++q) zero.v[q] = 0.0f;
      char* row = static_cast<char*>(a.y) + (row0 + (tid & ~63) + __builtin_ctzll(m)) * rowb;
      for (int c = tid & 63; c < a.pieces; c += 64) zero.store(row, c);
    }
  }
}

// One workgroup per token: dy's row stays in its caches for the k slots, and dw is
// a sum over the workgroup.  8192 tokens, k = 2, 4096 bf16 (0.34 GB): 65 us, 5.2 TB/s.
template <bool BF16, Rest REST>
__global__ __launch_bounds__(kThreads) void combine_grad_kernel(CombineArgs a) {
  using P = Piece<BF16>;
  __shared__ float part[BITSMOE_ROUTE_MAX_K][kThreads / 64];
  if constexpr (REST != kLeave) {
    if (static_cast<int>(blockIdx.x) < a.clear) {
      clear_unnamed<BF16, REST>(a);
      return;
    }
  }
  const int64_t t = static_cast<int64_t>(blockIdx.x) - (REST != kLeave ? a.clear : 0);
  const int64_t rowb = int64_t(a.pieces) * 16;
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

// A slot for every row that one names; what names [S] held before does not matter.
__global__ __launch_bounds__(kThreads) void combine_names_kernel(const int32_t* slots, int64_t n, int64_t S,
                                                                 int32_t* names) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    const int s = slots[i];
    if (s >= 0 && s < S) names[s] = static_cast<int32_t>(i);
  }
}

unsigned grid_for(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return static_cast<unsigned>(b < (1 << 20) ? b : (1 << 20));
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

// Both forms of the gradient: `all` gives the rows that no slot names 0.
bitsmoe_status run_grad(const char* who, const void* Z_dev, bitsmoe_dtype zt, int64_t S, const int32_t* slots_dev,
                        const float* weights_dev, const void* dY_dev, int64_t T, int64_t k, int64_t d, void* dZ_dev,
                        float* dweights_dev, bool all, int32_t* work_dev, void* stream) {
  auto bad = [who](bitsmoe_status st, const char* what) { return fail(st, std::string(who) + what); };
  if (bitsmoe_status st = check(who, zt, S, T, k, d)) return st;
  if (T >= (int64_t(1) << 24)) return bad(BITSMOE_ERR_SHAPE, ": needs T < 2^24");
  if (T == 0 && (!all || S == 0)) return ok();
  if ((T > 0 && (!slots_dev || !dY_dev || (dweights_dev && S > 0 && !Z_dev))) || (S > 0 && !dZ_dev))
    return bad(BITSMOE_ERR_ARG, ": null pointer");
  // Looking through the slots hides behind the tokens' work up to here (16384 slots, rows of 4096: 96 us forward and
  // back, as without; 16000, rows of 128: 16.4 instead of 14.4); marks take a launch of their own, 2.5 us: 65536 slots,
  // rows of 512, 65 us with marks, 68 by looking, 62 without either.
  const bool marks = all && S > 0 && T * k > BITSMOE_COMBINE_SCAN;
  if (marks && !work_dev) return bad(BITSMOE_ERR_ARG, ": this many slots need the workspace");
  if (!aligned16({Z_dev, slots_dev, weights_dev, dY_dev, dZ_dev, dweights_dev, work_dev}))
    return bad(BITSMOE_ERR_ARG, ": device pointers must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = zt == BITSMOE_BF16;
  CombineArgs a{Z_dev, slots_dev, weights_dev, dY_dev, dZ_dev, dweights_dev, S, T, static_cast<int>(k),
                static_cast<int>(d / (bf16 ? 8 : 4)), 0, work_dev};
  if (T == 0) {  // sums of no slots
    a.T = S;
    a.k = 0;
    auto* fn = bf16 ? combine_kernel<true> : combine_kernel<false>;
    fn<<<grid_for(S * a.pieces), kThreads, 0, s>>>(a);
    BITSMOE_LAUNCH_CHECK("combine_kernel");
    return ok();
  }
  int64_t grid = T;
  if (all) {
    // (a multiple of 8, so that a token stays on the XCD whose L2 has its rows from the forward form: 520 tokens, k = 8,
    // 2048 bf16, forward and back take 17 us, and 20 with 17 clearing workgroups)
    const int64_t clear = (S + 8 * kThreads - 1) / (8 * kThreads) * 8;
    a.clear = static_cast<int>(clear < 4096 ? clear : 4096);
    grid += a.clear;
  }
  if (marks) {
    combine_names_kernel<<<grid_for(T * k), kThreads, 0, s>>>(slots_dev, T * k, S, work_dev);
    BITSMOE_LAUNCH_CHECK("combine_names_kernel");
  }
  auto* fn = !all    ? (bf16 ? combine_grad_kernel<true, kLeave> : combine_grad_kernel<false, kLeave>)
             : marks ? (bf16 ? combine_grad_kernel<true, kMarks> : combine_grad_kernel<false, kMarks>)
                     : (bf16 ? combine_grad_kernel<true, kScan> : combine_grad_kernel<false, kScan>);
  if (grid >= (int64_t(1) << 24)) {  // (2^32 threads: the clearing goes by itself)
    auto* tokens = bf16 ? combine_grad_kernel<true, kLeave> : combine_grad_kernel<false, kLeave>;
    tokens<<<static_cast<unsigned>(T), kThreads, 0, s>>>(a);
    BITSMOE_LAUNCH_CHECK("combine_grad_kernel");
    grid = a.clear;
  }
  fn<<<static_cast<unsigned>(grid), kThreads, 0, s>>>(a);
  BITSMOE_LAUNCH_CHECK("combine_grad_kernel");
  return ok();
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
                static_cast<int>(d / (zt == BITSMOE_BF16 ? 8 : 4)), 0, nullptr};
  auto* fn = zt == BITSMOE_BF16 ? combine_kernel<true> : combine_kernel<false>;
  fn<<<grid_for(T * a.pieces), kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("combine_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_combine_grad(const void* Z_dev, bitsmoe_dtype zt, int64_t S,
                                               const int32_t* slots_dev, const float* weights_dev,
                                               const void* dY_dev, int64_t T, int64_t k, int64_t d, void* dZ_dev,
                                               float* dweights_dev, void* stream) {
  return run_grad("combine_grad", Z_dev, zt, S, slots_dev, weights_dev, dY_dev, T, k, d, dZ_dev, dweights_dev, false,
                  nullptr, stream);
}

extern "C" bitsmoe_status bitsmoe_combine_grad_all(const void* Z_dev, bitsmoe_dtype zt, int64_t S,
                                                   const int32_t* slots_dev, const float* weights_dev,
                                                   const void* dY_dev, int64_t T, int64_t k, int64_t d, void* dZ_dev,
                                                   float* dweights_dev, int32_t* work_dev, void* stream) {
  return run_grad("combine_grad_all", Z_dev, zt, S, slots_dev, weights_dev, dY_dev, T, k, d, dZ_dev, dweights_dev,
                  true, work_dev, stream);
}
