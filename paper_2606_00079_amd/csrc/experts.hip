// Products of tokens in expert order with bf16 expert weights.
//
//     y_s = W_e(s) x_row(s)                            (expert_product)
//     y_s = silu(g) u, [g; u] = W_e(s) x_row(s)        (the same with glu)
//     dx_s = W_e(s)^T dy_s                             (expert_product_grad)
//     dW_e = sum over e's slots of dy_s x_row(s)^T     (expert_weight_grad; _q: x in MX8)
//
// for S slots, expert e's being offsets[e] .. offsets[e+1].  Sums are fp32 and
// results are rounded once.
#include <cstdint>
#include <string>

#include "internal.hpp"
#include "mx8.hpp"
#include "slots.hpp"

namespace bitsmoe {
namespace {

constexpr int kThreads = 256;

struct ExpertArgs {
  const uint16_t* w;  // [E][N or 2 N][K]
  int E;
  int64_t N, K;
  const uint16_t* x;       // rows of K (weight gradient: or in MX8)
  const uint8_t* xcodes;
  const uint8_t* xscales;
  int64_t x_rows, ldx;
  const uint16_t* dy;  // rows of N
  int64_t lddy;
  const int32_t* offsets;
  const int32_t* rows;
  int64_t S;
  void* y;
  int64_t ldy;
  int yf32;
};

enum Form { kForward, kTokens, kWeights };

// 64 x 64 results a workgroup, the sum 32 entries at a time through LDS.
template <Form FORM, bool MX, bool GLU>
__global__ __launch_bounds__(kThreads) void expert_simple_kernel(ExpertArgs a) {
  constexpr int H = GLU ? 2 : 1, LD = 40;
  __shared__ __align__(16) uint16_t p[64 * LD], q[H][64 * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int e, lo = 0, hi = 0;
  int64_t m0, n0;  // of the results
  if constexpr (FORM == kWeights) {
    const int64_t nt = (a.N + 63) / 64, kt = (a.K + 63) / 64;
    e = static_cast<int>(blockIdx.x / (nt * kt));
    const int64_t in = blockIdx.x % (nt * kt);
    m0 = in / kt * 64;
    n0 = in % kt * 64;
    const int count = slots_of(a.offsets, a.E, static_cast<int>(a.S), e, &lo);
    hi = lo + count;
  } else {
    const int64_t cols = FORM == kForward ? a.N : a.K;
    Tile t;
    if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((cols + 63) / 64), 64, &t)) return;
    e = t.e;
    m0 = lo = t.lo;
    hi = t.hi;
    n0 = static_cast<int64_t>(t.col) * 64;
  }
  const int64_t L = FORM == kForward ? a.K : FORM == kTokens ? a.N : hi - lo;  // of the sum
  const int64_t mend = FORM == kWeights ? a.N : hi, nend = FORM == kForward ? a.N : a.K;
  f32x4 acc[H][4];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[h][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto token = [&](int64_t s) {  // the row of slot s; -1: none
    const int64_t r = a.rows ? a.rows[s] : s;
    return r >= 0 && r < a.x_rows ? r : -1;
  };
  if (FORM == kWeights || e < a.E) {
    for (int64_t k0 = 0; k0 < L; k0 += 32) {
      __syncthreads();
      for (int i = tid; i < 64 * 32; i += kThreads) {
        const int m = FORM == kWeights ? i % 64 : i / 32, k = FORM == kWeights ? i / 64 : i % 32;
        uint16_t v = 0;
        if (m0 + m < mend && k0 + k < L) {
          if constexpr (FORM == kForward) {
            const int64_t r = token(m0 + m);
            if (r >= 0) v = a.x[r * a.ldx + k0 + k];
          } else if constexpr (FORM == kTokens) {
            v = a.dy[(m0 + m) * a.lddy + k0 + k];
          } else {
            if (token(lo + k0 + k) >= 0) v = a.dy[(lo + k0 + k) * a.lddy + m0 + m];
          }
        }
        p[m * LD + k] = v;
      }
      for (int h = 0; h < H; ++h)
        for (int i = tid; i < 64 * 32; i += kThreads) {
          const int n = FORM == kForward ? i / 32 : i % 64, k = FORM == kForward ? i % 32 : i / 64;
          uint16_t v = 0;
          if (n0 + n < nend && k0 + k < L) {
            if constexpr (FORM == kForward) {
              v = a.w[((e * int64_t(H) + h) * a.N + n0 + n) * a.K + k0 + k];
            } else if constexpr (FORM == kTokens) {
              v = a.w[(e * a.N + k0 + k) * a.K + n0 + n];
            } else {
              const int64_t r = token(lo + k0 + k);
              if (r >= 0) {
                if constexpr (MX) {
                  const uint32_t c = a.xcodes[r * a.K + n0 + n];
                  const float scale = mx4_scale(a.xscales[(r * a.K + n0 + n) / 32]);
                  v = f32_to_bf16(__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, scale, false)[0]);
                } else {
                  v = a.x[r * a.ldx + n0 + n];
                }
              }
            }
          }
          q[h][n * LD + k] = v;
        }
      __syncthreads();
      const bf16x8 b = *reinterpret_cast<const bf16x8*>(p + (wave * 16 + (lane & 15)) * LD + 8 * (lane >> 4));
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[h][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              *reinterpret_cast<const bf16x8*>(q[h] + (i * 16 + (lane & 15)) * LD + 8 * (lane >> 4)), b, acc[h][i], 0,
              0, 0);
    }
  }
  const int64_t m = m0 + wave * 16 + (lane & 15);
  if (m >= mend) return;
  bool have = true;
  if constexpr (FORM == kForward) have = e < a.E && token(m) >= 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f32x4 v = acc[0][i];
    if constexpr (GLU) {
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = silu(v[u]) * acc[1][i][u];
    }
    if (!have) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    const int64_t n = n0 + i * 16 + 4 * (lane >> 4);
    if (n < nend) store4(a, FORM == kWeights ? e * a.N + m : m, n, nend, a.ldy % 4 == 0, v);
  }
}

constexpr int kLargestTile = 256;

bitsmoe_status check(const char* who, const ExpertArgs& a, bitsmoe_dtype t, bitsmoe_dtype yt, int64_t cols) {
  auto bad = [who](bitsmoe_status st, const char* what) { return fail(st, std::string(who) + what); };
  if (a.E <= 0 || a.N <= 0 || a.K <= 0 || a.S < 0 || a.x_rows < 0) return bad(BITSMOE_ERR_ARG, ": non-positive size");
  if (t != BITSMOE_BF16) return bad(BITSMOE_ERR_DTYPE, ": weights and rows must be bf16");
  if (yt != BITSMOE_F32 && yt != BITSMOE_BF16) return bad(BITSMOE_ERR_DTYPE, ": results are fp32 or bf16");
  // (slots are ints, and the end of a tile that begins at one is too)
  if (a.K % 8 != 0 || a.K > (1 << 24) || a.N > (1 << 24) || a.E > 65535 || a.S > 0x7FFFFFFF - kLargestTile ||
      a.x_rows > 0x7FFFFFFF)
    return bad(BITSMOE_ERR_SHAPE, ": needs K % 8 == 0, K and N <= 2^24, E <= 65535, S < 2^31 - 256 and rows < 2^31");
  if (a.ldy < cols || a.ldy > (int64_t(1) << 32))
    return bad(BITSMOE_ERR_SHAPE, ": the results' row stride is too small or too large");
  if (!a.offsets && a.E != 1) return bad(BITSMOE_ERR_ARG, ": no offsets, and more than one expert");
  if (!a.rows && a.x_rows < a.S) return bad(BITSMOE_ERR_SHAPE, ": fewer rows than slots");
  if (!aligned16({a.w, a.x, a.xcodes, a.xscales, a.dy, a.offsets, a.rows, a.y}))
    return bad(BITSMOE_ERR_ARG, ": device pointers must be 16-byte aligned");
  return BITSMOE_OK;
}

bitsmoe_status check_stride(const char* who, int64_t cols, int64_t ld) {
  if (ld < cols || ld % 8 != 0 || ld > (int64_t(1) << 32))
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": rows must not overlap, and lie a multiple of 16 bytes apart");
  return BITSMOE_OK;
}

// Workgroups for tiles of `tile` slots and `per` workgroups each.
bool grid_of(const ExpertArgs& a, int64_t tile, int64_t per, unsigned* grid) {
  const int64_t tiles = a.S / tile + (a.E + 2 < a.S ? a.E + 2 : a.S);  // (every run's last one may be part)
  if (tiles > ((int64_t(1) << 23) - 1) / per) return false;
  *grid = static_cast<unsigned>(tiles * per);
  return true;
}

int clip(int64_t E) { return static_cast<int>(E < 0x7FFFFFFF ? E : 0x7FFFFFFF); }

bitsmoe_status weight_grad(const char* who, const ExpertArgs& a, hipStream_t s) {
  const int64_t tiles = (a.N + 63) / 64 * ((a.K + 63) / 64);
  if (tiles > ((int64_t(1) << 23) - 1) / a.E) return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": too many weights");
  auto* fn = a.xcodes ? expert_simple_kernel<kWeights, true, false> : expert_simple_kernel<kWeights, false, false>;
  fn<<<static_cast<unsigned>(tiles * a.E), kThreads, 0, s>>>(a);
  BITSMOE_LAUNCH_CHECK("expert_simple_kernel");
  return ok();
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" bitsmoe_status bitsmoe_expert_product(const void* W_dev, bitsmoe_dtype t, int64_t E, int64_t N, int64_t K,
                                                 const void* X_dev, int64_t x_rows, int64_t ldx,
                                                 const int32_t* offsets_dev, const int32_t* rows_dev, int64_t S,
                                                 int glu, void* Y_dev, bitsmoe_dtype yt, int64_t ldy, void* stream) {
  const ExpertArgs a{static_cast<const uint16_t*>(W_dev), clip(E), N, K, static_cast<const uint16_t*>(X_dev),
                     nullptr, nullptr, x_rows, ldx, nullptr, 0, offsets_dev, rows_dev, S, Y_dev, ldy,
                     yt == BITSMOE_F32};
  if (bitsmoe_status st = check("expert_product", a, t, yt, N)) return st;
  if (bitsmoe_status st = check_stride("expert_product", K, ldx)) return st;
  if (S == 0) return ok();
  if (!W_dev || !Y_dev || (x_rows > 0 && !X_dev)) return fail(BITSMOE_ERR_ARG, "expert_product: null pointer");
  unsigned grid;
  if (!grid_of(a, 64, (N + 63) / 64, &grid))
    return fail(BITSMOE_ERR_SHAPE, "expert_product: too many slots and outputs for one call");
  auto* fn = glu ? expert_simple_kernel<kForward, false, true> : expert_simple_kernel<kForward, false, false>;
  fn<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("expert_simple_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_expert_product_grad(const void* W_dev, bitsmoe_dtype t, int64_t E, int64_t N,
                                                      int64_t K, const void* dY_dev, int64_t lddy,
                                                      const int32_t* offsets_dev, int64_t S, void* dX_dev,
                                                      bitsmoe_dtype xt, int64_t ldx, void* stream) {
  const ExpertArgs a{static_cast<const uint16_t*>(W_dev), clip(E), N, K, nullptr, nullptr, nullptr, S, 0,
                     static_cast<const uint16_t*>(dY_dev), lddy, offsets_dev, nullptr, S, dX_dev, ldx,
                     xt == BITSMOE_F32};
  if (bitsmoe_status st = check("expert_product_grad", a, t, xt, K)) return st;
  if (N % 8 != 0) return fail(BITSMOE_ERR_SHAPE, "expert_product_grad: needs N % 8 == 0");
  if (bitsmoe_status st = check_stride("expert_product_grad", N, lddy)) return st;
  if (S == 0) return ok();
  if (!W_dev || !dY_dev || !dX_dev) return fail(BITSMOE_ERR_ARG, "expert_product_grad: null pointer");
  unsigned grid;
  if (!grid_of(a, 64, (K + 63) / 64, &grid))
    return fail(BITSMOE_ERR_SHAPE, "expert_product_grad: too many slots and columns for one call");
  expert_simple_kernel<kTokens, false, false><<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("expert_simple_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_expert_weight_grad(const void* dY_dev, bitsmoe_dtype t, int64_t lddy, int64_t E,
                                                     int64_t N, int64_t K, const void* X_dev, int64_t x_rows,
                                                     int64_t ldx, const int32_t* offsets_dev, const int32_t* rows_dev,
                                                     int64_t S, void* dW_dev, bitsmoe_dtype wt, void* stream) {
  const ExpertArgs a{nullptr, clip(E), N, K, static_cast<const uint16_t*>(X_dev), nullptr, nullptr, x_rows, ldx,
                     static_cast<const uint16_t*>(dY_dev), lddy, offsets_dev, rows_dev, S, dW_dev, K,
                     wt == BITSMOE_F32};
  if (bitsmoe_status st = check("expert_weight_grad", a, t, wt, K)) return st;
  if (N % 8 != 0) return fail(BITSMOE_ERR_SHAPE, "expert_weight_grad: needs N % 8 == 0");
  if (bitsmoe_status st = check_stride("expert_weight_grad", N, lddy)) return st;
  if (bitsmoe_status st = check_stride("expert_weight_grad", K, ldx)) return st;
  if (!dW_dev || (S > 0 && (!dY_dev || (x_rows > 0 && !X_dev))))
    return fail(BITSMOE_ERR_ARG, "expert_weight_grad: null pointer");
  return weight_grad("expert_weight_grad", a, static_cast<hipStream_t>(stream));
}

extern "C" bitsmoe_status bitsmoe_expert_weight_grad_q(const void* dY_dev, bitsmoe_dtype t, int64_t lddy, int64_t E,
                                                       int64_t N, int64_t K, const uint8_t* xcodes_dev,
                                                       const uint8_t* xscales_dev, int64_t x_rows,
                                                       const int32_t* offsets_dev, const int32_t* rows_dev, int64_t S,
                                                       void* dW_dev, bitsmoe_dtype wt, void* stream) {
  const ExpertArgs a{nullptr, clip(E), N, K, nullptr, xcodes_dev, xscales_dev, x_rows, K,
                     static_cast<const uint16_t*>(dY_dev), lddy, offsets_dev, rows_dev, S, dW_dev, K,
                     wt == BITSMOE_F32};
  if (bitsmoe_status st = check("expert_weight_grad_q", a, t, wt, K)) return st;
  if (N % 8 != 0 || K % kMx8Block != 0)
    return fail(BITSMOE_ERR_SHAPE, "expert_weight_grad_q: needs N % 8 == 0 and K % 32 == 0");
  if (bitsmoe_status st = check_stride("expert_weight_grad_q", N, lddy)) return st;
  if (!dW_dev || (S > 0 && (!dY_dev || (x_rows > 0 && (!xcodes_dev || !xscales_dev)))))
    return fail(BITSMOE_ERR_ARG, "expert_weight_grad_q: null pointer");
  return weight_grad("expert_weight_grad_q", a, static_cast<hipStream_t>(stream));
}
