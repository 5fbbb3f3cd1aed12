// Rows to MX8 and back, and silu(gate) * up with its inputs kept in MX8.
//
//     h = silu(g) u, [g; u] also to MX8                         (glu_mx8)
//     dg = dh u' s (1 + g' (1 - s)),  du = dh g' s,  h' = g' s u',
//     s = 1 / (1 + exp(-g')), of the values g', u' kept         (glu_mx8_grad)
//
// All are bound by memory: eight entries a lane (of g and of u), four lanes a
// block, whose maximum takes two lane exchanges.  8192 x 7168 from bf16 to MX8 30 us (6.0 TB/s), 32768 x 2048 33 us, from
// MX8 to bf16 29 us (6.2 TB/s; what was written just before is partly in the last-level cache).  4096 rows of 2 x
// 14336, bf16: 93 us (473 MB at 5.1 TB/s), the gradient with h again 104 (592 MB at 5.7); 184
// rows of 2 x 768 fp32: 3 us each way.
//
// The gradient takes g' and u' as kept, so that it is that of the function at values
// that are off by 2^-4 of themselves at most, or by 2^-10 of their block's scale; h' again costs one more store here, where keeping h
// would cost 2 bytes an entry for the whole step.
#include <cstdint>
#include <string>

#include "internal.hpp"
#include "mx8.hpp"
#include "rows.hpp"

namespace bitsmoe {
namespace {

constexpr int kThreads = 256;

template <bool BF16>
__global__ __launch_bounds__(kThreads) void mx8_quantize_kernel(const void* x, int64_t rows, int pieces, int64_t ld,
                                                                uint2* codes, uint8_t* scales) {
  const int64_t n = rows * pieces;  // pieces of eight entries (four to a block: lanes end together)
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    const int64_t r = i / pieces;
    Eight<BF16> v;
    v.load(static_cast<const char*>(x) + r * ld * v.kBytes, i - r * pieces);
    uint32_t s;
    codes[i] = mx8_codes(v.v, &s);
    if ((threadIdx.x & 3) == 0) scales[i / 4] = static_cast<uint8_t>(s);
  }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void mx8_dequantize_kernel(const uint2* codes, const uint8_t* scales, int64_t n,
                                                                  void* y) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    Eight<BF16> v;
    mx8_values(codes[i], scales[i / 4], v.v);
    v.store(y, i);
  }
}

// 1 / (1 + exp(-v)) by the hardware's exponential and reciprocal, within 2^-21 of itself
// where it is above 2^-126.
__device__ __forceinline__ float sigmoid(float v) {
  return __builtin_amdgcn_rcpf(1.0f + exp_hw(__builtin_amdgcn_fmed3f(-v, -150.0f, 88.0f)));
}

struct GluArgs {
  const void* gu;  // [S] rows of 2 N entries, ld apart
  int64_t ld;
  uint2* codes;  // [S][2 N]
  uint8_t* scales;
  uint16_t* h;     // [S][N]
  const void* dh;  // [S] rows of N entries, ld apart
  uint16_t* dgu;   // [S][2 N]
  int64_t n;       // S pieces
  int pieces;      // N / 8
};

template <bool BF16>
__global__ __launch_bounds__(kThreads) void glu_mx8_kernel(GluArgs a) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < a.n; i += int64_t(gridDim.x) * kThreads) {
    const int64_t r = i / a.pieces;
    const int c = static_cast<int>(i - r * a.pieces);
    Eight<BF16> g, u;
    const char* row = static_cast<const char*>(a.gu) + r * a.ld * g.kBytes;
    g.load(row, c);
    u.load(row, a.pieces + c);
    const int64_t at = r * (2 * int64_t(a.pieces)) + c;
    uint32_t s;
    a.codes[at] = mx8_codes(g.v, &s);
    if ((threadIdx.x & 3) == 0) a.scales[at / 4] = static_cast<uint8_t>(s);
    a.codes[at + a.pieces] = mx8_codes(u.v, &s);
    if ((threadIdx.x & 3) == 0) a.scales[(at + a.pieces) / 4] = static_cast<uint8_t>(s);
    Eight<true> h;
#pragma unroll
    for (int q = 0; q < 8; ++q) h.v[q] = g.v[q] * sigmoid(g.v[q]) * u.v[q];
    h.store(a.h, i);
  }
}

template <bool BF16>
__global__ __launch_bounds__(kThreads) void glu_mx8_grad_kernel(GluArgs a) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < a.n; i += int64_t(gridDim.x) * kThreads) {
    const int64_t r = i / a.pieces;
    const int c = static_cast<int>(i - r * a.pieces);
    Eight<BF16> d;
    d.load(static_cast<const char*>(a.dh) + r * a.ld * d.kBytes, c);
    const int64_t at = r * (2 * int64_t(a.pieces)) + c;
    Eight<true> g, u, h;
    mx8_values(a.codes[at], a.scales[at / 4], g.v);
    mx8_values(a.codes[at + a.pieces], a.scales[(at + a.pieces) / 4], u.v);
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float s = sigmoid(g.v[q]), gs = g.v[q] * s;
      h.v[q] = gs * u.v[q];
      u.v[q] *= d.v[q] * (s + gs * (1.0f - s));  // of the gate
      g.v[q] = d.v[q] * gs;                      // of the up value
    }
    u.store(a.dgu, at);
    g.store(a.dgu, at + a.pieces);
    if (a.h) h.store(a.h, i);
  }
}

unsigned grid_for(int64_t n) {
  const int64_t b = (n + kThreads - 1) / kThreads;
  return static_cast<unsigned>(b < (1 << 20) ? b : (1 << 20));
}

bitsmoe_status check(const char* who, bitsmoe_dtype t, int64_t rows, int64_t cols) {
  if (rows < 0 || cols <= 0) return fail(BITSMOE_ERR_ARG, std::string(who) + ": non-positive size");
  if (t != BITSMOE_F32 && t != BITSMOE_BF16)
    return fail(BITSMOE_ERR_DTYPE, std::string(who) + ": rows must be fp32 or bf16");
  if (cols % kMx8Block != 0 || cols > (int64_t(1) << 30) || rows > (int64_t(1) << 40) / cols)
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": needs blocks of 32 columns, at most 2^30, and 2^40 entries");
  return BITSMOE_OK;
}

bitsmoe_status check_rows(const char* who, bitsmoe_dtype t, int64_t cols, int64_t ld) {
  if (ld < cols || ld > (int64_t(1) << 40) || ld * (t == BITSMOE_BF16 ? 2 : 4) % 16 != 0)
    return fail(BITSMOE_ERR_SHAPE,
                std::string(who) + ": rows must not overlap, and lie a multiple of 16 bytes apart");
  return BITSMOE_OK;
}

bitsmoe_status check_pointers(const char* who, std::initializer_list<const void*> needed,
                              std::initializer_list<const void*> optional = {}) {
  for (const void* p : needed)
    if (!p) return fail(BITSMOE_ERR_ARG, std::string(who) + ": null pointer");
  if (!aligned16(needed) || !aligned16(optional))
    return fail(BITSMOE_ERR_ARG, std::string(who) + ": device pointers must be 16-byte aligned");
  return BITSMOE_OK;
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" bitsmoe_status bitsmoe_mx8_quantize(const void* X_dev, bitsmoe_dtype xt, int64_t rows, int64_t cols,
                                               int64_t ld, uint8_t* codes_dev, uint8_t* scales_dev, void* stream) {
  if (bitsmoe_status st = check("mx8_quantize", xt, rows, cols)) return st;
  if (bitsmoe_status st = check_rows("mx8_quantize", xt, cols, ld)) return st;
  if (rows == 0) return ok();
  if (bitsmoe_status st = check_pointers("mx8_quantize", {X_dev, codes_dev, scales_dev})) return st;
  auto* fn = xt == BITSMOE_BF16 ? mx8_quantize_kernel<true> : mx8_quantize_kernel<false>;
  fn<<<grid_for(rows * (cols / 8)), kThreads, 0, static_cast<hipStream_t>(stream)>>>(
      X_dev, rows, static_cast<int>(cols / 8), ld, reinterpret_cast<uint2*>(codes_dev), scales_dev);
  BITSMOE_LAUNCH_CHECK("mx8_quantize_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_mx8_dequantize(const uint8_t* codes_dev, const uint8_t* scales_dev, int64_t rows,
                                                 int64_t cols, void* Y_dev, bitsmoe_dtype yt, void* stream) {
  if (bitsmoe_status st = check("mx8_dequantize", yt, rows, cols)) return st;
  if (rows == 0) return ok();
  if (bitsmoe_status st = check_pointers("mx8_dequantize", {codes_dev, scales_dev, Y_dev})) return st;
  const int64_t n = rows * (cols / 8);
  auto* fn = yt == BITSMOE_BF16 ? mx8_dequantize_kernel<true> : mx8_dequantize_kernel<false>;
  fn<<<grid_for(n), kThreads, 0, static_cast<hipStream_t>(stream)>>>(reinterpret_cast<const uint2*>(codes_dev),
                                                                     scales_dev, n, Y_dev);
  BITSMOE_LAUNCH_CHECK("mx8_dequantize_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_glu_mx8(const void* GU_dev, bitsmoe_dtype gut, int64_t S, int64_t N, int64_t ld,
                                          void* H_dev, uint8_t* codes_dev, uint8_t* scales_dev, void* stream) {
  if (N > (int64_t(1) << 29)) return fail(BITSMOE_ERR_SHAPE, "glu_mx8: needs N <= 2^29");
  if (bitsmoe_status st = check("glu_mx8", gut, S, N)) return st;
  if (bitsmoe_status st = check_rows("glu_mx8", gut, 2 * N, ld)) return st;
  if (S == 0) return ok();
  if (bitsmoe_status st = check_pointers("glu_mx8", {GU_dev, H_dev, codes_dev, scales_dev})) return st;
  const int pieces = static_cast<int>(N / 8);
  GluArgs a{GU_dev, ld, reinterpret_cast<uint2*>(codes_dev), scales_dev, static_cast<uint16_t*>(H_dev),
            nullptr, nullptr, S * pieces, pieces};
  auto* fn = gut == BITSMOE_BF16 ? glu_mx8_kernel<true> : glu_mx8_kernel<false>;
  fn<<<grid_for(a.n), kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("glu_mx8_kernel");
  return ok();
}

extern "C" bitsmoe_status bitsmoe_glu_mx8_grad(const uint8_t* codes_dev, const uint8_t* scales_dev, const void* dH_dev,
                                               bitsmoe_dtype dht, int64_t S, int64_t N, int64_t lddh, void* dGU_dev,
                                               void* H_dev, void* stream) {
  if (N > (int64_t(1) << 29)) return fail(BITSMOE_ERR_SHAPE, "glu_mx8_grad: needs N <= 2^29");
  if (bitsmoe_status st = check("glu_mx8_grad", dht, S, N)) return st;
  if (bitsmoe_status st = check_rows("glu_mx8_grad", dht, N, lddh)) return st;
  if (S == 0) return ok();
  if (bitsmoe_status st = check_pointers("glu_mx8_grad", {codes_dev, scales_dev, dH_dev, dGU_dev}, {H_dev})) return st;
  const int pieces = static_cast<int>(N / 8);
  GluArgs a{nullptr, lddh, reinterpret_cast<uint2*>(const_cast<uint8_t*>(codes_dev)),
            const_cast<uint8_t*>(scales_dev), static_cast<uint16_t*>(H_dev), dH_dev,
            static_cast<uint16_t*>(dGU_dev), S * pieces, pieces};
  auto* fn = dht == BITSMOE_BF16 ? glu_mx8_grad_kernel<true> : glu_mx8_grad_kernel<false>;
  fn<<<grid_for(a.n), kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("glu_mx8_grad_kernel");
  return ok();
}
