// Root-mean-square norm of rows with the residual's addition, and its gradient.
//
//     v = round(x + r),  inv = 1 / sqrt(mean(v^2) + eps),  y = v inv w,
//     g = dy w,  dx = inv (g - v^ mean(g v^)) + dsum,  dw = sum_t dy v^,  v^ = v inv.
//
// v is rounded to the rows' type before the norm is taken: that is what the next
// block adds to and what the gradient reads, so the gradient is that of the
// values used.  A row stays in registers between its reading and its writing, so
// both directions are bound by memory.  8192 x 7168 bf16 with the residual: the norm with its
// MX8 form 97 us (two rows read; sum, y and 1 byte an entry written: 531 MB at 5.4 TB/s), the
// gradient 119 (three rows read, one written: 470 MB at 3.9) and its join 5; one row of 2048 3.9.
#include <cstdint>
#include <string>

#include "internal.hpp"
#include "mx8.hpp"
#include "rows.hpp"

namespace bitsmoe {
namespace {

constexpr int kThreads = 256;

struct NormArgs {
  const void* x;
  const void* r;  // or null
  const void* w;
  int64_t T, ldx, ldr;
  int pieces;  // of eight entries in a row
  float eps, d;
  void* sum;   // v, where r is given
  void* y;     // or null
  uint2* codes;  // MX8 of y, or null
  uint8_t* scales;
  float* inv;
};

// Sum over the L lanes or threads that share a row (64: a wave; else the workgroup).
template <int L>
__device__ __forceinline__ float row_sum(float v, float* part) {
  v = wave_sum(v);
  if constexpr (L > 64) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[wave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < L / 64; ++i) v += part[i];
    __syncthreads();
  }
  return v;
}

// A row on L threads, PER pieces each: a wave where that is enough (1003 x 2048 fp32:
// 6.2 us), as sums within it need no barrier; else a workgroup.
template <bool XB, bool WB, int L, int PER>
__global__ __launch_bounds__(L > kThreads ? L : kThreads) void norm_kernel(NormArgs a) {
  constexpr int kRows = L == 64 ? kThreads / 64 : 1;
  __shared__ float part[L / 64];
  const int t = L == 64 ? threadIdx.x & 63 : threadIdx.x;
  for (int64_t row = int64_t(blockIdx.x) * kRows + (L == 64 ? threadIdx.x >> 6 : 0); row < a.T;
       row += int64_t(gridDim.x) * kRows) {
    Eight<XB> v[PER];
    const char* x = static_cast<const char*>(a.x) + row * a.ldx * Eight<XB>::kBytes;
    const char* r = static_cast<const char*>(a.r) + row * a.ldr * Eight<XB>::kBytes;
    const int64_t first = row * a.pieces;  // piece of the dense rows
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = i * L + t;
      if (c < a.pieces) {
        v[i].load(x, c);
        if (a.r) {
          Eight<XB> b;
          b.load(r, c);
#pragma unroll
          for (int q = 0; q < 8; ++q) v[i].v[q] += b.v[q];
          v[i].round();
          v[i].store(a.sum, first + c);
        }
      } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[i].v[q] = 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int q = 0; q < 8; ++q) ss = fmaf(v[i].v[q], v[i].v[q], ss);
    ss = row_sum<L>(ss, part);
    float inv = 1.0f / sqrtf(ss / a.d + a.eps);
    if (ss == __builtin_inff()) {  // squares past fp32: of the row by 2^-80 (what that loses is below 2^-100 of the sum)
      ss = 0.0f;
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const float s = v[i].v[q] * 0x1p-80f;
          ss = fmaf(s, s, ss);
        }
      ss = row_sum<L>(ss, part);
      inv = 0x1p-80f / sqrtf(ss / a.d);
    }
    if (t == 0) a.inv[row] = inv;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = i * L + t;
      if (c >= a.pieces) continue;
      Eight<WB> w;
      w.load(a.w, c);
#pragma unroll
      for (int q = 0; q < 8; ++q) v[i].v[q] = v[i].v[q] * inv * w.v[q];
      if (a.y) v[i].store(a.y, first + c);
      if (a.codes) {  // (pieces is a multiple of four)
        uint32_t s;
        a.codes[first + c] = mx8_codes(v[i].v, &s);
        if ((t & 3) == 0) a.scales[(first + c) / 4] = static_cast<uint8_t>(s);
      }
    }
  }
}

struct NormGradArgs {
  const void* v;
  const void* w;
  const float* inv;
  const void* dy;
  const void* dsum;  // or null
  const uint8_t* valid;  // of the rows, or null: all are
  int64_t T, ldv, lddy, ldds;
  int pieces;
  float d;
  void* dx;
  float* dw;    // [d], or null
  float* part;  // [gridDim.x][d]; where gridDim.x is 1, dw itself
};

// A row on L threads as above; each workgroup takes every gridDim.x-th (group of)
// row and keeps its columns' sums of dw in registers, so that dy and v are read once for
// both gradients, in an order that does not change.  The next row is on its way while this one is summed, as a
// workgroup's rows come one after another (8192 x 7168 bf16, forward and back: 290 to 245 us by that, one barrier a row
// and the join's loads).
template <bool XB, bool WB, int L, int PER>
__global__ __launch_bounds__(L > kThreads ? L : kThreads) void norm_grad_kernel(NormGradArgs a) {
  constexpr int kRows = L == 64 ? kThreads / 64 : 1;
  __shared__ float part[2][L / 64];
  const int t = L == 64 ? threadIdx.x & 63 : threadIdx.x;
  float dw[PER][8];
#pragma unroll
  for (int i = 0; i < PER; ++i)
#pragma unroll
    for (int q = 0; q < 8; ++q) dw[i][q] = 0.0f;
  struct Row {
    RawEight<XB> v[PER], g[PER], s[PER];
    float inv;
    bool counts;
  };
  auto load = [&](Row& r, int64_t row) {
    const char* vp = static_cast<const char*>(a.v) + row * a.ldv * Eight<XB>::kBytes;
    const char* gp = static_cast<const char*>(a.dy) + row * a.lddy * Eight<XB>::kBytes;
    const char* sp = static_cast<const char*>(a.dsum) + row * a.ldds * Eight<XB>::kBytes;
    const int pieces = a.valid && !a.valid[row] ? 0 : a.pieces;  // (nothing of a row that is not is read but dsum)
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = i * L + t;
      r.s[i].clear();
      if (a.dsum && c < a.pieces) r.s[i].load(sp, c);
      if (c < pieces) {
        r.v[i].load(vp, c);
        r.g[i].load(gp, c);
      } else {
        r.v[i].clear();
        r.g[i].clear();
      }
    }
    r.counts = pieces != 0;
    r.inv = r.counts ? a.inv[row] : 0.0f;
  };
  constexpr bool kAhead = L < 1024;  // (of the longest rows registers hold but one)
  const int64_t step = int64_t(gridDim.x) * kRows;
  int64_t row = int64_t(blockIdx.x) * kRows + (L == 64 ? threadIdx.x >> 6 : 0);
  Row cur, next;
  if (kAhead && row < a.T) load(cur, row);
  for (int turn = 0; row < a.T; row += step, turn ^= 1) {
    if constexpr (kAhead) {
      if (row + step < a.T) load(next, row + step);
    } else {
      load(cur, row);
    }
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = i * L + t;
      if (c >= a.pieces) continue;
      Eight<WB> w;
      w.load(a.w, c);
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float n = cur.v[i].value(q) * cur.inv, g = cur.g[i].value(q);
        dw[i][q] = fmaf(g, n, dw[i][q]);
        dot = fmaf(g * w.v[q], n, dot);
      }
    }
    dot = wave_sum(dot);
    if constexpr (L > 64) {
      if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = dot;
      __syncthreads();  // (one a row: the row after next writes where this one's was)
      dot = 0.0f;
#pragma unroll
      for (int i = 0; i < L / 64; ++i) dot += part[turn][i];
    }
    dot /= a.d;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int c = i * L + t;
      if (c >= a.pieces) continue;
      Eight<WB> w;
      w.load(a.w, c);
      Eight<XB> dx;
      // (a row that does not count is zeros here, and zeros times weights that are no numbers are NaN; the select costs 1
      // to 3 % at 8192 x 7168 bf16, a branch in its place 17 %)
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float n = cur.v[i].value(q) * cur.inv, ds = cur.s[i].value(q);
        const float from_y = cur.inv * (cur.g[i].value(q) * w.v[q] - n * dot);
        dx.v[q] = cur.counts ? from_y + ds : ds;
      }
      dx.store(a.dx, row * a.pieces + c);
    }
    if constexpr (kAhead) cur = next;
  }
  if (!a.dw) return;
  if constexpr (L == 64) {  // the four waves' sums, in the order of the waves
    __shared__ float join[kRows - 1][PER * 8 * 64];
    const int wave = threadIdx.x >> 6;
    if (wave > 0)
#pragma unroll
      for (int i = 0; i < PER; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) join[wave - 1][(i * 8 + q) * 64 + t] = dw[i][q];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int i = 0; i < PER; ++i)
#pragma unroll
      for (int q = 0; q < 8; ++q)
#pragma unroll
        for (int k = 0; k < kRows - 1; ++k) dw[i][q] += join[k][(i * 8 + q) * 64 + t];
  }
  float* out = a.part + int64_t(blockIdx.x) * a.pieces * 8;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int c = i * L + t;
    if (c >= a.pieces) continue;
    Eight<false> s;
#pragma unroll
    for (int q = 0; q < 8; ++q) s.v[q] = dw[i][q];
    s.store(out, c);
  }
}

// dw from the workgroups' sums: 64 columns a workgroup of sixteen waves, which take
// every sixteenth row of them, eight loads at a time (512 rows of 7168: 15 MB, 5 us; there
// are too few columns to fill the card, so that what counts is one chain of loads).
constexpr int kJoin = 16;
__global__ __launch_bounds__(64 * kJoin) void norm_join_kernel(const float* part, int rows, int64_t d, float* dw) {
  __shared__ float sums[kJoin][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t c = int64_t(blockIdx.x) * 64 + lane;
  float s = 0.0f;
  if (c < d)
    for (int r = wave; r < rows; r += 8 * kJoin) {  // eight loads under way
      float v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = r + u * kJoin < rows ? part[(r + u * kJoin) * d + c] : 0.0f;
#pragma unroll
      for (int u = 0; u < 8; ++u) s += v[u];
    }
  sums[wave][lane] = s;
  __syncthreads();
  if (wave > 0 || c >= d) return;
#pragma unroll
  for (int i = 1; i < kJoin; ++i) s += sums[i][lane];
  dw[c] = s;
}

// f<L, PER>() for the fewest threads and pieces each that hold a row.
template <class F>
void by_length(int pieces, F f) {
  if (pieces <= 64)
    f.template operator()<64, 1>();
  else if (pieces <= 128)
    f.template operator()<64, 2>();
  else if (pieces <= 256)
    f.template operator()<64, 4>();
  else if (pieces <= 512)
    f.template operator()<256, 2>();
  else if (pieces <= 1024)
    f.template operator()<256, 4>();
  else if (pieces <= 2048)
    f.template operator()<512, 4>();
  else
    f.template operator()<1024, 4>();
}

constexpr int64_t kMostCols = 32768;

int rows_at_once(int64_t d) { return d <= 2048 ? kThreads / 64 : 1; }

// Workgroups of the gradient: enough to fill the card, few enough that their sums of dw are little beside the rows.
int grad_groups(int64_t T, int64_t d) {
  const int64_t n = (T + rows_at_once(d) - 1) / rows_at_once(d), most = 2 * device_cus();
  return static_cast<int>(n < most ? n : most);
}

bitsmoe_status check(const char* who, bitsmoe_dtype xt, bitsmoe_dtype wt, int64_t T, int64_t d) {
  if (T < 0 || d <= 0) return fail(BITSMOE_ERR_ARG, std::string(who) + ": non-positive size");
  if ((xt != BITSMOE_F32 && xt != BITSMOE_BF16) || (wt != BITSMOE_F32 && wt != BITSMOE_BF16))
    return fail(BITSMOE_ERR_DTYPE, std::string(who) + ": rows and weights must be fp32 or bf16");
  if (d % 8 != 0 || d > kMostCols || T > (int64_t(1) << 40) / d)
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": needs d % 8 == 0, d <= 32768 and T d <= 2^40");
  return BITSMOE_OK;
}

bitsmoe_status check_stride(const char* who, bitsmoe_dtype t, int64_t d, int64_t ld) {
  if (ld < d || ld > (int64_t(1) << 32) || ld * (t == BITSMOE_BF16 ? 2 : 4) % 16 != 0)
    return fail(BITSMOE_ERR_SHAPE,
                std::string(who) + ": rows must not overlap, and lie a multiple of 16 bytes apart");
  return BITSMOE_OK;
}

template <bool XB, bool WB>
void launch(const NormArgs& a, hipStream_t s) {
  by_length(a.pieces, [&]<int L, int PER>() {
    const int64_t n = L == 64 ? (a.T + kThreads / 64 - 1) / (kThreads / 64) : a.T;
    norm_kernel<XB, WB, L, PER>
        <<<static_cast<unsigned>(n < (1 << 20) ? n : (1 << 20)), L > kThreads ? L : kThreads, 0, s>>>(a);
  });
}

template <bool XB, bool WB>
void launch_grad(const NormGradArgs& a, int groups, hipStream_t s) {
  by_length(a.pieces, [&]<int L, int PER>() {
    norm_grad_kernel<XB, WB, L, PER><<<groups, L > kThreads ? L : kThreads, 0, s>>>(a);
  });
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" bitsmoe_status bitsmoe_rms_norm(const void* X_dev, bitsmoe_dtype xt, int64_t ldx, const void* R_dev,
                                           int64_t ldr, const void* W_dev, bitsmoe_dtype wt, int64_t T, int64_t d,
                                           double eps, void* Sum_dev, void* Y_dev, uint8_t* codes_dev,
                                           uint8_t* scales_dev, float* inv_dev, void* stream) {
  if (bitsmoe_status st = check("rms_norm", xt, wt, T, d)) return st;
  if (!(static_cast<float>(eps) > 0.0f && eps < 1e30))
    return fail(BITSMOE_ERR_ARG, "rms_norm: eps must be positive, and in fp32 too");
  if (codes_dev && d % kMx8Block != 0) return fail(BITSMOE_ERR_SHAPE, "rms_norm: MX8 needs d % 32 == 0");
  if (bitsmoe_status st = check_stride("rms_norm", xt, d, ldx)) return st;
  if (R_dev)
    if (bitsmoe_status st = check_stride("rms_norm", xt, d, ldr)) return st;
  if (T == 0) return ok();
  if (!X_dev || !W_dev || !inv_dev || (R_dev && !Sum_dev) || (!codes_dev != !scales_dev))
    return fail(BITSMOE_ERR_ARG, "rms_norm: null pointer");
  if (!aligned16({X_dev, R_dev, W_dev, Sum_dev, Y_dev, codes_dev, scales_dev, inv_dev}))
    return fail(BITSMOE_ERR_ARG, "rms_norm: device pointers must be 16-byte aligned");
  const NormArgs a{X_dev, R_dev, W_dev, T, ldx, ldr, static_cast<int>(d / 8), static_cast<float>(eps),
                   static_cast<float>(d), Sum_dev, Y_dev, reinterpret_cast<uint2*>(codes_dev), scales_dev, inv_dev};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const bool xb = xt == BITSMOE_BF16, wb = wt == BITSMOE_BF16;
  xb ? (wb ? launch<true, true>(a, s) : launch<true, false>(a, s))
     : (wb ? launch<false, true>(a, s) : launch<false, false>(a, s));
  BITSMOE_LAUNCH_CHECK("norm_kernel");
  return ok();
}

extern "C" int64_t bitsmoe_rms_norm_grad_workspace(int64_t T, int64_t d) {
  if (T <= 0 || d <= 0 || d > kMostCols) return 0;
  const int groups = grad_groups(T, d);
  return groups > 1 ? groups * d * 4 : 0;
}

extern "C" bitsmoe_status bitsmoe_rms_norm_grad(const void* Sum_dev, bitsmoe_dtype xt, int64_t ldsum,
                                                const void* W_dev, bitsmoe_dtype wt, const float* inv_dev,
                                                const void* dY_dev, int64_t lddy, const void* dSum_dev,
                                                int64_t lddsum, const uint8_t* valid_dev, int64_t T, int64_t d,
                                                void* dX_dev, float* dW_dev, void* work_dev, int64_t work_bytes, void* stream) {
  if (bitsmoe_status st = check("rms_norm_grad", xt, wt, T, d)) return st;
  if (bitsmoe_status st = check_stride("rms_norm_grad", xt, d, ldsum)) return st;
  if (bitsmoe_status st = check_stride("rms_norm_grad", xt, d, lddy)) return st;
  if (dSum_dev)
    if (bitsmoe_status st = check_stride("rms_norm_grad", xt, d, lddsum)) return st;
  if (!aligned16({Sum_dev, W_dev, inv_dev, dY_dev, dSum_dev, dX_dev, dW_dev, work_dev}))
    return fail(BITSMOE_ERR_ARG, "rms_norm_grad: device pointers must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T == 0) {  // sums of no rows
    if (dW_dev) {
      norm_join_kernel<<<static_cast<unsigned>((d + 63) / 64), 64 * kJoin, 0, s>>>(nullptr, 0, d, dW_dev);
      BITSMOE_LAUNCH_CHECK("norm_join_kernel");
    }
    return ok();
  }
  if (!Sum_dev || !W_dev || !inv_dev || !dY_dev || !dX_dev)
    return fail(BITSMOE_ERR_ARG, "rms_norm_grad: null pointer");
  const int groups = grad_groups(T, d);
  if (dW_dev && groups > 1 && (!work_dev || work_bytes < groups * d * 4))
    return fail(BITSMOE_ERR_ARG, "rms_norm_grad: the workspace is missing or too small");
  const NormGradArgs a{Sum_dev, W_dev, inv_dev, dY_dev, dSum_dev, valid_dev, T, ldsum, lddy, lddsum, static_cast<int>(d / 8),
                       static_cast<float>(d), dX_dev, dW_dev, groups > 1 ? static_cast<float*>(work_dev) : dW_dev};
  const bool xb = xt == BITSMOE_BF16, wb = wt == BITSMOE_BF16;
  xb ? (wb ? launch_grad<true, true>(a, groups, s) : launch_grad<true, false>(a, groups, s))
     : (wb ? launch_grad<false, true>(a, groups, s) : launch_grad<false, false>(a, groups, s));
  BITSMOE_LAUNCH_CHECK("norm_grad_kernel");
  if (dW_dev && groups > 1) {
    norm_join_kernel<<<static_cast<unsigned>((d + 63) / 64), 64 * kJoin, 0, s>>>(static_cast<const float*>(work_dev),
                                                                                 groups, d, dW_dev);
    BITSMOE_LAUNCH_CHECK("norm_join_kernel");
  }
  return ok();
}
