// Products with expert weights held in MX4.
//
//     y_s = W_e(s) x_row(s)            (mx4_product: bf16 tokens; _q: MX4 tokens)
//     y_s = silu(g) u, [g; u] = W_e(s) x_row(s)        (the same with glu)
//     dx_s = W_e(s)^T dy_s             (mx4_product_grad)
//
// for S slots in expert order, expert e's being offsets[e] .. offsets[e+1].
#include <atomic>
#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include "internal.hpp"
#include "slots.hpp"

namespace bitsmoe {
namespace {

constexpr int kThreads = 256;

struct MulArgs {
  const uint8_t* codes;   // [E][N or 2N][K/2]
  const uint8_t* scales;  // [E][..][K/32]
  int E;
  int64_t N, K;
  const uint16_t* x;       // bf16 rows (product: tokens; grad: dy)
  const uint8_t* xcodes;   // or MX4 rows
  const uint8_t* xscales;
  int64_t x_rows, ldx;
  const int32_t* offsets;
  const int32_t* rows;
  int64_t S;
  void* y;
  int64_t ldy;
  int yf32;
};

// 16 outputs x 16 slots a workgroup.  The four waves share out K in segments
// of 128: lane l holds 32 codes of row l % 16 (block l / 16 of the segment),
// which one load fetches with their scale, and the same entries of slot l % 16.
// For the fewest slots: bound by launch and one chain of loads (four segments in
// flight a wave), so the sum is split and the workgroups are small and many.  One
// token's 8 experts, 2 x 768 x 2048 with glu (13 MB): 8.2 us.
template <bool MX, bool GLU>
__global__ __launch_bounds__(kThreads) void mx4_rows_kernel(MulArgs a) {
  constexpr int H = GLU ? 2 : 1;
  __shared__ f32x4 part[kThreads / 64][H][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((a.N + 15) / 16), 16, &t)) return;
  const int64_t n0 = static_cast<int64_t>(t.col) * 16;
  f32x4 acc[H];
#pragma unroll
  for (int h = 0; h < H; ++h) acc[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bool have = false;  // the row of this lane's slot exists
  if (t.e < a.E) {
    const int64_t n = min(n0 + r, a.N - 1);
    const int64_t slot = t.lo + r;
    const int64_t row = slot < t.hi ? (a.rows ? static_cast<int64_t>(a.rows[slot]) : slot) : -1;
    have = row >= 0 && row < a.x_rows;
    const int64_t kb = a.K / 32;
    const int64_t wrow = static_cast<int64_t>(t.e) * (a.N * H) + n;
    for (int64_t seg = wave; seg * 4 < kb; seg += kThreads / 64) {
      const int64_t b = seg * 4 + q;  // this lane's block
      uint4 xc = make_uint4(0, 0, 0, 0);
      uint4 xv[4] = {xc, xc, xc, xc};
      int xs = 127;
      if (b < kb && have) {
        if constexpr (MX) {
          xc = *reinterpret_cast<const uint4*>(a.xcodes + (row * kb + b) * 16);
          xs = a.xscales[row * kb + b];
        } else {
          const uint4* p = reinterpret_cast<const uint4*>(a.x + row * a.ldx + b * 32);
#pragma unroll
          for (int i = 0; i < 4; ++i) xv[i] = p[i];
        }
      }
#pragma unroll
      for (int h = 0; h < H; ++h) {
        uint4 c = make_uint4(0, 0, 0, 0);
        int s = 127;
        if (b < kb) {
          const int64_t at = (wrow + h * a.N) * kb + b;
          c = *reinterpret_cast<const uint4*>(a.codes + at * 16);
          s = a.scales[at];
        }
        if constexpr (MX) {
          const i32x8 A = {(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
          const i32x8 B = {(int)xc.x, (int)xc.y, (int)xc.z, (int)xc.w, 0, 0, 0, 0};
          acc[h] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc[h], 4, 4, 0, s, 0, xs);
        } else {
          const float scale = mx4_scale(s);
          const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(mx4_bf16(w[i], scale), __builtin_bit_cast(bf16x8, xv[i]),
                                                             acc[h], 0, 0, 0);
        }
      }
    }
  }
#pragma unroll
  for (int h = 0; h < H; ++h) part[wave][h][lane] = acc[h];
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) acc[h] += part[w][h][lane];
  if constexpr (GLU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[0][i] = silu(acc[0][i]) * acc[1][i];
  }
  if (!have) acc[0] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (zeros times a lost block of weights are NaN)
  const int64_t slot = t.lo + r, n = n0 + 4 * q;  // (a lane holds four outputs of one slot)
  const bool wide = a.ldy % 4 == 0;
  if (slot < t.hi && n < a.N) store4(a, slot, n, a.N, wide, acc[0]);
}

// 16 TB slots x 256 weight rows a workgroup, 64 rows a wave: for a few slots an
// expert and many experts, where reading the weights is all.  The slots' tokens
// go through LDS 1024 entries of K at a time; the weights come straight into
// registers, two steps of 128 entries (four rows' tiles, 64 bytes of a row) ahead:
// four steps ahead leave room for two waves a SIMD instead of four, and take 30 us
// where these take 23.
// 16-byte chunk c of a slot lies at c ^ (slot mod 16): the sixteen slots of a
// fragment read in different banks.  Bound by the weights' bytes: 512 slots over
// 128 experts, 2048 x 768 (110 MB), take 22 us, 5.0 TB/s.
template <bool MX, bool GLU, int TB>
__global__ __launch_bounds__(kThreads, TB == 1 ? 4 : 3) void mx4_few_kernel(MulArgs a) {
  constexpr int R = 4, AHEAD = 2, KC = 1024, XB = MX ? KC / 2 : 2 * KC, XC = XB / 16, SL = 16 * TB;
  constexpr int NO = GLU ? 128 : 256;  // results of a slot
  __shared__ __align__(16) char xs[SL * XB];
  __shared__ uint8_t ss[MX ? SL * (KC / 32) : 1];
  __shared__ __align__(16) uint32_t sw[kThreads][KC / 128];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, q = lane >> 4;
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((a.N + NO - 1) / NO), SL, &t)) return;
  const int64_t n0 = static_cast<int64_t>(t.col) * NO;
  f32x4 acc[R][TB];
#pragma unroll
  for (int i = 0; i < R; ++i)
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  uint64_t there = 0;  // bit i: the row of slot i exists (a wave's mask: neither vector registers nor LDS to spare)
  if (t.e < a.E) {
    const int mine = t.lo + (lane & (SL - 1));
    const int row_of_mine = mine >= t.hi ? -1 : a.rows ? a.rows[mine] : mine;
    const int kb = static_cast<int>(a.K / 32);
    // row r of the wave's tile i (glu: gate and up in turn)
    auto row_of = [&](int i) {
      if constexpr (GLU)
        return static_cast<int64_t>(t.e) * 2 * a.N + min(n0 + wave * 32 + (i >> 1) * 16 + r, a.N - 1) + (i & 1) * a.N;
      else
        return static_cast<int64_t>(t.e) * a.N + min(n0 + wave * 64 + i * 16 + r, a.N - 1);
    };
    const uint8_t* pc[R];  // at this lane's block of 32 in the first step
#pragma unroll
    for (int i = 0; i < R; ++i) pc[i] = a.codes + (row_of(i) * kb + q) * 16;
    uint4 c[AHEAD][R];
    auto load = [&](int u, int step) {
      const bool in = 4 * step + q < kb;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        c[u][i] = make_uint4(0, 0, 0, 0);
        if (in) c[u][i] = *reinterpret_cast<const uint4*>(pc[i] + static_cast<int64_t>(step) * 64);
      }
    };
    // The scales of a row, 32 blocks at a time by one lane (row r of tile q), go through LDS: read byte by byte as
    // they are used, each would find its line still on its way.  Those past K are 0.
    const uint8_t* ps = a.scales + row_of(q) * kb;
    uint4 s[2];
    auto load_scales = [&](int at) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int left = kb - at - 16 * h;
        const uint8_t* p = ps + at + 16 * h;
        s[h] = make_uint4(0, 0, 0, 0);
        if (left >= 16) {
          __builtin_memcpy(&s[h], p, 16);
        } else if (left > 0 && kb >= 16) {  // the row's last sixteen, those before shifted out
          uint64_t v[2];
          __builtin_memcpy(v, p + left - 16, 16);
          const int out = 8 * (16 - left);
          v[0] = out < 64 ? (v[0] >> out) | ((v[1] << 1) << (63 - out)) : v[1] >> (out - 64);
          v[1] = out < 64 ? v[1] >> out : 0;
          __builtin_memcpy(&s[h], v, 16);
        } else if (left > 0) {
          uint32_t d[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            d[w] = 0;
#pragma unroll
            for (int v = 0; v < 4; ++v) d[w] |= static_cast<uint32_t>(4 * w + v < left ? p[4 * w + v] : 0) << (8 * v);
          }
          s[h] = make_uint4(d[0], d[1], d[2], d[3]);
        }
      }
    };
    const int steps = (kb + 3) / 4;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(u, u);
    load_scales(0);
    for (int k0 = 0; k0 < steps; k0 += KC / 128) {
      if (k0 > 0) __syncthreads();
      for (int i = tid; i < SL * XC; i += kThreads) {
        const int sl = i / XC, ch = i % XC;  // (powers of two)
        const int64_t slot = t.lo + sl;
        const int64_t row = slot < t.hi ? (a.rows ? static_cast<int64_t>(a.rows[slot]) : slot) : -1;
        const int at = (k0 * 128 + ch * (MX ? 32 : 8)) / 32;  // block of the chunk
        uint4 v = make_uint4(0, 0, 0, 0);
        int sc = 127;
        if (row >= 0 && row < a.x_rows && at < kb) {
          if constexpr (MX) {
            v = *reinterpret_cast<const uint4*>(a.xcodes + (row * kb + at) * 16);
            sc = a.xscales[row * kb + at];
          } else {
            v = *reinterpret_cast<const uint4*>(a.x + row * a.ldx + k0 * 128 + ch * 8);
          }
        }
        *reinterpret_cast<uint4*>(xs + sl * XB + ((ch ^ (sl & 15)) * 16)) = v;
        if constexpr (MX) ss[sl * (KC / 32) + ch] = static_cast<uint8_t>(sc);
      }
      if (k0 == 0) there = __ballot(row_of_mine >= 0 && row_of_mine < a.x_rows);
      *reinterpret_cast<uint4*>(&sw[tid][0]) = s[0];
      *reinterpret_cast<uint4*>(&sw[tid][4]) = s[1];
      __syncthreads();
      load_scales(k0 * 4 + KC / 32);
      const int end = min(steps - k0, KC / 128);
      for (int st0 = 0; st0 < end; st0 += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
          const int st = st0 + u;
          if (st >= end) break;
          uint4 w[R];
          int scale[R];
#pragma unroll
          for (int i = 0; i < R; ++i) {
            w[i] = c[u][i];
            scale[i] = (sw[wave * 64 + i * 16 + r][st] >> (8 * q)) & 255;
          }
          load(u, k0 + st + AHEAD);
          if constexpr (MX) {
#pragma unroll
            for (int b = 0; b < TB; ++b) {
              const int sl = 16 * b + r, ch = 4 * st + q;
              const uint4 v = *reinterpret_cast<const uint4*>(xs + sl * XB + ((ch ^ r) * 16));
              const i32x8 B = {(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
              const int sx = ss[sl * (KC / 32) + ch];
#pragma unroll
              for (int i = 0; i < R; ++i) {
                const i32x8 A = {(int)w[i].x, (int)w[i].y, (int)w[i].z, (int)w[i].w, 0, 0, 0, 0};
                acc[i][b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, acc[i][b], 4, 4, 0, scale[i], 0, sx);
              }
            }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              bf16x8 xv[TB];
#pragma unroll
              for (int b = 0; b < TB; ++b)
                xv[b] = *reinterpret_cast<const bf16x8*>(xs + (16 * b + r) * XB + (((16 * st + 4 * q + j) ^ r) * 16));
#pragma unroll
              for (int i = 0; i < R; ++i) {
                const uint32_t d = j == 0 ? w[i].x : j == 1 ? w[i].y : j == 2 ? w[i].z : w[i].w;
                const bf16x8 wv = mx4_bf16(d, mx4_scale(scale[i]));
#pragma unroll
                for (int b = 0; b < TB; ++b)
                  acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xv[b], acc[i][b], 0, 0, 0);
              }
            }
          }
        }
      }
    }
  }
  const bool wide = a.ldy % 4 == 0;
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int64_t slot = t.lo + 16 * b + r;
    if (slot >= t.hi) continue;
    const bool have = there >> (16 * b + r) & 1;
#pragma unroll
    for (int i = 0; i < (GLU ? R / 2 : R); ++i) {
      f32x4 v;
      if constexpr (GLU) {
        v = acc[2 * i][b];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = silu(v[u]) * acc[2 * i + 1][b][u];
      } else {
        v = acc[i][b];
      }
      if (!have) v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (zeros times a lost block of weights are NaN)
      const int64_t n = n0 + wave * (GLU ? 32 : 64) + i * 16 + 4 * q;
      if (n < a.N) store4(a, slot, n, a.N, wide, v);
    }
  }
}

// ---------------------------------------------------------------------------
// Large tiles: 128 slots x 256 outputs a workgroup of eight waves.
//
// Wave (wm, wn) of 2 x 4 owns 64 slots x 64 outputs as 32 x 32 accumulators,
// the weights on the matrix core's row side, so that a lane holds runs of four
// outputs of one slot.  With bf16 tokens a wave widens each fragment of codes in
// registers (exact; two conversions a matrix-core op) and uses it for its two
// blocks of slots; with MX4 tokens the scaled matrix-core form takes codes and
// scales as they lie.
//
// Direct global->LDS loads fill rings of stages: weights 256 entries of K at a
// time and tokens 64 (bf16) or 256 (MX4), so that a row of either is a whole
// cache line of 128 bytes; two loads in flight that share a line make the
// second wait for the first's data.  For the same reason scales, 1/32 of a
// byte an entry, come 512 entries at a time (16 bytes a row) where rows of
// scales are a multiple of that (AL: K % 512 == 0), else a byte a lane with
// each stage of weights.  A step that finds its stage read by every wave refills
// the ring at once.
//
// A workgroup stays on its compute unit and takes tile after tile; the loads run
// on into the next tile, so its first stages are there when the results of one
// have been stored.
//
// Bound by the matrix cores, whose clock gives way under load (about 1.3 PFLOP/s
// bf16 without a pause), and by the tiles that an expert's last slots do not fill.
// bf16, 32768 slots over 128 experts, 2 x 768 x 2048 with glu: 254 us, 0.81
// PFLOP/s (1.0 with what pads the tiles).  MX4, 32768 slots over 256 experts, 2048
// x 7168: 600 us, 1.6 PFLOP/s (2.4 padded) and 3.6 TB/s; half of its time
// goes with the weights' bytes, which every XCD's share reads once.
// ---------------------------------------------------------------------------
constexpr int kTileThreads = 512, kWaves = 8, kTM = 128, kTN = 256, kLds = 163840;

template <bool MX_, bool AL_>
struct Shape {
  static constexpr bool MX = MX_, AL = AL_;
  static constexpr int WK = 256, XK = MX ? 256 : 64;  // entries of K in a stage of weights, of tokens
  static constexpr int kXStage = kTM * 128, kWStage = kTN * 128;
  // scales: of a stage of weights, a word each; or of 512 entries, a byte each
  static constexpr int kWS = AL ? 0 : kTN * 8 * 4, kXS = AL || !MX ? 0 : kTM * 8 * 4;
  static constexpr int kChunk = AL ? (kTN + (MX ? kTM : 0)) * 16 : 0;
  static constexpr int NX = MX ? (AL ? 3 : 2) : (AL ? 5 : 4), NW = MX ? NX : 2;
  // LDS: the token ring, the weight ring (codes, then scales), two chunks of scales, rows of X of three tiles
  static constexpr int oW = NX * kXStage, kWRing = kWStage + kWS + kXS, oC = oW + NW * kWRing;
  static constexpr int oRows = oC + 2 * kChunk, kBytes = oRows + 3 * kTM * 4;
  static_assert(kBytes <= kLds);
  // direct loads of a wave for a stage
  static constexpr int LX = kXStage / 1024 / kWaves, LW = kWStage / 1024 / kWaves;
  static constexpr int LWS = kWS / 256 / kWaves, LXS = kXS / 256 / kWaves;
  static constexpr int kWLoads = LW + LWS + LXS;
  static constexpr int MB = 2, NB = 2;
  // stages of weights a tile has at least, so that the rings never reach past the next tile
  static constexpr int kLeast = MX ? (AL ? 4 : 2) : 2;
};

// What lanes past the end of a row read: zeros, and scales of 1.
__device__ const uint8_t kPad[32] __attribute__((aligned(16))) = {
    0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,
    127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127};

// Place of scale c of row r among the eight words of its row.
__device__ __forceinline__ int scale_slot(int r, int c) { return c ^ (2 * ((r >> 3) & 3)); }

// MX4 tokens: the operand fragments of 64 entries of K, a quarter of a stage,
// read while the quarter before is multiplied.
template <class H>
struct Frags {
  uint4 w[H::NB], x[H::MB];
  int ws[H::NB], xs[H::MB];
  // Quarter u of the stages at xst and wst; sc: this stage's scales of row 0 (AL).
  __device__ __forceinline__ void read(const char* xst, const char* wst, const char* sc, int u, int wrow, int xrow,
                                       int half) {
    const int c = 2 * u + half;  // this lane's block of 32
#pragma unroll
    for (int n = 0; n < H::NB; ++n) {
      const int r = wrow + 32 * n;
      w[n] = *reinterpret_cast<const uint4*>(wst + r * 128 + chunk_slot(r, c) * 16);
      if constexpr (H::AL)
        ws[n] = *reinterpret_cast<const uint8_t*>(sc + r * 16 + c);
      else
        ws[n] = *reinterpret_cast<const int*>(wst + H::kWStage + (r * 8 + scale_slot(r, c)) * 4);
    }
#pragma unroll
    for (int m = 0; m < H::MB; ++m) {
      const int r = xrow + 32 * m;
      x[m] = *reinterpret_cast<const uint4*>(xst + r * 128 + chunk_slot(r, c) * 16);
      if constexpr (H::AL)
        xs[m] = *reinterpret_cast<const uint8_t*>(sc + (kTN + r) * 16 + c);
      else
        xs[m] = *reinterpret_cast<const int*>(wst + H::kWStage + H::kWS + (r * 8 + scale_slot(r, c)) * 4);
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void multiply(f32x16 (&acc)[H::NB][H::MB]) const {
#pragma unroll
    for (int n = 0; n < H::NB; ++n)
#pragma unroll
      for (int m = 0; m < H::MB; ++m)
        acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes(w[n]), codes(x[m]), acc[n][m], 4, 4, 0, ws[n],
                                                                    0, xs[m]);
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ static i32x8 codes(uint4 v) {
    return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
  }
};

// bf16 tokens: half a stage of tokens at a time (32 entries of K).  A half goes
// through three phases: its codes and scales are read; they are widened and its
// tokens read; it is multiplied.  The phases of three halves run together, one
// read and two conversions behind each matrix-core op: both waves of a SIMD
// leave a barrier together, so what stands before or after the ops would leave
// the matrix cores idle in both.
template <class H>
struct Codes {
  uint2 w[H::NB];
  int s[H::NB];
  // row n's part of half u of stage g of tokens, in the weights' stage at wst
  __device__ __forceinline__ void read(int n, const char* wst, const char* sc, int g, int u, int wrow, int half) {
    const int c = 2 * g + half, r = wrow + 32 * n;
    w[n] = *reinterpret_cast<const uint2*>(wst + r * 128 + chunk_slot(r, c) * 16 + 8 * u);
    if constexpr (H::AL)
      s[n] = *reinterpret_cast<const uint8_t*>(sc + r * 16 + c);
    else
      s[n] = *reinterpret_cast<const int*>(wst + H::kWStage + (r * 8 + scale_slot(r, c)) * 4);
  }
};
template <class H>
struct Wide {
  uint4 w[2][H::NB];
  // words 2 i and 2 i + 1 of entry group j of row n, (j, n, i) the digits of k = 0 .. 7
  __device__ __forceinline__ void convert(int k, const Codes<H>& c) {
    const int j = k >> 2, n = (k >> 1) & 1;
    const uint32_t v = j ? c.w[n].y : c.w[n].x;
    const float s = mx4_scale(c.s[n]);
    if ((k & 1) == 0) {
      w[j][n].x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 0));
      w[j][n].y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 1));
    } else {
      w[j][n].z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 2));
      w[j][n].w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v, s, 3));
    }
  }
};
template <class H>
struct Tokens {
  uint4 x[H::MB][2];
  __device__ __forceinline__ void read(int m, int j, const char* xst, int u, int xrow, int half) {
    const int r = xrow + 32 * m;
    x[m][j] = *reinterpret_cast<const uint4*>(xst + r * 128 + chunk_slot(r, 4 * half + 2 * u + j) * 16);
  }
};

template <bool MX, bool AL, bool GLU>
__global__ __launch_bounds__(kTileThreads, 2) void mx4_tile_kernel(MulArgs a) {
  using H = Shape<MX, AL>;
  extern __shared__ __align__(16) char smem[];
  int32_t* const rowbuf = reinterpret_cast<int32_t*>(smem + H::oRows);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int TNO = GLU ? kTN / 2 : kTN;  // results a tile has of a slot
  const int wm = wave >> 2, wn = wave & 3, r32 = lane & 31, half = lane >> 5;
  const int K = static_cast<int>(a.K), kb = K / 32;
  const int nb = max((K + H::WK - 1) / H::WK, H::kLeast);  // stages of weights of a tile
  const int nx = nb * (H::WK / H::XK);                     // and of tokens
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const char *const zero = reinterpret_cast<const char*>(kPad), *const one = zero + 16;

  int head, none;
  Walk walk;
  Tile cur, next;
  bool more = walk.start(a.offsets, a.E, a.S, static_cast<int>((a.N + TNO - 1) / TNO), kTM, &head, &none);
  // slots of no expert: zeros
  for (int64_t i = blockIdx.x; i < head + (a.S - none); i += gridDim.x) {
    const int64_t s = i < head ? i : none + (i - head);
    for (int64_t n = threadIdx.x; n < a.N; n += kTileThreads) {
      if (a.yf32)
        static_cast<float*>(a.y)[s * a.ldy + n] = 0.0f;
      else
        static_cast<uint16_t*>(a.y)[s * a.ldy + n] = 0;
    }
  }
  if (!more) return;
  walk.get(&cur);

  // ---- where the loads come from: 8 lanes a row of tokens or weights, and of scales by bytes
  const char *px[H::LX], *pw[H::LW], *pws[AL ? 1 : H::LWS], *pxs[H::LXS ? H::LXS : 1], *pc = nullptr;
  auto row_of = [&](int q) { return (wave + kWaves * q) * 8 + lane / 8; };
  auto load_rows = [&](const Tile& t, int buf) {  // the rows of a tile's slots (past its end: its last)
    if (a.rows && wave < kTM / 64)
      load_lds4(a.rows + min(t.lo + wave * 64 + lane, t.hi - 1), lds0 + H::oRows + (buf * kTM + wave * 64) * 4);
  };
  auto token = [&](const Tile& t, int buf, int r) {  // (a row that does not exist: row 0, its results are replaced)
    if (!a.rows) return static_cast<int64_t>(min(t.lo + r, t.hi - 1));
    const int row = rowbuf[buf * kTM + r];
    return static_cast<int64_t>(row >= 0 && row < a.x_rows ? row : 0);
  };
  auto weight = [&](const Tile& t, int r) {
    const int64_t n0 = static_cast<int64_t>(t.col) * TNO;
    if constexpr (GLU)  // 32 gate rows, then the 32 up rows of the same outputs
      return static_cast<int64_t>(t.e) * 2 * a.N + min(n0 + (r >> 6) * 32 + (r & 31), a.N - 1) + ((r >> 5) & 1) * a.N;
    else
      return static_cast<int64_t>(t.e) * a.N + min(n0 + r, a.N - 1);
  };
  auto aim_x = [&](const Tile& t, int buf) {
#pragma unroll
    for (int q = 0; q < H::LX; ++q) {
      const int r = row_of(q), c = chunk_slot(r, lane & 7);
      const int64_t row = token(t, buf, r);
      px[q] = MX ? reinterpret_cast<const char*>(a.xcodes + row * kb * 16 + c * 16)
                 : reinterpret_cast<const char*>(a.x + row * a.ldx + c * 8);
    }
    if constexpr (!AL) {
#pragma unroll
      for (int q = 0; q < H::LXS; ++q) {
        const int r = row_of(q);
        pxs[q] = reinterpret_cast<const char*>(a.xscales + token(t, buf, r) * kb + scale_slot(r, lane & 7));
      }
    } else if (MX && wave >= 4 && wave < 6) {
      pc = reinterpret_cast<const char*>(a.xscales + token(t, buf, (wave - 4) * 64 + lane) * kb);
    }
  };
  auto aim_w = [&](const Tile& t) {
#pragma unroll
    for (int q = 0; q < H::LW; ++q) {
      const int r = row_of(q);
      pw[q] = reinterpret_cast<const char*>(a.codes + weight(t, r) * kb * 16 + chunk_slot(r, lane & 7) * 16);
    }
    if constexpr (!AL) {
#pragma unroll
      for (int q = 0; q < H::LWS; ++q) {
        const int r = row_of(q);
        pws[q] = reinterpret_cast<const char*>(a.scales + weight(t, r) * kb + scale_slot(r, lane & 7));
      }
    } else if (wave < 4) {
      pc = reinterpret_cast<const char*>(a.scales + weight(t, wave * 64 + lane) * kb);
    }
  };

  // ---- the loads of the next stage of tokens and of weights
  int xstep = 0, xto = 0, wstep = 0, wto = 0, cto = 0;
  auto issue_x = [&]() {
    const int rem = K - xstep * H::XK;  // entries from this stage on
#pragma unroll
    for (int q = 0; q < H::LX; ++q) {
      const char* p = px[q];
      if (rem < H::XK) {
        asm volatile("");  // (a branch, not three selects at every step)
        p = chunk_slot(row_of(q), lane & 7) * (MX ? 32 : 8) < rem ? p : zero;
      }
      load_lds16(p, lds0 + xto * H::kXStage + (wave + kWaves * q) * 1024);
      px[q] += 128;
    }
    ++xstep;
    xto = xto + 1 == H::NX ? 0 : xto + 1;
  };
  auto issue_w = [&]() {
    const int rem = K - wstep * H::WK;
    const uint32_t s = lds0 + H::oW + wto * H::kWRing;
    if constexpr (AL) {
      if ((wstep & 1) == 0) {  // the scales of 512 entries
        if (wave < (MX ? 6 : 4)) {
          load_lds16(rem > 0 ? pc : one, lds0 + H::oC + cto * H::kChunk + wave * 1024);
          pc += 16;
        }
        cto ^= 1;
      }
    }
#pragma unroll
    for (int q = 0; q < H::LW; ++q) {
      const char* p = pw[q];
      if (rem < H::WK) p = chunk_slot(row_of(q), lane & 7) * 32 < rem ? p : zero;
      load_lds16(p, s + (wave + kWaves * q) * 1024);
      pw[q] += 128;
    }
    if constexpr (!AL) {
#pragma unroll
      for (int q = 0; q < H::LWS; ++q) {
        const char* p = pws[q];
        if (rem < H::WK) p = scale_slot(row_of(q), lane & 7) * 32 < rem ? p : one;
        load_lds1(p, s + H::kWStage + (wave + kWaves * q) * 256);
        pws[q] += 8;
      }
#pragma unroll
      for (int q = 0; q < H::LXS; ++q) {
        const char* p = pxs[q];
        if (rem < H::WK) p = scale_slot(row_of(q), lane & 7) * 32 < rem ? p : one;
        load_lds1(p, s + H::kWStage + H::kWS + (wave + kWaves * q) * 256);
        pxs[q] += 8;
      }
    }
    ++wstep;
    wto = wto + 1 == H::NW ? 0 : wto + 1;
  };

  // ---- going on into the next tile
  int buf = 0;    // of rowbuf: the tile multiplied; the next one's is the one after
  int since = 0;  // steps since the next tile's rows were asked for
  bool xdry = false, wdry = false;  // loads of tokens, of weights are left out: there is no next tile
  auto after = [&](int b) { return b == 2 ? 0 : b + 1; };
  auto find_next = [&]() {
    walk.l += walk.step;
    more = walk.find();
    if (more) {
      walk.get(&next);
      load_rows(next, after(buf));
    }
    since = 0;
  };
  auto next_x = [&]() {  // whether there is a stage of tokens to load
    if (xstep < nx) return true;
    if (!more) return false;
    // the next tile's rows have landed if the tokens asked for since then fill the ring
    if (a.rows && since < H::NX) wait_loads<0>();
    aim_x(next, after(buf));
    xstep = 0;
    return true;
  };
  auto next_w = [&]() {
    if (wstep < nb) return true;
    if (!more) return false;
    aim_w(next);
    wstep = 0;
    return true;
  };

  load_rows(cur, 0);
  wait_loads<0>();
  aim_x(cur, 0);
  aim_w(cur);
  // the order of the main loop, which the counts of its waits go by
  issue_w();
  if constexpr (MX) {
    issue_x();
#pragma unroll
    for (int i = 1; i < H::NW; ++i) {
      issue_w();
      issue_x();
    }
    wait_loads<(H::NW - 1) * (H::kWLoads + H::LX)>();
  } else {
#pragma unroll
    for (int i = 0; i < H::NX - 1; ++i) issue_x();
    issue_w();
    issue_x();
    wait_loads<(H::NX - 1) * H::LX + H::kWLoads>();
  }
  find_next();

  const int wrow = wn * 64 + r32, xrow = wm * (kTM / 2) + r32;
  f32x16 acc[H::NB][H::MB];
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < H::NB; ++i)
#pragma unroll
      for (int j = 0; j < H::MB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  };
  clear();
  const char *xst = smem, *wst = smem + H::oW, *sc = smem + H::oC;
  auto advance_x = [&]() { xst = xst + H::kXStage == smem + H::oW ? smem : xst + H::kXStage; };
  int chunk = 0;
  auto advance_w = [&](int b) {  // to stage b of its tile
    wst = wst + H::kWRing == smem + H::oC ? smem + H::oW : wst + H::kWRing;
    if constexpr (AL) {
      if ((b & 1) == 0) chunk ^= 1;
      sc = smem + H::oC + chunk * H::kChunk + (b & 1) * 8;
    }
  };
  // MX4 tokens
  Frags<H> p, q;
  // bf16 tokens: halves 0 and 1 of a stage
  Codes<H> c0, c1;
  Wide<H> w0, w1;
  Tokens<H> x0, x1;
  // Multiplies a half by (w, x), widens the next (c to wn), and reads that one's tokens and the codes after those.
  auto work = [&](const Wide<H>& w, const Tokens<H>& x, const Codes<H>& c, Wide<H>& wnext, auto reads) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int j = k >> 2, n = (k >> 1) & 1, m = k & 1;
      acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, w.w[j][n]),
                                                          __builtin_bit_cast(bf16x8, x.x[m][j]), acc[n][m], 0, 0, 0);
      reads(k);
      wnext.convert(k, c);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if constexpr (MX) {
    p.read(xst, wst, sc, 0, wrow, xrow, half);
  } else {
#pragma unroll
    for (int n = 0; n < H::NB; ++n) {
      c0.read(n, wst, sc, 0, 0, wrow, half);
      c1.read(n, wst, sc, 0, 1, wrow, half);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) x0.read(k & 1, k >> 1, xst, 0, xrow, half);
#pragma unroll
    for (int k = 0; k < 8; ++k) w0.convert(k, c0);
  }
  for (;;) {
    for (int b = 0; b < nb; ++b) {
      if constexpr (MX) {
        q.read(xst, wst, sc, 1, wrow, xrow, half);
        p.multiply(acc);
        p.read(xst, wst, sc, 2, wrow, xrow, half);
        q.multiply(acc);
        q.read(xst, wst, sc, 3, wrow, xrow, half);
        p.multiply(acc);
        // the next stage has landed (but for the NW - 2 after it), and every wave has read this one
        if (xdry)
          wait_loads<0>();
        else
          wait_loads<(H::NW - 2) * (H::kWLoads + H::LX)>();
        ++since;
        if (next_x() && next_w()) {
          issue_w();
          issue_x();
        } else {
          xdry = true;
        }
        advance_x();
        advance_w(b + 1 == nb ? 0 : b + 1);
        p.read(xst, wst, sc, 0, wrow, xrow, half);  // (unused after the last tile)
        q.multiply(acc);
      } else {
        auto step = [&](auto gg) {  // stage of tokens 4 b + g
          constexpr int g = decltype(gg)::value;
          // codes are read a stage of tokens ahead
          if constexpr (g == 3) advance_w(b + 1 == nb ? 0 : b + 1);
          work(w0, x0, c1, w1, [&](int k) {
            if (k < 4)
              x1.read(k & 1, k >> 1, xst, 1, xrow, half);
            else if (k < 6)
              c0.read(k - 4, wst, sc, (g + 1) & 3, 0, wrow, half);
          });
          // The next stage of tokens has landed, and before the last step of a stage of weights the next one too:
          // later than those loads are those of NX - 2 stages of tokens, and of a stage of weights if the last step
          // of a stage of weights is among the steps they were issued in.
          if (xdry)
            wait_loads<0>();
          else if (wdry)
            wait_loads<(H::NX - 2) * H::LX>();
          else
            wait_loads<(H::NX - 2) * H::LX + (g < 2 && g <= H::NX - 3 ? H::kWLoads : 0)>();
          ++since;
          if constexpr (g == 3) {  // (every wave has read the codes before: their buffer is free)
            if (next_w())
              issue_w();
            else
              wdry = true;
          }
          if (next_x())
            issue_x();
          else
            xdry = true;
          advance_x();
          work(w1, x1, c0, w0, [&](int k) {  // (what is read after the last tile is not used)
            if (k < 4)
              x0.read(k & 1, k >> 1, xst, 0, xrow, half);
            else if (k < 6)
              c1.read(k - 4, wst, sc, (g + 1) & 3, 1, wrow, half);
          });
        };
        step(std::integral_constant<int, 0>());
        step(std::integral_constant<int, 1>());
        step(std::integral_constant<int, 2>());
        step(std::integral_constant<int, 3>());
      }
    }
    const int64_t n0 = static_cast<int64_t>(cur.col) * TNO;
    const bool whole = n0 + TNO <= a.N && a.ldy % 8 == 0;
#pragma unroll
    for (int m = 0; m < H::MB; ++m) {
      const int r = wm * (kTM / 2) + 32 * m + r32;
      const int64_t slot = cur.lo + r;
      if (slot >= cur.hi) continue;
      bool have = true;
      if (a.rows) have = rowbuf[buf * kTM + r] >= 0 && rowbuf[buf * kTM + r] < a.x_rows;
#pragma unroll
      for (int n = 0; n < (GLU ? 1 : H::NB); ++n) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          v[i] = acc[n][m][i];
          if constexpr (GLU) v[i] = silu(v[i]) * acc[1][m][i];
          v[i] = have ? v[i] : 0.0f;
        }
        store32(a, slot, n0 + wn * (GLU ? 32 : 64) + 32 * n, half, whole, a.N, v);
      }
    }
    if (!more) return;
    cur = next;
    buf = after(buf);
    clear();
    find_next();
  }
}

// ---------------------------------------------------------------------------
// dx in large tiles: 128 slots x 256 columns a workgroup of eight waves, which
// stays and takes tile after tile like the forward form.  n advances 64 rows of
// W a step.  The sum runs over W's rows, along which its scales change, so a
// step's codes (64 rows x 256 columns) are widened to bf16 once by the whole
// workgroup, a block of 32 a thread, into an LDS tile that the transposing LDS
// read takes fragments from.  Two such tiles: the next step's is made while this
// one's is multiplied, and between the matrix-core ops go the reads of the next
// sixteen rows' fragments and the conversions.  32768 slots over 128 experts, 2048
// x 768: 165 us, 0.62 PFLOP/s (0.78 with what pads the tiles), bound by the matrix
// cores' clock and, at half of their time, by the LDS (fragments used twice).
// ---------------------------------------------------------------------------
struct GradShape {
  static constexpr int KT = 256, NS = 64;  // columns, rows of W a step
  static constexpr int NX = 4, NW = 3;     // rings of dy and of codes with their scales
  static constexpr int kXStage = kTM * NS * 2, kCodes = NS * KT / 2, kWStage = kCodes + NS * (KT / 32) * 4;
  static constexpr int kTile = NS * KT * 2;
  static constexpr int oW = NX * kXStage, oTile = oW + NW * kWStage, kBytes = oTile + 2 * kTile;
  static constexpr int LX = kXStage / 1024 / kWaves, kWLoads = 2;
  static constexpr int MB = 2, NB = 2, kLeast = NX;
  static_assert(kBytes <= kLds);
};

__global__ __launch_bounds__(kTileThreads, 2) void mx4_grad_tile_kernel(MulArgs a) {
  using H = GradShape;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3, r32 = lane & 31, half = lane >> 5;
  const int64_t kb = a.K / 32;
  const int N = static_cast<int>(a.N), nk = max((N + H::NS - 1) / H::NS, H::kLeast);
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const char *const zero = reinterpret_cast<const char*>(kPad), *const one = zero + 16;

  int head, none;
  Walk walk;
  Tile cur, next;
  bool more = walk.start(a.offsets, a.E, a.S, static_cast<int>((a.K + H::KT - 1) / H::KT), kTM, &head, &none);
  for (int64_t i = blockIdx.x; i < head + (a.S - none); i += gridDim.x) {
    const int64_t s = i < head ? i : none + (i - head);
    for (int64_t k = tid; k < a.K; k += kTileThreads) {
      if (a.yf32)
        static_cast<float*>(a.y)[s * a.ldy + k] = 0.0f;
      else
        static_cast<uint16_t*>(a.y)[s * a.ldy + k] = 0;
    }
  }
  if (!more) return;
  walk.get(&cur);

  // ---- loads: dy's rows 8 lanes each; codes and scales of row wr, block lane % 8 of the tile
  const char *px[H::LX], *pw, *ps;
  const int wr = wave * 8 + lane / 8;
  const int64_t wstep = H::NS * kb * 16, sstep = H::NS * kb;
  auto row_of = [&](int q) { return (wave + kWaves * q) * 8 + lane / 8; };
  auto aim = [&](const Tile& t) {
#pragma unroll
    for (int q = 0; q < H::LX; ++q)
      px[q] = reinterpret_cast<const char*>(a.x + static_cast<int64_t>(min(t.lo + row_of(q), t.hi - 1)) * a.ldx +
                                            8 * chunk_slot(row_of(q), lane & 7));
    const int64_t block = min(static_cast<int64_t>(t.col) * (H::KT / 32) + (lane & 7), kb - 1);
    const int64_t row = static_cast<int64_t>(t.e) * a.N + wr;
    pw = reinterpret_cast<const char*>(a.codes + (row * kb + block) * 16);
    ps = reinterpret_cast<const char*>(a.scales + row * kb + block);
  };
  int step = 0, xto = 0, wto = 0;
  auto issue = [&]() {
    const int rem = N - step * H::NS;  // rows of W from this step on
    const char *w = pw, *s = ps;
    if (rem < H::NS) {
      asm volatile("");  // (a branch, not selects at every step)
      w = wr < rem ? w : zero;
      s = wr < rem ? s : one;
    }
    load_lds16(w, lds0 + H::oW + wto * H::kWStage + wave * 1024);
    load_lds1(s, lds0 + H::oW + wto * H::kWStage + H::kCodes + wave * 256);
    pw += wstep;
    ps += sstep;
#pragma unroll
    for (int q = 0; q < H::LX; ++q) {
      const char* p = px[q];
      if (rem < H::NS) {
        asm volatile("");
        p = 8 * chunk_slot(row_of(q), lane & 7) < rem ? p : zero;
      }
      load_lds16(p, lds0 + xto * H::kXStage + (wave + kWaves * q) * 1024);
      px[q] += H::NS * 2;
    }
    ++step;
    xto = xto + 1 == H::NX ? 0 : xto + 1;
    wto = wto + 1 == H::NW ? 0 : wto + 1;
  };
  bool dry = false;
  auto find_next = [&]() {
    walk.l += walk.step;
    more = walk.find();
    if (more) walk.get(&next);
  };
  auto go_on = [&]() {  // the loads of the next step, if there is one
    if (step == nk) {
      if (!more) {
        dry = true;
        return;
      }
      aim(next);
      step = 0;
    }
    issue();
  };

  // ---- a block of codes a thread, widened into row wr of a tile (chunk c of row r lies at c ^ 4 (r mod 4))
  const char* wst = smem + H::oW;
  auto advance_w = [&]() { wst = wst + H::kWStage == smem + H::oTile ? smem + H::oW : wst + H::kWStage; };
  uint4 codes;
  float scale;
  auto take = [&]() {
    codes = *reinterpret_cast<const uint4*>(wst + tid * 16);
    scale = mx4_scale(*reinterpret_cast<const uint32_t*>(wst + H::kCodes + tid * 4));
  };
  char* const into = smem + H::oTile + wr * (H::KT * 2);
  auto widen = [&](int i, int tile) {
    const uint32_t d = i == 0 ? codes.x : i == 1 ? codes.y : i == 2 ? codes.z : codes.w;
    *reinterpret_cast<uint4*>(into + tile * H::kTile + (((4 * (lane & 7) + i) ^ (4 * (wr & 3))) * 16)) =
        mx4_bf16_words(d, scale);
  };

  // ---- fragments of sixteen rows of W
  struct Part {
    bf16x8 x[H::MB];
    s16x4 w[H::NB][2];
  };
  const int xrow = wm * (kTM / 2) + r32;
  // read k (0 .. 5) of part j of the step at xst, in tile `tile`
  auto read = [&](Part& f, int k, int j, const char* xst, int tile) {
    if (k < 2) {
      const int r = xrow + 32 * k;
      f.x[k] = *reinterpret_cast<const bf16x8*>(xst + r * 128 + chunk_slot(r, 2 * j + half) * 16);
    } else {
      // rows 16 j + 8 half + 4 q + (lane % 16) / 4, column 16 ((lane / 16) % 2) + 4 (lane % 4) of block n
      const int n = (k - 2) >> 1, q = k & 1;
      const int col = wn * 64 + 32 * n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
      const int r = 16 * j + 8 * half + 4 * q + ((lane & 15) >> 2);
      f.w[n][q] = read_transposed(smem + H::oTile + tile * H::kTile + r * (H::KT * 2) +
                                  (((col >> 3) ^ (4 * (r & 3))) << 4) + (col & 7) * 2);
    }
  };
  f32x16 acc[H::NB][H::MB];
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < H::NB; ++i)
#pragma unroll
      for (int j = 0; j < H::MB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  };
  // The four ops of a part, with `between(k)` after op k.
  auto multiply = [&](const Part& f, auto between) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int n = k >> 1, m = k & 1;
      const bf16x8 w =
          __builtin_bit_cast(bf16x8, __builtin_shufflevector(f.w[n][0], f.w[n][1], 0, 1, 2, 3, 4, 5, 6, 7));
      acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, f.x[m], acc[n][m], 0, 0, 0);
      between(k);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  aim(cur);
  issue();
  issue();
  issue();
  wait_loads<2 * (H::kWLoads + H::LX)>();
  take();
#pragma unroll
  for (int i = 0; i < 4; ++i) widen(i, 0);
  advance_w();
  find_next();
  wait_loads<H::LX + H::kWLoads + H::LX>();  // (step 1's codes, too)
  go_on();
  clear();
  const char* xst = smem;
  int tile = 0;
  Part f0, f1;
#pragma unroll
  for (int k = 0; k < 6; ++k) read(f0, k, 0, xst, tile);
  for (;;) {
    for (int i = 0; i < nk; ++i) {
      multiply(f0, [&](int k) {
        if (k == 0) take();
        if (k == 0 || k == 1) read(f1, k, 1, xst, tile);
        if (k >= 2) {
          read(f1, 2 * k - 2, 1, xst, tile);
          read(f1, 2 * k - 1, 1, xst, tile);
        }
      });
      multiply(f1, [&](int k) {
        if (k < 2) read(f0, k, 2, xst, tile);
        if (k >= 2) {
          read(f0, 2 * k - 2, 2, xst, tile);
          read(f0, 2 * k - 1, 2, xst, tile);
        }
        if (k == 1) widen(0, tile ^ 1);
        if (k == 3) widen(1, tile ^ 1);
      });
      multiply(f0, [&](int k) {
        if (k < 2) read(f1, k, 3, xst, tile);
        if (k >= 2) {
          read(f1, 2 * k - 2, 3, xst, tile);
          read(f1, 2 * k - 1, 3, xst, tile);
        }
        if (k == 1) widen(2, tile ^ 1);
        if (k == 2) widen(3, tile ^ 1);
      });
      advance_w();
      // The next step's tile is whole, its dy and the codes after it have landed (but for what was asked for later: dy
      // of one step, and a step), and every wave has read all of this step.
      if (dry)
        wait_loads<0>();
      else
        wait_loads<H::LX + H::kWLoads + H::LX>();
      go_on();
      xst = xst + H::kXStage == smem + H::oW ? smem : xst + H::kXStage;
      tile ^= 1;
      multiply(f1, [&](int k) {  // (what is read after the last tile is not used)
        if (k < 2) read(f0, k, 0, xst, tile);
        if (k >= 2) {
          read(f0, 2 * k - 2, 0, xst, tile);
          read(f0, 2 * k - 1, 0, xst, tile);
        }
      });
    }
    const int64_t k0 = static_cast<int64_t>(cur.col) * H::KT;
    const bool whole = k0 + H::KT <= a.K && a.ldy % 8 == 0;
#pragma unroll
    for (int m = 0; m < H::MB; ++m) {
      const int64_t slot = cur.lo + wm * (kTM / 2) + 32 * m + r32;
      if (slot >= cur.hi) continue;
#pragma unroll
      for (int n = 0; n < H::NB; ++n) {
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = acc[n][m][i];
        store32(a, slot, k0 + wn * 64 + 32 * n, half, whole, a.K, v);
      }
    }
    if (!more) return;
    cur = next;
    clear();
    find_next();
  }
}

// dx for few slots an expert: 16 TB slots x 128 columns a workgroup.  As in the
// large tiles the codes of 64 rows of W are widened into an LDS tile for the
// transposing read, two tiles in turn; they come through registers, four steps
// ahead.  With few workgroups what counts is the length of one's chain of
// steps, so two groups of four waves take every other step, and join their sums
// at the end.  194 slots over 8 experts, 1024 x 4096: 17 us, launch and eight steps
// of load, widen, barrier and multiply; the bytes alone would take 5.
template <int TB>
__global__ __launch_bounds__(kTileThreads) void mx4_grad_few_kernel(MulArgs a) {
  constexpr int KT = 128, NS = 64, AHEAD = 4, C = KT / 64;
  constexpr int kTile = NS * KT * 2;
  __shared__ __align__(16) char tiles[2][2][kTile];
  __shared__ __align__(16) char dys[2][2][16 * TB * NS * 2];  // dy of a step: 128 bytes a slot
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int group = threadIdx.x >> 8, tid = threadIdx.x & 255, wave = tid >> 6;
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((a.K + KT - 1) / KT), 16 * TB, &t)) return;
  const int64_t k0 = static_cast<int64_t>(t.col) * KT;
  f32x4 acc[C][TB];
#pragma unroll
  for (int i = 0; i < C; ++i)
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[i][b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  if (t.e < a.E) {
    const int64_t kb = a.K / 32;
    const int N = static_cast<int>(a.N), trips = (N + 2 * NS - 1) / (2 * NS);
    // this thread's block of a step: row wr, block tid % 4
    const int wr = tid >> 2;
    const int64_t block = min(k0 / 32 + (tid & 3), kb - 1), row0 = static_cast<int64_t>(t.e) * a.N + wr;
    // and its eight entries of dy: slot tid / 8 (past the tile's end: its last), chunk tid % 8
    const int sl = tid >> 3, ch = tid & 7;
    const uint16_t* dy = a.x + static_cast<int64_t>(min(t.lo + min(sl, 16 * TB - 1), t.hi - 1)) * a.ldx + 8 * ch;
    uint4 c[AHEAD], x[AHEAD];
    int s[AHEAD];
    auto load = [&](int u, int trip) {
      const int n0 = (2 * trip + group) * NS;
      c[u] = x[u] = make_uint4(0, 0, 0, 0);
      s[u] = 127;
      if (n0 + wr < N) {
        c[u] = *reinterpret_cast<const uint4*>(a.codes + ((row0 + n0) * kb + block) * 16);
        s[u] = a.scales[(row0 + n0) * kb + block];
      }
      if (n0 + 8 * ch < N) x[u] = *reinterpret_cast<const uint4*>(dy + n0);
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(u, u);
    for (int t0 = 0; t0 < trips; t0 += AHEAD) {
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (t0 + u >= trips) break;
        char* w = tiles[group][u & 1];
        const uint32_t d[4] = {c[u].x, c[u].y, c[u].z, c[u].w};
        const float scale = mx4_scale(s[u]);
#pragma unroll
        for (int i = 0; i < 4; ++i)  // 16-byte chunk 4 (tid % 4) + i of the row, at c ^ 4 (row mod 4)
          *reinterpret_cast<uint4*>(w + wr * (KT * 2) + (((4 * (tid & 3) + i) ^ (4 * (wr & 3))) * 16)) =
              mx4_bf16_words(d[i], scale);
        char* g = dys[group][u & 1];
        if (sl < 16 * TB) *reinterpret_cast<uint4*>(g + sl * 128 + chunk_slot(sl, ch) * 16) = x[u];
        load(u, t0 + u + AHEAD);
        __syncthreads();
        bf16x8 y[2][TB];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < TB; ++b)
            y[h][b] = *reinterpret_cast<const bf16x8*>(g + (16 * b + r) * 128 + chunk_slot(16 * b + r, 4 * h + q) * 16);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < C; ++i) {
            // rows 32 h + 8 q + 4 p + (lane % 16) / 4, column 4 (lane % 4) of the block of sixteen
            const int col = wave * (16 * C) + 16 * i + 4 * (lane & 3);
            s16x4 v[2];
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const int n = 32 * h + 8 * q + 4 * p + (r >> 2);
              v[p] = read_transposed(w + n * (KT * 2) + (((col >> 3) ^ (4 * (n & 3))) << 4) + (col & 7) * 2);
            }
            const bf16x8 wf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int b = 0; b < TB; ++b)
              acc[i][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, y[h][b], acc[i][b], 0, 0, 0);
          }
      }
    }
  }
  __syncthreads();
  f32x4* join = reinterpret_cast<f32x4*>(&tiles[0][0][0]);  // [C * TB][256]
  static_assert(C * TB * 256 * 16 <= sizeof(tiles));
#pragma unroll
  for (int b = 0; b < TB; ++b)
#pragma unroll
    for (int i = 0; i < C; ++i)
      if (group == 1) join[(b * C + i) * 256 + tid] = acc[i][b];
  __syncthreads();
  if (group == 1) return;
#pragma unroll
  for (int b = 0; b < TB; ++b) {
    const int64_t slot = t.lo + 16 * b + r;
    if (slot >= t.hi) continue;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int64_t k = k0 + wave * (16 * C) + 16 * i + 4 * q;
      if (k < a.K) store4(a, slot, k, a.K, a.ldy % 4 == 0, acc[i][b] + join[(b * C + i) * 256 + tid]);
    }
  }
}

bitsmoe_status check(const char* who, const MulArgs& a, bitsmoe_dtype yt, int64_t wide) {
  auto bad = [who](bitsmoe_status st, const char* what) { return fail(st, std::string(who) + what); };
  if (a.E <= 0 || a.N <= 0 || a.K <= 0 || a.S < 0 || a.x_rows < 0)
    return bad(BITSMOE_ERR_ARG, ": non-positive size");
  if (yt != BITSMOE_F32 && yt != BITSMOE_BF16) return bad(BITSMOE_ERR_DTYPE, ": results are fp32 or bf16");
  // (slots are ints, and the end of a tile that begins at one is too)
  if (a.K % kMx4Block != 0 || a.K > (1 << 24) || a.N > (1 << 24) || a.E > 65535 || a.S > 0x7FFFFFFF - 2 * kTM ||
      a.x_rows > 0x7FFFFFFF)
    return bad(BITSMOE_ERR_SHAPE,
               ": needs K % 32 == 0, K and N <= 2^24, E <= 65535, S < 2^31 - 256 and rows < 2^31");
  if (a.ldy < wide || a.ldy > (int64_t(1) << 32))
    return bad(BITSMOE_ERR_SHAPE, ": the results' row stride is too small or too large");
  if (!a.offsets && a.E != 1) return bad(BITSMOE_ERR_ARG, ": no offsets, and more than one expert");
  if (a.S > 0 && (!a.codes || !a.scales || !a.y)) return bad(BITSMOE_ERR_ARG, ": null pointer");
  if (!a.rows && a.x_rows < a.S) return bad(BITSMOE_ERR_SHAPE, ": fewer rows than slots");
  if (!aligned16({a.codes, a.scales, a.x, a.xcodes, a.xscales, a.offsets, a.rows, a.y}))
    return bad(BITSMOE_ERR_ARG, ": device pointers must be 16-byte aligned");
  return BITSMOE_OK;
}

// Workgroups for tiles of `tile` slots and `per` workgroups each.
bool grid_of(const MulArgs& a, int64_t tile, int64_t per, unsigned* grid) {
  const int64_t tiles = a.S / tile + (a.E + 2 < a.S ? a.E + 2 : a.S);  // (every run's last one may be part)
  if (tiles > ((int64_t(1) << 23) - 1) / per) return false;  // (2^32 threads of 512 a workgroup)
  *grid = static_cast<unsigned>(tiles * per);
  return true;
}

// Which kernel takes a call.  The counts of an expert's slots are on the device;
// the host goes by S and E alone: about
//     tiles(m) = max(active, S / m + active / 2),  active = E (1 - exp(-S / E))
// tiles of m slots (as of slots that choose by chance), whose workgroups either run side by side (the length of one's
// chain of steps counts) or fill the card (their number does).  The constants (us;
// L entries of the sum) fit timings of all kernels at thirty shapes, E 1 .. 256,
// 1/8 .. 4096 slots an expert, outputs 256 .. 14336, sums of 512 .. 14336 entries:
// the choice is within 1.25 times the best of them (1 % on average), and the worst of
// them is mostly two to four times that, fourteen at most (one expert, 64 slots,
// 1024 x 4096: 50 us in large tiles, 41 in few-slot ones, 9 by rows; 4096 slots,
// 4096 x 4096: 150, 257, 1341).
enum Kernel { kByRows, kFewSlots, kLargeTiles };

double tiles_of(const MulArgs& a, int64_t m) {
  const double E = static_cast<double>(a.E), active = E * (1.0 - std::exp(-static_cast<double>(a.S) / E));
  const double t = static_cast<double>(a.S) / static_cast<double>(m) + active / 2;
  return t > active ? t : active;
}
// Slots of a tile of the kernels for few.
int64_t few_slots(const MulArgs& a) { return a.S > 8 * static_cast<int64_t>(a.E) ? 32 : 16; }

// us of `groups` workgroups whose chain takes `chain`, and `each` where they fill the card.
double side_by_side(double groups, double chain, double each) {
  const double full = groups * each;
  return chain > full ? chain : full;
}
// us of large tiles, a workgroup a compute unit
double in_rounds(double tiles, double each) {
  const int64_t rounds = (static_cast<int64_t>(tiles) + device_cus() - 1) / device_cus();
  return 3.0 + static_cast<double>(rounds < 1 ? 1 : rounds) * each;
}

Kernel product_kernel(const MulArgs& a, bool mx, bool glu) {
  const int64_t wide = a.N * (glu ? 2 : 1);
  const double L = static_cast<double>(a.K), c16 = static_cast<double>((wide + 15) / 16),
               c256 = static_cast<double>((wide + 255) / 256);
  const double rows = 6.0 + tiles_of(a, 16) * c16 * L * (mx ? 3.6e-6 : 5.2e-6);
  const double few = 4.0 + L * side_by_side(tiles_of(a, few_slots(a)) * c256, mx ? 0.006 : 0.0095, mx ? 3e-5 : 4e-5);
  const double large = in_rounds(tiles_of(a, kTM) * c256, L * (mx ? 0.0058 : 0.0117) + (mx ? 4.0 : 5.0));
  if (a.x_rows > 0 && large <= rows && large <= few) return kLargeTiles;
  return few <= rows ? kFewSlots : kByRows;
}

Kernel grad_kernel(const MulArgs& a) {
  const double L = static_cast<double>(a.N), c128 = static_cast<double>((a.K + 127) / 128),
               c256 = static_cast<double>((a.K + 255) / 256);
  const double few = 4.0 + L * side_by_side(tiles_of(a, few_slots(a)) * c128, 0.0055, 2.4e-5);
  const double large = in_rounds(tiles_of(a, kTM) * c256, L * 0.0165 + 4.0);
  return large <= few ? kLargeTiles : kFewSlots;
}

// One workgroup a compute unit, as many on every XCD.
unsigned tile_grid() {
  const int cus = device_cus();
  return static_cast<unsigned>(cus < 8 ? 8 : cus / 8 * 8);
}

template <bool MX, bool AL, bool GLU>
bitsmoe_status tile_product(const MulArgs& a, hipStream_t s) {
  constexpr int lds = Shape<MX, AL>::kBytes;
  auto* fn = mx4_tile_kernel<MX, AL, GLU>;
  static std::atomic<uint64_t> allowed{0};
  if (bitsmoe_status st = allow_lds(reinterpret_cast<const void*>(fn), lds, &allowed)) return st;
  KernelTimer timer("mx4_tile", s);
  fn<<<tile_grid(), kTileThreads, lds, s>>>(a);
  BITSMOE_LAUNCH_CHECK("mx4_tile_kernel");
  return ok();
}

// A call with more tiles than a launch takes goes to the resident workgroups of the large tiles, unless it has few
// slots an expert (their walk over the experts is long) or no row that they could read for a slot without one.
bool large_instead(const MulArgs& a) { return a.S > 8 * static_cast<int64_t>(a.E) && a.x_rows > 0; }

bitsmoe_status product(const char* who, const MulArgs& a, bool mx, bool glu, hipStream_t s) {
  Kernel kernel = product_kernel(a, mx, glu);
  unsigned grid = 0;
  const bool fits = kernel == kLargeTiles ||
                    (kernel == kFewSlots ? grid_of(a, few_slots(a), (a.N + (glu ? 127 : 255)) / (glu ? 128 : 256), &grid)
                                         : grid_of(a, 16, (a.N + 15) / 16, &grid));
  if (!fits) {
    if (!large_instead(a))
      return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": too many slots and outputs for one call");
    kernel = kLargeTiles;
  }
  if (kernel == kLargeTiles) {
    // (with MX4 tokens four stages of weights a tile at least, so that a chunk of scales outlives its two)
    const bool al = a.K % 512 == 0 && (!mx || a.K >= 1024);
    if (mx && al) return glu ? tile_product<true, true, true>(a, s) : tile_product<true, true, false>(a, s);
    if (mx) return glu ? tile_product<true, false, true>(a, s) : tile_product<true, false, false>(a, s);
    if (al) return glu ? tile_product<false, true, true>(a, s) : tile_product<false, true, false>(a, s);
    return glu ? tile_product<false, false, true>(a, s) : tile_product<false, false, false>(a, s);
  }
  if (kernel == kFewSlots) {
    const bool two = few_slots(a) == 32;
    auto* fn = two ? (mx ? (glu ? mx4_few_kernel<true, true, 2> : mx4_few_kernel<true, false, 2>)
                         : (glu ? mx4_few_kernel<false, true, 2> : mx4_few_kernel<false, false, 2>))
                   : (mx ? (glu ? mx4_few_kernel<true, true, 1> : mx4_few_kernel<true, false, 1>)
                         : (glu ? mx4_few_kernel<false, true, 1> : mx4_few_kernel<false, false, 1>));
    KernelTimer timer("mx4_few", s);
    fn<<<grid, kThreads, 0, s>>>(a);
    BITSMOE_LAUNCH_CHECK("mx4_few_kernel");
    return ok();
  }
  auto* fn = mx ? (glu ? mx4_rows_kernel<true, true> : mx4_rows_kernel<true, false>)
                : (glu ? mx4_rows_kernel<false, true> : mx4_rows_kernel<false, false>);
  KernelTimer timer("mx4_rows", s);
  fn<<<grid, kThreads, 0, s>>>(a);
  BITSMOE_LAUNCH_CHECK("mx4_rows_kernel");
  return ok();
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" bitsmoe_status bitsmoe_mx4_product(const uint8_t* codes_dev, const uint8_t* scales_dev, int64_t E,
                                              int64_t N, int64_t K, const void* X_dev, bitsmoe_dtype xt,
                                              int64_t x_rows, int64_t ldx, const int32_t* offsets_dev,
                                              const int32_t* rows_dev, int64_t S, int glu, void* Y_dev,
                                              bitsmoe_dtype yt, int64_t ldy, void* stream) {
  MulArgs a{codes_dev, scales_dev, static_cast<int>(E < 0x7FFFFFFF ? E : 0x7FFFFFFF), N, K,
            static_cast<const uint16_t*>(X_dev), nullptr, nullptr, x_rows, ldx, offsets_dev, rows_dev, S,
            Y_dev, ldy, yt == BITSMOE_F32};
  if (bitsmoe_status st = check("mx4_product", a, yt, N)) return st;
  if (xt != BITSMOE_BF16) return fail(BITSMOE_ERR_DTYPE, "mx4_product: tokens must be bf16");
  if (ldx < K || ldx % 8 != 0 || ldx > (int64_t(1) << 32))
    return fail(BITSMOE_ERR_SHAPE, "mx4_product: needs ldx >= K and ldx % 8 == 0");
  if (S == 0) return ok();
  if (x_rows > 0 && !X_dev) return fail(BITSMOE_ERR_ARG, "mx4_product: null pointer");
  return product("mx4_product", a, false, glu != 0, static_cast<hipStream_t>(stream));
}

extern "C" bitsmoe_status bitsmoe_mx4_product_q(const uint8_t* codes_dev, const uint8_t* scales_dev, int64_t E,
                                                int64_t N, int64_t K, const uint8_t* xcodes_dev,
                                                const uint8_t* xscales_dev, int64_t x_rows,
                                                const int32_t* offsets_dev, const int32_t* rows_dev, int64_t S,
                                                int glu, void* Y_dev, bitsmoe_dtype yt, int64_t ldy,
                                                void* stream) {
  MulArgs a{codes_dev, scales_dev, static_cast<int>(E < 0x7FFFFFFF ? E : 0x7FFFFFFF), N, K,
            nullptr, xcodes_dev, xscales_dev, x_rows, 0, offsets_dev, rows_dev, S,
            Y_dev, ldy, yt == BITSMOE_F32};
  if (bitsmoe_status st = check("mx4_product_q", a, yt, N)) return st;
  if (S == 0) return ok();
  if (x_rows > 0 && (!xcodes_dev || !xscales_dev)) return fail(BITSMOE_ERR_ARG, "mx4_product_q: null pointer");
  return product("mx4_product_q", a, true, glu != 0, static_cast<hipStream_t>(stream));
}

extern "C" bitsmoe_status bitsmoe_mx4_product_grad(const uint8_t* codes_dev, const uint8_t* scales_dev, int64_t E,
                                                   int64_t N, int64_t K, const void* dY_dev, bitsmoe_dtype dyt,
                                                   int64_t lddy, const int32_t* offsets_dev, int64_t S,
                                                   void* dX_dev, bitsmoe_dtype xt, int64_t ldx, void* stream) {
  MulArgs a{codes_dev, scales_dev, static_cast<int>(E < 0x7FFFFFFF ? E : 0x7FFFFFFF), N, K,
            static_cast<const uint16_t*>(dY_dev), nullptr, nullptr, S, lddy, offsets_dev, nullptr, S,
            dX_dev, ldx, xt == BITSMOE_F32};
  if (bitsmoe_status st = check("mx4_product_grad", a, xt, K)) return st;
  if (dyt != BITSMOE_BF16) return fail(BITSMOE_ERR_DTYPE, "mx4_product_grad: dY must be bf16");
  if (N % 8 != 0 || lddy < N || lddy % 8 != 0 || lddy > (int64_t(1) << 32))
    return fail(BITSMOE_ERR_SHAPE, "mx4_product_grad: needs N % 8 == 0, lddy >= N and lddy % 8 == 0");
  if (S == 0) return ok();
  if (!dY_dev) return fail(BITSMOE_ERR_ARG, "mx4_product_grad: null pointer");
  unsigned grid = 0;
  Kernel kernel = grad_kernel(a);
  if (kernel != kLargeTiles && !grid_of(a, few_slots(a), (K + 127) / 128, &grid)) {
    if (!large_instead(a))
      return fail(BITSMOE_ERR_SHAPE, "mx4_product_grad: too many slots and columns for one call");
    kernel = kLargeTiles;
  }
  if (kernel == kLargeTiles) {
    static std::atomic<uint64_t> allowed{0};
    if (bitsmoe_status st = allow_lds(reinterpret_cast<const void*>(mx4_grad_tile_kernel), GradShape::kBytes, &allowed))
      return st;
    KernelTimer timer("mx4_grad_tile", stream);
    mx4_grad_tile_kernel<<<tile_grid(), kTileThreads, GradShape::kBytes, static_cast<hipStream_t>(stream)>>>(a);
    BITSMOE_LAUNCH_CHECK("mx4_grad_tile_kernel");
    return ok();
  }
  auto* fn = few_slots(a) == 32 ? mx4_grad_few_kernel<2> : mx4_grad_few_kernel<1>;
  KernelTimer timer("mx4_grad_few", stream);
  fn<<<grid, kTileThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("mx4_grad_few_kernel");
  return ok();
}
