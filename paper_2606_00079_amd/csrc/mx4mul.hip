// Products with expert weights held in MX4.
//
//     y_s = W_e(s) x_row(s)            (mx4_product: bf16 tokens; _q: MX4 tokens)
//     y_s = silu(g) u, [g; u] = W_e(s) x_row(s)        (the same with glu)
//     dx_s = W_e(s)^T dy_s             (mx4_product_grad)
//
// for S slots in expert order, expert e's being offsets[e] .. offsets[e+1].
#include <cstdint>
#include <string>

#include "internal.hpp"
#include "mx4.hpp"

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

// Inclusive sums over the wave (a step inside a row of 16 lanes shifts by 1, 2,
// 4, 8; then a row's last lane is added to the next row, and lane 31 to the
// upper half).
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}
__device__ __forceinline__ int lane_value(int v, int l) { return __builtin_amdgcn_readlane(v, l); }

// The slots of one workgroup, `lo` .. `hi` of expert e, and its column tile.
// Each expert's slots are cut into tiles of `tile` from its first on; e = E
// holds the slots of no expert, whose results are zero.
//
// Workgroup ids go to the eight XCDs in turn; each XCD gets a contiguous range of
// the tiles that exist (ids past them find none), ordered by expert, and there
// up to eight slot tiles of a column tile in a row: the workgroups that run on
// an XCD at a time share weights and tokens in its L2.  Every wave looks by
// itself: a lane sums up a run of experts, the waves' sums tell the run, and a
// second pass of one expert a lane the expert.
struct Tile {
  int e, lo, hi, col;
};
__device__ __forceinline__ int slots_of(const int32_t* offsets, int E, int S, int e, int* lo) {
  *lo = offsets ? min(max(offsets[e], 0), S) : (e == 0 ? 0 : S);
  return (e < E && offsets ? min(max(offsets[e + 1], *lo), S) : S) - *lo;
}
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int E, int64_t S, int cols, int tile, Tile* out) {
  const int s = static_cast<int>(S), lane = threadIdx.x & 63;
  const int per = E / 64 + 1;  // experts a lane, of E + 1
  int lo, tiles = 0;
  for (int i = 0; i < per; ++i) {
    const int e = lane * per + i;
    if (e <= E) tiles += (slots_of(offsets, E, s, e, &lo) + tile - 1) / tile;
  }
  int sum = wave_scan(tiles);
  const int64_t n = static_cast<int64_t>(lane_value(sum, 63)) * cols, id = blockIdx.x;
  if (id >= n) return false;
  const int64_t x = id & 7, q = n >> 3, rem = n & 7;
  const int64_t l = x * q + (x < rem ? x : rem) + (id >> 3);
  const int g = static_cast<int>(l / cols);
  const int run = __builtin_ctzll(__ballot(sum > g));
  int base = run ? lane_value(sum, run - 1) : 0;
  int e = run * per;
  for (;; e += 64) {  // (one pass up to 4095 experts)
    const int f = e + lane;
    const int have = f <= E && f < (run + 1) * per ? slots_of(offsets, E, s, f, &lo) : 0;
    tiles = (have + tile - 1) / tile;
    sum = base + wave_scan(tiles);
    const uint64_t hit = __ballot(sum > g);
    if (hit || e + 64 >= (run + 1) * per) {
      const int at = hit ? __builtin_ctzll(hit) : 63;
      const int m = lane_value(tiles, at), first = lane_value(lo, at), count = lane_value(have, at);
      const int64_t in = l - static_cast<int64_t>(lane_value(sum, at) - m) * cols;
      const int group = static_cast<int>(in / (8 * static_cast<int64_t>(cols)));
      const int rest = static_cast<int>(in - group * 8 * static_cast<int64_t>(cols));
      const int high = min(8, m - 8 * group);
      const int row = 8 * group + rest % high;
      out->e = e + at;
      out->col = rest / high;
      out->lo = first + row * tile;
      out->hi = min(first + count, out->lo + tile);
      return true;
    }
    base = lane_value(sum, 63);
  }
}

// The same order of tiles for a workgroup that stays and takes one tile after
// another (without those of e = E): it goes on from expert to expert with
// scalar loads, which do not touch the count of its vector loads.
struct Walk {
  const __attribute__((address_space(4))) int32_t* offsets;
  int E, S, cols, tile;
  int64_t l, end, step;       // this workgroup's tile, the end of its XCD's range
  int e, before, first, count;  // expert, tiles before it, its first slot and their number
  __device__ __forceinline__ int tiles() const { return (count + tile - 1) / tile; }
  __device__ __forceinline__ void load() {
    first = offsets ? min(max(offsets[e], 0), S) : 0;
    count = (offsets ? min(max(offsets[e + 1], first), S) : S) - first;
  }
  // to the expert of tile l; false if there is none
  __device__ __forceinline__ bool find() {
    if (l >= end) return false;
    const int g = static_cast<int>(l / cols);
    while (g >= before + tiles()) {
      before += tiles();
      ++e;
      load();
    }
    return true;
  }
  __device__ __forceinline__ void get(Tile* out) const {
    const int64_t in = l - static_cast<int64_t>(before) * cols;
    const int group = static_cast<int>(in / (8 * static_cast<int64_t>(cols)));
    const int rest = static_cast<int>(in - group * 8 * static_cast<int64_t>(cols));
    const int high = min(8, tiles() - 8 * group), row = 8 * group + rest % high;
    out->e = e;
    out->col = rest / high;
    out->lo = first + row * tile;
    out->hi = min(first + count, out->lo + tile);
  }
  // The first tile of this workgroup; *none: where the slots of no expert begin.
  __device__ __forceinline__ bool start(const int32_t* off, int E_, int64_t S_, int cols_, int tile_, int* none) {
    offsets = (const __attribute__((address_space(4))) int32_t*)reinterpret_cast<uintptr_t>(off);
    E = E_, S = static_cast<int>(S_), cols = cols_, tile = tile_;
    const int lane = threadIdx.x & 63, per = (E + 63) / 64;
    int lo, sum = 0;
    for (int i = 0; i < per; ++i) {
      const int f = lane * per + i;
      if (f < E) sum += (slots_of(off, E, S, f, &lo) + tile - 1) / tile;
    }
    const int own = sum;
    sum = wave_scan(sum);
    *none = offsets ? min(max(offsets[E], 0), S) : S;
    const int64_t n = static_cast<int64_t>(lane_value(sum, 63)) * cols;
    const int64_t x = blockIdx.x & 7, q = n >> 3, rem = n & 7;
    const int64_t begin = x * q + (x < rem ? x : rem);
    end = begin + q + (x < rem ? 1 : 0);
    step = gridDim.x >> 3;
    l = begin + (blockIdx.x >> 3);
    if (l >= end) return false;
    const int run = __builtin_ctzll(__ballot(sum > static_cast<int>(l / cols)));
    before = lane_value(sum, run) - lane_value(own, run);
    e = run * per;
    load();
    return find();
  }
};

__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }

// Four consecutive results n .. n + 3 of slot s.
__device__ __forceinline__ void store4(const MulArgs& a, int64_t s, int64_t n, int64_t N, bool wide, f32x4 v) {
  if (a.yf32) {
    float* p = static_cast<float*>(a.y) + s * a.ldy + n;
    if (wide && n + 4 <= N) {
      *reinterpret_cast<f32x4*>(p) = v;
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) p[i] = v[i];
  } else {
    uint16_t* p = static_cast<uint16_t*>(a.y) + s * a.ldy + n;
    uint16_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v[i]));
    if (wide && n + 4 <= N) {
      *reinterpret_cast<uint2*>(p) = make_uint2(h[0] | (uint32_t(h[1]) << 16), h[2] | (uint32_t(h[3]) << 16));
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) p[i] = h[i];
  }
}

// 16 outputs x 16 slots a workgroup.  The four waves share out K in segments
// of 128: lane l holds 32 codes of row l % 16 (block l / 16 of the segment),
// which one load fetches with their scale, and the same entries of slot l % 16.
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
  if (t.e < a.E) {
    const int64_t n = min(n0 + r, a.N - 1);
    const int64_t slot = t.lo + r;
    const int64_t row = slot < t.hi ? (a.rows ? static_cast<int64_t>(a.rows[slot]) : slot) : -1;
    const bool have = row >= 0 && row < a.x_rows;
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
  const int64_t slot = t.lo + r, n = n0 + 4 * q;  // (a lane holds four outputs of one slot)
  const bool wide = a.ldy % 4 == 0;
  if (slot < t.hi && n < a.N) store4(a, slot, n, a.N, wide, acc[0]);
}

// ---------------------------------------------------------------------------
// Large tiles: TM slots x 256 outputs a workgroup of eight waves.
//
// K advances KS entries at a time through kStages LDS stages that direct
// global->LDS loads fill (16 bytes a lane for codes and tokens, one byte a lane,
// widened to a word, for scales): codes stay four bits wide up to the registers.
// Wave (wm, wn) of 2 x 4 owns TM/2 slots x 64 outputs as 32 x 32 accumulators,
// the weights on the matrix core's row side, so that a lane holds runs of four
// outputs of one slot.  With bf16 tokens a wave widens each fragment of codes
// once (exact) and uses it for its TM/64 blocks of slots; with MX4 tokens the
// scaled matrix-core form takes codes and scales as they lie.
// ---------------------------------------------------------------------------
constexpr int kTileThreads = 512, kWaves = 8, kTN = 256;

template <bool MX, int TM_>
struct Shape {
  static constexpr int TM = TM_;
  static constexpr int KS = MX ? 256 : 128;      // entries of K a step
  static constexpr int XB = MX ? KS / 2 : 2 * KS;  // bytes of a token's row in a stage
  static constexpr int WB = KS / 2;              // bytes of a weight row in a stage
  static constexpr int SC = KS / 32;             // scales of a row in a stage (a word each)
  static constexpr int kX = 0, kW = TM * XB, kWS = kW + kTN * WB, kXS = kWS + kTN * SC * 4;
  static constexpr int kStage = kXS + (MX ? TM * SC * 4 : 0);
  static constexpr int kStages = 163840 / kStage;
  // direct loads of a wave for a stage
  static constexpr int LX = TM * XB / 1024 / kWaves, LW = kTN * WB / 1024 / kWaves;
  static constexpr int LWS = kTN * SC / 64 / kWaves, LXS = MX ? TM * SC / 64 / kWaves : 0;
  static constexpr int kLoads = LX + LW + LWS + LXS;
  static constexpr int MB = TM / 64, NB = 2;
  static_assert(kStages >= 2 && (kStages - 1) * kLoads < 64);
};

// What lanes past the end of a row read: zeros, and scales of 1.
__device__ const uint8_t kPad[32] __attribute__((aligned(16))) = {
    0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,   0,
    127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127, 127};

// One wave-wide direct load: lane l's 16 bytes (or byte) at p go to lds + 16 l
// (lds + 4 l, as a word).  `lds` is wave-uniform.  The compiler does not track
// it: callers wait by count (wait_loads) and synchronize before the data is read.
__device__ __forceinline__ void load_lds16(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory");
}
__device__ __forceinline__ void load_lds1(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_ubyte %0, off" ::"v"(p),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory");
}
// Waits until at most N of this wave's loads, and none of its LDS reads, are
// under way, and for the workgroup.
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Slot of 16-byte chunk c of row r in a stage whose rows have `chunks` of them:
// sixteen rows read at the same chunk (what the LDS serves together) then lie in
// different banks.
template <int chunks>
__device__ __forceinline__ int chunk_slot(int r, int c) {
  return c ^ ((r / (16 / chunks)) & (chunks - 1));
}

// Place of scale c of row r among the SC words of its row: as above, for words
// that two half-waves read at neighbouring places.
template <int SC>
__device__ __forceinline__ int scale_slot(int r, int c) {
  return c ^ (2 * ((r * SC / 64) & (SC / 2 - 1)));
}

// The operand fragments of a quarter of a step (32 entries of K with bf16
// tokens, 64 with MX4 ones): read from a stage while the quarter before is
// multiplied.
template <bool MX, int TM>
struct Frags {
  using H = Shape<MX, TM>;
  uint4 w[H::NB];  // bf16 tokens: two words of each in use
  uint4 x[H::MB][MX ? 1 : 2];
  int ws[H::NB], xs[MX ? H::MB : 1];
  // quarter u of the stage at s; wrow, xrow: this lane's first rows
  template <int u>
  __device__ __forceinline__ void read(const char* s, int wrow, int xrow, int half) {
    const int c = 2 * (MX ? u : u / 2) + half;  // this lane's block of 32 in the step
    constexpr int WC = H::WB / 16, XC = H::XB / 16;
#pragma unroll
    for (int n = 0; n < H::NB; ++n) {
      const int r = wrow + 32 * n;
      const char* at = s + H::kW + r * H::WB + chunk_slot<WC>(r, c) * 16;
      if constexpr (MX) {
        w[n] = *reinterpret_cast<const uint4*>(at);
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(at + 8 * (u % 2));
        w[n].x = v.x;
        w[n].y = v.y;
      }
      ws[n] = *reinterpret_cast<const int*>(s + H::kWS + (r * H::SC + scale_slot<H::SC>(r, c)) * 4);
    }
#pragma unroll
    for (int m = 0; m < H::MB; ++m) {
      const int r = xrow + 32 * m;
      const char* row = s + H::kX + r * H::XB;
      if constexpr (MX) {
        x[m][0] = *reinterpret_cast<const uint4*>(row + chunk_slot<XC>(r, c) * 16);
        xs[m] = *reinterpret_cast<const int*>(s + H::kXS + (r * H::SC + scale_slot<H::SC>(r, c)) * 4);
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          x[m][j] = *reinterpret_cast<const uint4*>(row + chunk_slot<XC>(r, 4 * c + 2 * (u % 2) + j) * 16);
      }
    }
  }
  __device__ __forceinline__ void multiply(f32x16 (&acc)[H::NB][H::MB]) const {
    if constexpr (MX) {
#pragma unroll
      for (int n = 0; n < H::NB; ++n)
#pragma unroll
        for (int m = 0; m < H::MB; ++m)
          acc[n][m] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(codes(w[n]), codes(x[m][0]), acc[n][m], 4, 4, 0,
                                                                      ws[n], 0, xs[m]);
    } else {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int n = 0; n < H::NB; ++n) {
          const bf16x8 wf = mx4_bf16(j ? w[n].y : w[n].x, mx4_scale(ws[n]));
#pragma unroll
          for (int m = 0; m < H::MB; ++m)
            acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf, __builtin_bit_cast(bf16x8, x[m][j]), acc[n][m], 0,
                                                                0, 0);
        }
    }
  }
  __device__ __forceinline__ static i32x8 codes(uint4 v) {
    return i32x8{(int)v.x, (int)v.y, (int)v.z, (int)v.w, 0, 0, 0, 0};
  }
};

template <bool MX, bool GLU, int TM>
__global__ __launch_bounds__(kTileThreads, 2) void mx4_tile_kernel(MulArgs a) {
  using H = Shape<MX, TM>;
  extern __shared__ __align__(16) char smem[];
  // rows of X of the slots of three tiles: the one multiplied, the next, and one before
  int32_t* const rowbuf = reinterpret_cast<int32_t*>(smem + H::kStages * H::kStage);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int TNO = GLU ? kTN / 2 : kTN;  // results a tile has of a slot
  const int wm = wave >> 2, wn = wave & 3, r32 = lane & 31, half = lane >> 5;
  const int64_t kb = a.K / 32;
  const int nk = static_cast<int>((a.K + H::KS - 1) / H::KS);
  const int last = static_cast<int>(a.K - static_cast<int64_t>(nk - 1) * H::KS);  // entries of the last step
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));

  int none;
  Walk walk;
  Tile cur, next;
  bool more = walk.start(a.offsets, a.E, a.S, static_cast<int>((a.N + TNO - 1) / TNO), TM, &none);
  // slots of no expert: zeros
  for (int64_t s = none + static_cast<int64_t>(blockIdx.x); s < a.S; s += gridDim.x)
    for (int64_t n = threadIdx.x; n < a.N; n += kTileThreads) {
      if (a.yf32)
        static_cast<float*>(a.y)[s * a.ldy + n] = 0.0f;
      else
        static_cast<uint16_t*>(a.y)[s * a.ldy + n] = 0;
    }
  if (!more) return;
  walk.get(&cur);

  // Direct loads.  They run through the stages of one tile after another, a
  // ring of kStages ahead of the multiplication and at most into the tile after
  // the one multiplied, so that a tile's results are stored while the next
  // one's first stages are on their way.
  constexpr int XC = H::XB / 16, WC = H::WB / 16;
  const char *px[H::LX], *pw[H::LW], *pws[H::LWS], *pxs[MX ? H::LXS : 1];
  auto row_of = [&](int q, int per) { return (wave + kWaves * q) * per + lane / (64 / per); };
  auto load_rows = [&](const Tile& t, int buf) {  // the rows of a tile's slots (past its end: its last)
    if (a.rows && wave < TM / 64) {
      const int32_t* p = a.rows + min(t.lo + wave * 64 + lane, t.hi - 1);
      asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" ::"v"(p),
                   "s"(__builtin_amdgcn_readfirstlane(lds0 + H::kStages * H::kStage + (buf * TM + wave * 64) * 4))
                   : "memory");
    }
  };
  auto aim = [&](const Tile& t, int buf) {  // the loads' addresses in the first stage of a tile
    auto token = [&](int r) {  // (a row that does not exist: row 0, its results are replaced)
      if (!a.rows) return static_cast<int64_t>(min(t.lo + r, t.hi - 1));
      const int row = rowbuf[buf * TM + r];
      return static_cast<int64_t>(row >= 0 && row < a.x_rows ? row : 0);
    };
    const int64_t n0 = static_cast<int64_t>(t.col) * TNO;
    auto weight = [&](int r) {
      if constexpr (GLU)  // 32 gate rows, then the 32 up rows of the same outputs
        return static_cast<int64_t>(t.e) * 2 * a.N + min(n0 + (r >> 6) * 32 + (r & 31), a.N - 1) +
               ((r >> 5) & 1) * a.N;
      else
        return static_cast<int64_t>(t.e) * a.N + min(n0 + r, a.N - 1);
    };
#pragma unroll
    for (int q = 0; q < H::LX; ++q) {
      const int r = row_of(q, 64 / XC), c = chunk_slot<XC>(r, lane % XC);
      px[q] = MX ? reinterpret_cast<const char*>(a.xcodes + token(r) * kb * 16 + c * 16)
                 : reinterpret_cast<const char*>(a.x + token(r) * a.ldx + c * 8);
    }
#pragma unroll
    for (int q = 0; q < H::LW; ++q) {
      const int r = row_of(q, 64 / WC), c = chunk_slot<WC>(r, lane % WC);
      pw[q] = reinterpret_cast<const char*>(a.codes + weight(r) * kb * 16 + c * 16);
    }
#pragma unroll
    for (int q = 0; q < H::LWS; ++q) {
      const int r = row_of(q, 64 / H::SC), c = scale_slot<H::SC>(r, lane % H::SC);
      pws[q] = reinterpret_cast<const char*>(a.scales + weight(r) * kb + c);
    }
    if constexpr (MX) {
#pragma unroll
      for (int q = 0; q < H::LXS; ++q) {
        const int r = row_of(q, 64 / H::SC), c = scale_slot<H::SC>(r, lane % H::SC);
        pxs[q] = reinterpret_cast<const char*>(a.xscales + token(r) * kb + c);
      }
    }
  };
  int step = 0, to = 0, ahead = 0;  // the next stage of the tile loaded, its buffer, and stages not yet multiplied
  auto issue = [&]() {
    const uint32_t s = lds0 + to * H::kStage;
    if (step == nk - 1 && last < H::KS) {  // lanes past K: zeros
      const char *zero = reinterpret_cast<const char*>(kPad), *one = zero + 16;
#pragma unroll
      for (int q = 0; q < H::LX; ++q)
        px[q] = chunk_slot<XC>(row_of(q, 64 / XC), lane % XC) * (MX ? 32 : 8) < last ? px[q] : zero;
#pragma unroll
      for (int q = 0; q < H::LW; ++q) pw[q] = chunk_slot<WC>(row_of(q, 64 / WC), lane % WC) * 32 < last ? pw[q] : zero;
#pragma unroll
      for (int q = 0; q < H::LWS; ++q)
        pws[q] = scale_slot<H::SC>(row_of(q, 64 / H::SC), lane % H::SC) * 32 < last ? pws[q] : one;
      if constexpr (MX) {
#pragma unroll
        for (int q = 0; q < H::LXS; ++q)
          pxs[q] = scale_slot<H::SC>(row_of(q, 64 / H::SC), lane % H::SC) * 32 < last ? pxs[q] : one;
      }
    }
#pragma unroll
    for (int q = 0; q < H::LX; ++q) {
      load_lds16(px[q], s + H::kX + (wave + kWaves * q) * 1024);
      px[q] += H::XB;
    }
#pragma unroll
    for (int q = 0; q < H::LW; ++q) {
      load_lds16(pw[q], s + H::kW + (wave + kWaves * q) * 1024);
      pw[q] += H::WB;
    }
#pragma unroll
    for (int q = 0; q < H::LWS; ++q) {
      load_lds1(pws[q], s + H::kWS + (wave + kWaves * q) * 256);
      pws[q] += H::SC;
    }
    if constexpr (MX) {
#pragma unroll
      for (int q = 0; q < H::LXS; ++q) {
        load_lds1(pxs[q], s + H::kXS + (wave + kWaves * q) * 256);
        pxs[q] += H::SC;
      }
    }
    ++step;
    ++ahead;
    to = to + 1 == H::kStages ? 0 : to + 1;
  };
  // Waits for all stages but the last `after` issued, and for the workgroup.
  auto landed = [&](int after) {
    if (H::kStages > 2 && after >= H::kStages - 1)
      wait_loads<(H::kStages - 1) * H::kLoads>();
    else if (after >= 1)
      wait_loads<H::kLoads>();
    else
      wait_loads<0>();
  };
  static_assert(H::kStages <= 3);

  int buf = 0;                    // of rowbuf: the tile multiplied; the next one's is buf + 1
  bool into_next = false;         // the loads have reached the next tile
  int since = 0;                  // steps since the next tile's rows were asked for
  auto find_next = [&]() {
    walk.l += walk.step;
    more = walk.find();
    if (more) {
      walk.get(&next);
      load_rows(next, buf == 2 ? 0 : buf + 1);
    }
    into_next = false;
    since = 0;
  };
  // Fills the ring as far as it goes.
  auto refill = [&]() {
    while (ahead < H::kStages) {
      if (step == nk) {
        if (!more || into_next) break;
        // the rows have landed if the stages asked for since then fill the ring
        if (a.rows && since < H::kStages) wait_loads<0>();
        aim(next, buf == 2 ? 0 : buf + 1);
        step = 0;
        into_next = true;
      }
      issue();
    }
    ++since;
  };

  load_rows(cur, 0);
  wait_loads<0>();
  aim(cur, 0);
  while (ahead < H::kStages && step < nk) issue();
  find_next();
  refill();

  const int wrow = wn * 64 + r32, xrow = wm * (TM / 2) + r32;
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
  Frags<MX, TM> p, q;
  landed(ahead - 1);
  const char* s = smem;
  p.template read<0>(s, wrow, xrow, half);
  for (;;) {
    for (int i = 0; i < nk; ++i) {
      q.template read<1>(s, wrow, xrow, half);
      __builtin_amdgcn_sched_barrier(0);
      p.multiply(acc);
      __builtin_amdgcn_sched_barrier(0);
      p.template read<2>(s, wrow, xrow, half);
      __builtin_amdgcn_sched_barrier(0);
      q.multiply(acc);
      __builtin_amdgcn_sched_barrier(0);
      q.template read<3>(s, wrow, xrow, half);
      __builtin_amdgcn_sched_barrier(0);
      p.multiply(acc);
      __builtin_amdgcn_sched_barrier(0);
      // the next stage has landed, and every wave has read all of this one: its buffer is free
      landed(ahead - 2);
      --ahead;
      refill();
      s = s + H::kStage == smem + H::kStages * H::kStage ? smem : s + H::kStage;
      p.template read<0>(s, wrow, xrow, half);  // (of the next tile after a tile's last step; unused at the end)
      __builtin_amdgcn_sched_barrier(0);
      q.multiply(acc);
      __builtin_amdgcn_sched_barrier(0);
    }
    const int64_t n0 = static_cast<int64_t>(cur.col) * TNO;
    const bool wide = a.ldy % 4 == 0;
#pragma unroll
    for (int m = 0; m < H::MB; ++m) {
      const int r = wm * (TM / 2) + 32 * m + r32;
      const int64_t slot = cur.lo + r;
      if (slot >= cur.hi) continue;
      bool have = true;
      if (a.rows) have = rowbuf[buf * TM + r] >= 0 && rowbuf[buf * TM + r] < a.x_rows;
#pragma unroll
      for (int n = 0; n < (GLU ? 1 : H::NB); ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[i] = acc[n][m][4 * e + i];
            if constexpr (GLU) v[i] = silu(v[i]) * acc[1][m][4 * e + i];
            v[i] = have ? v[i] : 0.0f;
          }
          const int64_t at = n0 + wn * (GLU ? 32 : 64) + 32 * n + 8 * e + 4 * half;
          if (at < a.N) store4(a, slot, at, a.N, wide, v);
        }
    }
    if (!more) return;
    cur = next;
    buf = buf == 2 ? 0 : buf + 1;
    clear();
    find_next();
    refill();
  }
}

// dx: 64 columns x 16 slots a workgroup, 16 columns a wave.  The weights' tile
// (32 rows x 64 columns) is widened to bf16 and transposed in LDS.
__global__ __launch_bounds__(kThreads) void mx4_grad_kernel(MulArgs a) {
  constexpr int KT = 64, LD = 40;  // (LD: rows 80 bytes apart)
  __shared__ __align__(16) uint16_t wt[KT * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 15, q = lane >> 4;
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((a.K + KT - 1) / KT), 16, &t)) return;
  const int64_t k0 = static_cast<int64_t>(t.col) * KT;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t slot = t.lo + r;
  if (t.e < a.E) {
    const int64_t kb = a.K / 32;
    const int wr = tid >> 3, wc = tid & 7;  // this thread's row and word of the tile
    for (int64_t n0 = 0; n0 < a.N; n0 += 32) {
      uint32_t w = 0;
      float scale = 1.0f;
      if (n0 + wr < a.N && k0 + 8 * wc < a.K) {
        const int64_t row = static_cast<int64_t>(t.e) * a.N + n0 + wr;
        w = *reinterpret_cast<const uint32_t*>(a.codes + row * kb * 16 + k0 / 2 + 4 * wc);
        scale = mx4_scale(a.scales[row * kb + (k0 + 8 * wc) / 32]);
      }
      const uint4 v4 = mx4_bf16_words(w, scale);
      const uint32_t v[4] = {v4.x, v4.y, v4.z, v4.w};
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 8; ++i) wt[(8 * wc + i) * LD + wr] = static_cast<uint16_t>(v[i / 2] >> (16 * (i & 1)));
      __syncthreads();
      uint4 xv = make_uint4(0, 0, 0, 0);
      const int64_t n = n0 + 8 * q;
      if (slot < t.hi && n < a.N) xv = *reinterpret_cast<const uint4*>(a.x + slot * a.ldx + n);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
          *reinterpret_cast<const bf16x8*>(&wt[(16 * wave + r) * LD + 8 * q]), __builtin_bit_cast(bf16x8, xv), acc,
          0, 0, 0);
    }
  }
  const int64_t k = k0 + 16 * wave + 4 * q;
  if (slot < t.hi && k < a.K) store4(a, slot, k, a.K, a.ldy % 4 == 0, acc);
}

// ---------------------------------------------------------------------------
// dx in large tiles: 128 slots x 256 columns a workgroup of eight waves, n
// advancing 64 rows of W a step.  The sum runs over W's rows, along which its
// scales change, so the codes of a step (64 rows x 256 columns, loaded as the
// forward form loads them) are widened to bf16 once by the whole workgroup, one
// block of 32 a thread, into an LDS tile that the transposing LDS read takes
// the fragments from.  Two such tiles: the next step is widened while this one
// is multiplied.
// ---------------------------------------------------------------------------
struct GradShape {
  static constexpr int TM = 128, KT = 256, NS = 64;  // slots, columns, rows of W a step
  static constexpr int kX = 0, kW = TM * NS * 2, kWS = kW + NS * KT / 2, kStage = kWS + NS * (KT / 32) * 4;
  static constexpr int kStages = 3;
  static constexpr int kTile = NS * KT * 2;
  static constexpr int kBytes = kStages * kStage + 2 * kTile;
  static constexpr int LX = 2, kLoads = LX + 2;
  static constexpr int MB = 2, NB = 2;
};
static_assert(GradShape::kBytes <= 163840);

typedef __attribute__((ext_vector_type(4))) short s16x4;
__device__ __forceinline__ s16x4 read_transposed(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(reinterpret_cast<uintptr_t>(p)));
}

__global__ __launch_bounds__(kTileThreads) void mx4_grad_tile_kernel(MulArgs a) {
  using H = GradShape;
  extern __shared__ __align__(16) char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((a.K + H::KT - 1) / H::KT), H::TM, &t)) return;
  const int64_t k0 = static_cast<int64_t>(t.col) * H::KT;
  const int wm = wave >> 2, wn = wave & 3, r32 = lane & 31, half = lane >> 5;
  f32x16 acc[H::NB][H::MB];
#pragma unroll
  for (int i = 0; i < H::NB; ++i)
#pragma unroll
    for (int j = 0; j < H::MB; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;

  if (t.e < a.E) {
    const int64_t kb = a.K / 32;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
    char* wide = smem + H::kStages * H::kStage;
    const char *px[H::LX], *pw, *ps;
    int nx[H::LX];
#pragma unroll
    for (int q = 0; q < H::LX; ++q) {
      const int r = (wave + kWaves * q) * 8 + lane / 8, c = chunk_slot<8>(r, lane % 8);
      nx[q] = 8 * c;
      px[q] = reinterpret_cast<const char*>(a.x + min(t.lo + r, t.hi - 1) * a.ldx + 8 * c);
    }
    // codes and scales of row wave * 8 + lane / 8 of a step, block lane % 8 of the tile
    const int wr = wave * 8 + lane / 8;
    const int64_t block = min(k0 / 32 + lane % 8, kb - 1);
    pw = reinterpret_cast<const char*>(a.codes + ((static_cast<int64_t>(t.e) * a.N + wr) * kb + block) * 16);
    ps = reinterpret_cast<const char*>(a.scales + (static_cast<int64_t>(t.e) * a.N + wr) * kb + block);
    const int64_t wstep = H::NS * kb * 16, sstep = H::NS * kb;
    const int nk = static_cast<int>((a.N + H::NS - 1) / H::NS);
    const int last = static_cast<int>(a.N - static_cast<int64_t>(nk - 1) * H::NS);
    int issued = 0, to = 0;
    auto issue = [&]() {
      const uint32_t s = lds0 + to * H::kStage;
      if (issued == nk - 1 && last < H::NS) {
#pragma unroll
        for (int q = 0; q < H::LX; ++q) px[q] = nx[q] < last ? px[q] : reinterpret_cast<const char*>(kPad);
        pw = wr < last ? pw : reinterpret_cast<const char*>(kPad);
        ps = wr < last ? ps : reinterpret_cast<const char*>(kPad + 16);
      }
#pragma unroll
      for (int q = 0; q < H::LX; ++q) {
        load_lds16(px[q], s + H::kX + (wave + kWaves * q) * 1024);
        px[q] += H::NS * 2;
      }
      load_lds16(pw, s + H::kW + wave * 1024);
      load_lds1(ps, s + H::kWS + wave * 256);
      pw += wstep;
      ps += sstep;
      ++issued;
      to = to + 1 == H::kStages ? 0 : to + 1;
    };
    // this thread's block of stage `s`, widened into row wr of tile `w`
    auto widen = [&](const char* s, char* w) {
      const uint4 c = *reinterpret_cast<const uint4*>(s + H::kW + tid * 16);
      const float scale = mx4_scale(*reinterpret_cast<const uint32_t*>(s + H::kWS + tid * 4));
      const uint32_t d[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)  // 16-byte chunk 4 (lane % 8) + i of the row
        *reinterpret_cast<uint4*>(w + wr * (H::KT * 2) + ((4 * (lane % 8) + i) ^ (4 * (wr & 3))) * 16) =
            mx4_bf16_words(d[i], scale);
    };
    for (int i = 0; i < H::kStages - 1 && i < nk; ++i) issue();
    if (issued > 1)
      wait_loads<H::kLoads>();
    else
      wait_loads<0>();
    widen(smem, wide);
    const int xrow = wm * (H::TM / 2) + r32;
    int from = 0;
    for (int i = 0; i < nk; ++i) {
      // step i + 1 has landed, step i is widened, and every wave is past step i - 1
      wait_loads<0>();
      if (issued < nk) issue();
      const char* s = smem + from * H::kStage;
      from = from + 1 == H::kStages ? 0 : from + 1;
      if (i + 1 < nk) widen(smem + from * H::kStage, wide + ((i + 1) & 1) * H::kTile);
      const char* w = wide + (i & 1) * H::kTile;
#pragma unroll
      for (int j = 0; j < 4; ++j) {  // 16 rows of W
        bf16x8 xf[H::MB];
#pragma unroll
        for (int m = 0; m < H::MB; ++m) {
          const int r = xrow + 32 * m;
          xf[m] = *reinterpret_cast<const bf16x8*>(s + H::kX + r * (H::NS * 2) + chunk_slot<8>(r, 2 * j + half) * 16);
        }
#pragma unroll
        for (int n = 0; n < H::NB; ++n) {
          // rows 16 j + 8 half + 4 q + (lane % 16) / 4, column 16 ((lane / 16) % 2) + 4 (lane % 4) of the block
          const int col = wn * 64 + 32 * n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
          s16x4 h[2];
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const int r = 16 * j + 8 * half + 4 * q + ((lane & 15) >> 2);
            h[q] = read_transposed(w + r * (H::KT * 2) + (((col >> 3) ^ (4 * (r & 3))) << 4) + (col & 7) * 2);
          }
          const bf16x8 wf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int m = 0; m < H::MB; ++m)
            acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf, xf[m], acc[n][m], 0, 0, 0);
        }
      }
    }
  }
  const bool aligned = a.ldy % 4 == 0;
#pragma unroll
  for (int m = 0; m < H::MB; ++m) {
    const int64_t slot = t.lo + wm * (H::TM / 2) + 32 * m + r32;
    if (slot >= t.hi) continue;
#pragma unroll
    for (int n = 0; n < H::NB; ++n)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = acc[n][m][4 * q + i];
        const int64_t at = k0 + wn * 64 + 32 * n + 8 * q + 4 * half;
        if (at < a.K) store4(a, slot, at, a.K, aligned, v);
      }
  }
}

bitsmoe_status check(const char* who, const MulArgs& a, bitsmoe_dtype yt, int64_t wide) {
  const std::string w(who);
  if (a.E <= 0 || a.N <= 0 || a.K <= 0 || a.S < 0 || a.x_rows < 0)
    return fail(BITSMOE_ERR_ARG, w + ": non-positive size");
  if (yt != BITSMOE_F32 && yt != BITSMOE_BF16) return fail(BITSMOE_ERR_DTYPE, w + ": results are fp32 or bf16");
  if (a.K % kMx4Block != 0 || a.K > (1 << 24) || a.N > (1 << 24) || a.E > 65535 || a.S > 0x7FFFFFF0 ||
      a.x_rows > 0x7FFFFFFF)
    return fail(BITSMOE_ERR_SHAPE, w + ": needs K % 32 == 0, K and N <= 2^24, E <= 65535, S and rows < 2^31");
  if (a.ldy < wide || a.ldy > (int64_t(1) << 32))
    return fail(BITSMOE_ERR_SHAPE, w + ": the results' row stride is too small or too large");
  if (!a.offsets && a.E != 1) return fail(BITSMOE_ERR_ARG, w + ": no offsets, and more than one expert");
  if (a.S > 0 && (!a.codes || !a.scales || !a.y)) return fail(BITSMOE_ERR_ARG, w + ": null pointer");
  if (!a.rows && a.x_rows < a.S) return fail(BITSMOE_ERR_SHAPE, w + ": fewer rows than slots");
  if (!aligned16({a.codes, a.scales, a.x, a.xcodes, a.xscales, a.offsets, a.rows, a.y}))
    return fail(BITSMOE_ERR_ARG, w + ": device pointers must be 16-byte aligned");
  return BITSMOE_OK;
}

// Workgroups for tiles of `tile` slots and `per` workgroups each.
bool grid_of(const MulArgs& a, int64_t tile, int64_t per, unsigned* grid) {
  const int64_t tiles = a.S / tile + (a.E + 1 < a.S ? a.E + 1 : a.S);
  if (tiles > ((int64_t(1) << 24) - 1) / per) return false;
  *grid = static_cast<unsigned>(tiles * per);
  return true;
}

// Large tiles pay from about this many slots an expert on.
constexpr int64_t kTileSlots = 32;

template <bool MX, bool GLU, int TM>
bitsmoe_status tile_product(const char* who, const MulArgs& a, hipStream_t s) {
  using H = Shape<MX, TM>;
  constexpr int TNO = GLU ? kTN / 2 : kTN;
  unsigned grid;
  if (!grid_of(a, TM, (a.N + TNO - 1) / TNO, &grid))
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": too many slots and outputs for one call");
  grid = static_cast<unsigned>(device_cus());  // one workgroup a compute unit, a multiple of the XCDs
  grid = grid < 8 ? 8 : grid / 8 * 8;
  constexpr int lds = H::kStages * H::kStage + 3 * TM * 4;
  static_assert(lds <= 163840);
  auto* fn = mx4_tile_kernel<MX, GLU, TM>;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(fn),
                                           hipFuncAttributeMaxDynamicSharedMemorySize, lds);
  if (e != hipSuccess) return device_error("mx4_product: shared memory", e);
  fn<<<grid, kTileThreads, lds, s>>>(a);
  BITSMOE_LAUNCH_CHECK("mx4_tile_kernel");
  return ok();
}

bitsmoe_status product(const char* who, const MulArgs& a, bool glu, hipStream_t s) {
  const bool mx = a.xcodes != nullptr;
  if (a.S >= kTileSlots * a.E && a.x_rows > 0) {
    if (mx) return glu ? tile_product<true, true, 128>(who, a, s) : tile_product<true, false, 128>(who, a, s);
    return glu ? tile_product<false, true, 128>(who, a, s) : tile_product<false, false, 128>(who, a, s);
  }
  unsigned grid;
  if (!grid_of(a, 16, (a.N + 15) / 16, &grid))
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": too many slots and outputs for one call");
  auto* fn = mx ? (glu ? mx4_rows_kernel<true, true> : mx4_rows_kernel<true, false>)
                : (glu ? mx4_rows_kernel<false, true> : mx4_rows_kernel<false, false>);
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
  return product("mx4_product", a, glu != 0, static_cast<hipStream_t>(stream));
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
  if (!xcodes_dev || !xscales_dev) return fail(BITSMOE_ERR_ARG, "mx4_product_q: null pointer");
  return product("mx4_product_q", a, glu != 0, static_cast<hipStream_t>(stream));
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
  unsigned grid;
  if (S >= kTileSlots * E) {
    if (!grid_of(a, GradShape::TM, (K + GradShape::KT - 1) / GradShape::KT, &grid))
      return fail(BITSMOE_ERR_SHAPE, "mx4_product_grad: too many slots and columns for one call");
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(mx4_grad_tile_kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, GradShape::kBytes);
    if (e != hipSuccess) return device_error("mx4_product_grad: shared memory", e);
    mx4_grad_tile_kernel<<<grid, kTileThreads, GradShape::kBytes, static_cast<hipStream_t>(stream)>>>(a);
    BITSMOE_LAUNCH_CHECK("mx4_grad_tile_kernel");
    return ok();
  }
  if (!grid_of(a, 16, (K + 63) / 64, &grid))
    return fail(BITSMOE_ERR_SHAPE, "mx4_product_grad: too many slots and columns for one call");
  mx4_grad_kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  BITSMOE_LAUNCH_CHECK("mx4_grad_kernel");
  return ok();
}
