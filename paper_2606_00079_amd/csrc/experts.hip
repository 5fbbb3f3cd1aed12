// Products of tokens in expert order with bf16 expert weights.
//
//     y_s = W_e(s) x_row(s)                            (expert_product)
//     y_s = silu(g) u, [g; u] = W_e(s) x_row(s)        (the same with glu)
//     dx_s = W_e(s)^T dy_s                             (expert_product_grad)
//     dW_e = sum over e's slots of dy_s x_row(s)^T     (expert_weight_grad; _q: x in MX8)
//
// for S slots, expert e's being offsets[e] .. offsets[e+1].  Sums are fp32 and
// results are rounded once; with glu silu(g) u is taken of the fp32 sums.
//
// Few slots an expert: bound by the weights' bytes (every byte of W is used S / E times);
// many: by the matrix cores, whose clock gives way under real data (8192^3 by the
// library 1.53 to 1.61 PFLOP/s).  Between the two lie a factor of about 320 slots an expert.
#include <atomic>
#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include "internal.hpp"
#include "mx8.hpp"
#include "rows.hpp"
#include "slot_range.hpp"
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
  int parts;  // (weights' gradient) the sum is cut into, each with results of its own in y
};

enum Form { kForward, kTokens, kWeights };

// 16 outputs x 16 slots a workgroup.  Its eight waves share out K in segments of
// 64 entries, a cache line of a row: lane l holds chunks l / 16 and 4 + l / 16 of row
// l % 16, and of slot l % 16.  For the fewest slots: bound by launch and one chain of
// loads, so the sum is split and the workgroups are small and many (8 slots of 128
// experts, 1536 x 2048: 11.8 us, 50 MB at 4.3 TB/s; 2 slots of 8 experts, 1024 x 4096: 7.6 us,
// where the large tiles below take 30 to 72).  More slots an expert read the
// weights again for every 16, which tiles do for every 32 to 256.
constexpr int kRowWaves = 8;
template <bool GLU>
__global__ __launch_bounds__(64 * kRowWaves) void expert_rows_kernel(ExpertArgs a) {
  constexpr int H = GLU ? 2 : 1, AHEAD = 4;
  __shared__ f32x4 part[kRowWaves][H][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, q = lane >> 4;
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, static_cast<int>((a.N + 15) / 16), 16, &t)) return;
  const int64_t n0 = static_cast<int64_t>(t.col) * 16;
  f32x4 acc[H];
#pragma unroll
  for (int h = 0; h < H; ++h) acc[h] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  bool have = false;  // the row of this lane's slot exists
  if (t.e < a.E) {
    const int64_t slot = t.lo + r;
    const int64_t row = slot < t.hi ? (a.rows ? static_cast<int64_t>(a.rows[slot]) : slot) : -1;
    have = row >= 0 && row < a.x_rows;
    const uint16_t* w[H];
#pragma unroll
    for (int h = 0; h < H; ++h)
      w[h] = a.w + ((static_cast<int64_t>(t.e) * H + h) * a.N + min(n0 + r, a.N - 1)) * a.K;
    const uint16_t* x = a.x + row * a.ldx;
    const int segments = static_cast<int>((a.K + 63) / 64);
    for (int s0 = wave; s0 < segments; s0 += kRowWaves * AHEAD) {
      uint4 wv[AHEAD][H][2], xv[AHEAD][2];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const int64_t k = static_cast<int64_t>(s0 + u * kRowWaves) * 64 + 32 * c + 8 * q;
          const bool in = k < a.K;
#pragma unroll
          for (int h = 0; h < H; ++h)
            wv[u][h][c] = in ? *reinterpret_cast<const uint4*>(w[h] + k) : make_uint4(0, 0, 0, 0);
          xv[u][c] = in && have ? *reinterpret_cast<const uint4*>(x + k) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int h = 0; h < H; ++h)
            acc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, wv[u][h][c]),
                                                             __builtin_bit_cast(bf16x8, xv[u][c]), acc[h], 0, 0, 0);
    }
  }
#pragma unroll
  for (int h = 0; h < H; ++h) part[wave][h][lane] = acc[h];
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 1; i < kRowWaves; ++i) acc[h] += part[i][h][lane];
  if constexpr (GLU) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[0][i] = silu(acc[0][i]) * acc[1][i];
  }
  if (!have) acc[0] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};  // (zeros times weights that are no numbers are NaN)
  const int64_t slot = t.lo + r, n = n0 + 4 * q;      // (a lane holds four outputs of one slot)
  if (slot < t.hi && n < a.N) store4(a, slot, n, a.N, a.ldy % 4 == 0, acc[0]);
}

// ---------------------------------------------------------------------------
// Tiles: MT x 256 results a workgroup, which stays and takes tile after tile.
//
// Two operands go into a matrix-core op: Q, whose 256 rows are results that lie
// side by side in memory, on its row side, so that a lane holds runs of four of
// them; and P, the MT others (slots; for the weights' gradient outputs).  Either
// comes as its rows' entries of the sum lie, or, where the sum runs over the rows
// of a matrix (W for the tokens' gradient, dy and x for the weights'), as those rows
// do, and is then read through the transposing LDS read.
//
// Direct global->LDS loads fill a ring of stages of 64 entries of the sum, whole
// cache lines of 128 bytes; a step that finds its stage read by every wave refills
// it at once, across the end of a tile too.
//
// 256 x 256 results take 8 waves of 64 x 128, two a SIMD: each fragment of 16 entries
// that is read feeds two or four ops (a step of 64 entries: 32 ops a wave, beside
// 24 KB read and 8 KB loaded by it).  Four waves of 128 x 128 read a third less but
// stood still at every wait, and were slower.  What there is of branches around the
// ops costs most: without any 8192^3 went from 939 to 827 us (1.33 PFLOP/s; the library
// 682 to 718 us with the sum along both operands' rows), W^T dy to 832 (785 to 845); dy x^T takes 938 to 957 (900
// to 980).  32 and 128 slots a tile are for experts with fewer (512 slots of 128 experts,
// 2048 x 768: 71 us in tiles of 32 slots, 403 MB at 5.7 TB/s; 74 and 93 in larger ones).
//
// Tokens in MX8 (the weights' gradient) are widened to bf16 on their way: every
// wave loads the codes of eight slots of a stage for itself, and in the step before
// that stage's writes what they stand for into one of two tiles, between the ops
// (8192^3: 1202 us, where bf16 tokens take 946; 128 experts of 1536 x 2048, 32768 slots 403 and 343).
// An entry is widened again for every tile that reads it, so what this spares who kept MX8 is the 2 bytes an entry
// that widened tokens would take, not time: mx8_dequantize and the bf16 form after it take 967 and 348 us there.
//
// The weights' gradient has short sums and much to write (there 256 entries and 805 MB of
// results a call): it is bound by that writing, which does not overlap with the next tile's
// ops, as loads and stores of a wave are waited for in their order.  (Two workgroups of 128 x 256 results a compute
// unit with stages of 32 entries overlap them, but go through a sum a third slower: 470 us, 8192^3 1367.)
// ---------------------------------------------------------------------------
template <Form FORM, int MT_, bool MX = false>
struct Shape {
  static constexpr int MT = MT_, QT = 256, KS = 64;
  static constexpr int WM = MT == 32 ? 1 : 2, WN = 4, kWaves = WM * WN, kThreads = 64 * kWaves;
  static constexpr int MB = MT / WM / 32, NB = 2;
  static constexpr bool kPCols = FORM == kWeights, kQCols = FORM != kForward;  // operands whose sum runs over rows
  static constexpr int kPStage = MT * KS * 2, kQStage = QT * KS * 2, kStage = kPStage + (MX ? 0 : kQStage);
  static constexpr int NX = MT == 32 ? 4 : MT == 128 ? 3 : 2;
  static constexpr int kRows = MT < 64 ? 64 : MT;  // of a buffer of row numbers
  static constexpr int oRows = NX * kStage;  // (the ring's end)
  // MX8: two widened tiles, then a wave's codes and its scales, a word each
  static constexpr int oTiles = oRows, oCodes = oTiles + 2 * kQStage, kCodes = 8 * QT, oScales = oCodes + kWaves * kCodes;
  // weights: lists of the rows of a wave's eight slots of eight stages: the first of three tiles, two others
  static constexpr int oLists = MX ? oScales + kWaves * 8 * (QT / 32) * 4 : oRows, kLists = 5;
  // where a wave turns its results into whole rows of its columns (with MX8 its own rows of a widened tile)
  static constexpr int oTurn = oLists + (FORM == kForward ? 3 * kRows * 4 : FORM == kWeights ? kWaves * kLists * 256 : 0);
  static constexpr bool kTurn = MT == 256;
  static constexpr bool kShort = FORM != kWeights && MT >= 128;
  static constexpr int kBytes = oTurn + (kTurn && !MX ? kWaves * 2048 : 0);
  static_assert(kBytes <= 163840);
  static_assert(FORM != kWeights || (MT == 256 && NX == 2));

  static constexpr int LP = kPStage / 1024 / kWaves, LQ = MX ? 0 : kQStage / 1024 / kWaves, kLoads = LP + LQ;
  // Loads 0 .. kFirst, .. kSecond and .. kLoads of a stage go out in the third and fourth part of the step that frees
  // its place and in the first of the next.
  static constexpr int kFirst = (kLoads + 2) / 3, kSecond = kFirst + (kLoads + 1) / 3;
};

// What lanes past an end read.
__device__ const uint8_t kZeros[16] __attribute__((aligned(16))) = {};
__device__ const uint8_t kOne[4] = {127, 127, 127, 127};  // (scales)
__device__ const int32_t kNoRow = -1;

// A tile: the slots lo .. hi of expert e, and its first results.
struct ResultTile {
  int e, lo, hi, m0, n0, part;
};

template <Form FORM, int MT, bool GLU, bool MX>
__global__ __launch_bounds__(MT == 32 ? 256 : 512, MT == 32 ? 1 : 2) void expert_tile_kernel(ExpertArgs a) {
  using H = Shape<FORM, MT, MX>;
  extern __shared__ __align__(16) char smem[];
  int32_t* const rowbuf = reinterpret_cast<int32_t*>(smem + H::oRows);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  constexpr int QTO = GLU ? H::QT / 2 : H::QT;  // results a tile has in a row
  const int wm = wave / H::WN, wn = wave % H::WN, r32 = lane & 31, half = lane >> 5;
  const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem));
  const char* const zero = reinterpret_cast<const char*>(kZeros);
  const int N = static_cast<int>(a.N), K = static_cast<int>(a.K);
  const int width = FORM == kForward ? N : K;  // of a row of results

  // ---- which tiles
  Walk walk;
  ResultTile cur, next;
  int64_t l = 0, end = 0, step_l = 0;  // (weights)
  int more;
  // (weights) a tile is the `in`th of expert e's; 64-bit divisions for every tile would take as long as one of its steps
  const uint32_t kt = static_cast<uint32_t>((a.K + H::QT - 1) / H::QT), nt = static_cast<uint32_t>((a.N + MT - 1) / MT);
  const uint32_t per = nt * kt * static_cast<uint32_t>(a.parts);  // (below 2^31)
  int at_e = 0;
  uint32_t at_in = 0;
  auto weight_tile = [&](ResultTile* t) __attribute__((always_inline)) {
    const int e = at_e;
    uint32_t in = at_in;
    int part = 0;
    if (a.parts > 1) {
      part = static_cast<int>(in % a.parts);
      in /= a.parts;
    }
    const auto* off = (const __attribute__((address_space(4))) int32_t*)reinterpret_cast<uintptr_t>(a.offsets);
    const int S = static_cast<int>(a.S);
    t->e = e;
    t->lo = off ? min(max(off[e], 0), S) : 0;
    t->hi = off ? min(max(off[e + 1], t->lo), S) : S;
    if (a.parts > 1) take_part(&t->lo, &t->hi, part, a.parts, H::KS);
    t->part = part;
    // In groups of up to eight rows of tiles, column by column, so that what an XCD works on at a time shares both
    // operands (128 experts of 1536 x 2048, 32768 slots: 395 us row by row, 397, 382, 372 and 372 in groups of 2, 4, 8
    // and 16 rows; 8192^3 1011, 982, 967, 957 and 975).
    const uint32_t group = in / (8 * kt), rest = in - group * 8 * kt, high = min(8u, nt - 8 * group), col = rest / high;
    t->m0 = static_cast<int>(8 * group + rest - col * high) * MT;
    t->n0 = static_cast<int>(col) * H::QT;
  };
  auto slot_tile = [&](ResultTile* t) __attribute__((always_inline)) {
    Tile s;
    walk.get(&s);
    t->e = s.e;
    t->lo = s.lo;
    t->hi = s.hi;
    t->m0 = s.lo;
    t->n0 = s.col * QTO;
  };
  ResultTile later;  // (weights) the one after next
  auto find_later = [&]() __attribute__((always_inline)) {
    at_in += static_cast<uint32_t>(step_l);
    while (at_in >= per) {
      at_in -= per;
      ++at_e;
    }
    weight_tile(&later);
  };
  if constexpr (FORM == kWeights) {
    // Each XCD gets an eighth of the work: an expert's tiles cost its steps, and the writing of results about as much as
    // four steps (fp32: eight).
    const int runs = (a.E + 63) / 64;  // experts a lane
    auto cost = [&](int e) __attribute__((always_inline)) {
      int lo;
      const int count = slots_of(a.offsets, a.E, static_cast<int>(a.S), e, &lo);
      return ((count + H::KS - 1) / H::KS + a.parts - 1) / a.parts + (a.yf32 ? 8 : 4);
    };
    int own = 0;
    for (int i = 0; i < runs; ++i)
      if (lane * runs + i < a.E) own += cost(lane * runs + i);
    const int sum = wave_scan(own);
    const int64_t total = static_cast<int64_t>(lane_value(sum, 63)) * per;
    auto border = [&](int x) __attribute__((always_inline)) {  // first tile whose cost begins at x eighths or after
      const int64_t target = total * x / 8;
      const uint64_t past = __ballot(static_cast<int64_t>(sum) * per > target);
      if (!past) return static_cast<int64_t>(a.E) * per;
      const int run = __builtin_ctzll(past);
      int e = run * runs, c = cost(e);
      int64_t before = static_cast<int64_t>(lane_value(sum, run) - lane_value(own, run)) * per;
      while (before + static_cast<int64_t>(c) * per <= target) {
        before += static_cast<int64_t>(c) * per;
        c = cost(++e);
      }
      return static_cast<int64_t>(e) * per + (target - before + c - 1) / c;
    };
    l = border(blockIdx.x & 7);
    end = border((blockIdx.x & 7) + 1);
    step_l = gridDim.x >> 3;
    l += blockIdx.x >> 3;
    more = l < end;
    at_e = static_cast<int>(l / per);
    at_in = static_cast<uint32_t>(l - static_cast<int64_t>(at_e) * per);
  } else {
    int head, none;
    more = walk.start(a.offsets, a.E, a.S, static_cast<int>((width + QTO - 1) / QTO), MT, &head, &none);
    // slots of no expert: zeros
    for (int64_t i = blockIdx.x; i < head + (a.S - none); i += gridDim.x) {
      const int64_t s = i < head ? i : none + (i - head);
      for (int64_t n = tid; n < width; n += H::kThreads) {
        if (a.yf32)
          static_cast<float*>(a.y)[s * a.ldy + n] = 0.0f;
        else
          static_cast<uint16_t*>(a.y)[s * a.ldy + n] = 0;
      }
    }
  }
  if (!more) return;
  if constexpr (FORM == kWeights) {
    weight_tile(&cur);
    if (l + step_l < end) find_later();
  } else {
    slot_tile(&cur);
  }
  // (NX at least, so that the ring never reaches past the next tile)
  auto steps_of = [&](const ResultTile& t) __attribute__((always_inline)) {
    const int L = FORM == kForward ? K : FORM == kTokens ? N : t.hi - t.lo;
    return max((L + H::KS - 1) / H::KS, H::NX);
  };

  // ---- where the loads come from
  const char *pp[H::LP], *pq[H::LQ ? H::LQ : 1];
  // operands by rows: 8 lanes a row; row of load q, and the chunk of it that goes to this lane's place
  // (the chunk is the same for all of them, as every wave's rows are eight of 32 or 64 apart)
  auto row_of = [&](int q, int l) __attribute__((always_inline)) { return (wave + H::kWaves * q) * 8 + l / 8; };
  const int chunk = chunk_slot(row_of(0, lane), lane & 7);
  // the rows of a tile's slots (past its end: its last)
  auto load_rows = [&](const ResultTile& t, int buf) __attribute__((always_inline)) {
    if constexpr (FORM == kForward)
      if (a.rows && wave < H::kRows / 64)
        load_lds4(a.rows + min(t.lo + wave * 64 + lane, t.hi - 1), lds0 + H::oRows + (buf * H::kRows + wave * 64) * 4);
  };
  const char* px[2];  // weights: x at this lane's columns, for even and odd loads
  auto aim = [&](const ResultTile& t, int buf) __attribute__((always_inline)) {
    const int lane = opaque(tid) & 63, r32 = lane & 31, half = lane >> 5;  // (not kept in registers between the tiles)
    if constexpr (FORM == kWeights) {  // two slots a load, 32 chunks each (columns past the end: the last ones)
      auto col = [&](int first, int q, int end) __attribute__((always_inline)) {
        return min(first + 8 * (r32 ^ (4 * ((2 * q + half) & 3))), end - 8);
      };
#pragma unroll
      for (int q = 0; q < H::LP; ++q)
        pp[q] = reinterpret_cast<const char*>(
            a.dy + (static_cast<int64_t>(t.lo) + wave * 8 + 2 * q + half) * a.lddy + col(t.m0, q, N));
#pragma unroll
      for (int q = 0; q < 2; ++q) px[q] = reinterpret_cast<const char*>(a.x + col(t.n0, q, K));
    } else {
#pragma unroll
      for (int q = 0; q < H::LP; ++q) {
        const int r = row_of(q, lane), c = chunk_slot(r, lane & 7);
        if constexpr (FORM == kForward) {
          int64_t row = min(t.lo + r, t.hi - 1);
          if (a.rows) {  // (one that does not exist: row 0, its results are replaced)
            row = rowbuf[buf * H::kRows + r];
            row = row >= 0 && row < a.x_rows ? row : 0;
          }
          pp[q] = reinterpret_cast<const char*>(a.x + row * a.ldx + c * 8);
        } else {
          pp[q] = reinterpret_cast<const char*>(a.dy + static_cast<int64_t>(min(t.lo + r, t.hi - 1)) * a.lddy + c * 8);
        }
      }
#pragma unroll
      for (int q = 0; q < H::LQ; ++q) {
        if constexpr (FORM == kForward) {
          const int r = row_of(q, lane), c = chunk_slot(r, lane & 7);
          int64_t row;
          if constexpr (GLU)  // 32 gate rows, then the 32 up rows of the same outputs
            row = static_cast<int64_t>(t.e) * 2 * a.N + min(t.n0 + (r >> 6) * 32 + (r & 31), N - 1) +
                  ((r >> 5) & 1) * a.N;
          else
            row = static_cast<int64_t>(t.e) * a.N + min(t.n0 + r, N - 1);
          pq[q] = reinterpret_cast<const char*>(a.w + row * a.K + c * 8);
        } else {  // two rows of W a load, 32 chunks each
          const int r = (wave + H::kWaves * q) * 2 + half;
          const int col = min(t.n0 + 8 * (r32 ^ (4 * (r & 3))), K - 8);
          pq[q] = reinterpret_cast<const char*>(a.w + (static_cast<int64_t>(t.e) * a.N + r) * a.K + col);
        }
      }
    }
  };

  // ---- the loads of the next stage
  int step = 0, to = 0, steps_to = 0;  // of the tile being loaded: its next step, ring place, steps
  ResultTile ld;                       // that tile
  // weights: the rows of slots come through LDS, asked for eight stages at once and long before
  int row[4] = {};  // of this lane's slots in the stage being loaded; negative: none
  int head = 0;     // list of the first stages of the tile being loaded
  auto list_at = [&](int at) __attribute__((always_inline)) { return H::oLists + (wave * H::kLists + at) * 256; };
  auto ask_rows = [&](const ResultTile& t, int chunk, int at) __attribute__((always_inline)) {
    const int lane = opaque(tid) & 63;
    const int s = slot_ahead(t.lo, t.hi, static_cast<unsigned>(chunk * 8 + lane / 8) * H::KS + wave * 8 + lane % 8);
    load_lds4(s >= 0 ? a.rows + s : &kNoRow, lds0 + list_at(at));
  };
  auto row_of_slot = [&](int slot) __attribute__((always_inline)) {  // (of this wave's eight)
    const int s = ld.lo + step * H::KS + wave * 8 + slot;
    const int list = step < 8 ? head : 3 + (step >> 3 & 1);
    const int r = a.rows ? *reinterpret_cast<const int*>(smem + list_at(list) + (step & 7) * 32 + slot * 4)
                         : s < ld.hi ? s : -1;
    return r < a.x_rows ? r : -1;
  };
  auto take_rows = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) row[q] = row_of_slot(2 * q + half);
  };
  auto load = [&](int k) __attribute__((always_inline)) {  // load k of the stage's LP + LQ
    const uint32_t base = lds0 + to * H::kStage;
    const bool of_p = k < H::LP;
    const int q = of_p ? k : k - H::LP;
    if constexpr (FORM == kWeights) {
      const int r = row[q];
      if (of_p) {
        load_lds16(r >= 0 ? pp[q] : zero, base + (wave * H::LP + q) * 1024);
        pp[q] += a.lddy * (H::KS * 2);
      } else {
        load_lds16(r >= 0 ? px[q & 1] + static_cast<uint64_t>(static_cast<uint32_t>(r)) * static_cast<uint32_t>(2 * a.ldx)
                          : zero,
                   base + H::kPStage + (wave * H::LQ + q) * 1024);
      }
    } else {
      load_lds16(of_p ? pp[q] : pq[q], base + (of_p ? 0 : H::kPStage) + (wave + H::kWaves * q) * 1024);
      if (of_p)
        pp[q] += H::KS * 2;
      else
        pq[q] += FORM == kForward ? H::KS * 2 : H::KS * 2 * a.K;
    }
  };
  // Before the loads of a stage in which the sum ends, or past its end: zeros from there on.
  auto cut = [&](int rem) __attribute__((always_inline)) {
    if (FORM == kWeights || rem >= H::KS) return;
#pragma unroll
    for (int q = 0; q < H::LP; ++q) pp[q] = 8 * chunk < rem ? pp[q] : zero;
#pragma unroll
    for (int q = 0; q < H::LQ; ++q)
      pq[q] = (FORM == kForward ? 8 * chunk : (wave + H::kWaves * q) * 2 + half) < rem ? pq[q] : zero;
  };
  auto entries_left = [&]() __attribute__((always_inline)) { return (FORM == kForward ? K : N) - step * H::KS; };
  auto loaded = [&]() __attribute__((always_inline)) {
    ++step;
    to = to + 1 == H::NX ? 0 : to + 1;
  };
  auto issue = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < H::kLoads; ++k) load(k);
    loaded();
  };
  // MX8: this wave's codes of the next stage, four slots of 256 bytes a load, and their scales, a lane slot lane / 8's
  // block lane % 8
  auto issue_codes = [&]() __attribute__((always_inline)) {
    const int lane = opaque(tid) & 63;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int r = row_of_slot(4 * q + lane / 16), col = min(ld.n0 + 16 * (lane % 16), K - 16);
      const uint8_t* p = a.xcodes + static_cast<int64_t>(r) * a.K + col;
      load_lds16(r >= 0 ? reinterpret_cast<const char*>(p) : zero, lds0 + H::oCodes + wave * H::kCodes + q * 1024);
    }
    const int r = row_of_slot(lane / 8), block = min(ld.n0 / 32 + lane % 8, K / 32 - 1);
    const uint8_t* p = a.xscales + static_cast<int64_t>(r) * (a.K / 32) + block;
    load_lds1(r >= 0 ? p : kOne, lds0 + H::oScales + wave * 256);
  };
  auto widen = [&](int i, int tile) __attribute__((always_inline)) {  // entries 8 i .. 8 i + 7 of this lane's block
    const int lane = opaque(tid) & 63;
    const uint2 c = *reinterpret_cast<const uint2*>(smem + H::oCodes + wave * H::kCodes + lane * 32 + i * 8);
    const float scale = mx4_scale(*reinterpret_cast<const uint32_t*>(smem + H::oScales + wave * 256 + lane * 4));
    const int slot = wave * 8 + lane / 8, at = 4 * (lane % 8) + i;
    *reinterpret_cast<uint4*>(smem + H::oTiles + tile * H::kQStage + slot * (H::QT * 2) + ((at ^ (4 * (slot & 3))) << 4)) =
        make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.x, scale, true)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, scale, false)),
                   __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.y, scale, true)));
  };
  // until at most N of this wave's loads are under way: its own codes are there (no other wave reads them)
  auto wait_own = [](auto n) { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(n)::value) : "memory"); };

  // ---- going on into the next tile
  int buf = 0, since = 0;
  int dry = 0;
  auto after = [&](int b) __attribute__((always_inline)) { return b == 2 ? 0 : b + 1; };
  auto find_next = [&]() __attribute__((always_inline)) {
    if constexpr (FORM == kWeights) {
      l += step_l;
      more = l < end;
    } else {
      walk.l += walk.step;
      more = walk.find();
    }
    if (more) {
      if constexpr (FORM == kWeights) {
        next = later;
        if (l + step_l < end) {
          find_later();
          if (a.rows) ask_rows(later, 0, after(after(head)));
        }
      } else {
        slot_tile(&next);
        load_rows(next, after(buf));
      }
    }
    since = 0;
  };
  auto turn = [&]() __attribute__((always_inline)) {  // to the next tile if the loads are through with theirs
    const int over = step == steps_to;
    dry |= over && !more;
    if (dry) {  // (zeros: so waits go by count to the end)
      if constexpr (FORM == kWeights) {
#pragma unroll
        for (int q = 0; q < 4; ++q) row[q] = -1;
      }
      cut(0);
      return;
    }
    if (over) {
      // (the next tile's rows have landed if as many steps as the ring has stages waited since they were asked for)
      if (FORM == kForward && a.rows && since < H::NX) wait_loads<0>();
      aim(next, after(buf));
      steps_to = steps_of(next);
      step = 0;
      ld = next;
      head = after(head);
    }
    cut(entries_left());
    if constexpr (FORM == kWeights) {
      take_rows();
      // (entering a list: the one after it)
      if (a.rows && (step & 7) == 0 && step + 8 < steps_to) ask_rows(ld, step / 8 + 1, 3 + ((step >> 3) + 1 & 1));
    }
  };

  // ---- fragments of sixteen entries of the sum
  struct Part {
    bf16x8 p[H::MB], q[H::NB];
  };
  struct Ahead {  // a part to be read: the j-th of its stage
    Part* part;
    int j;
  };
  // A tile of at most MT / 2 slots (an expert's last) goes through steps of its own, in which every wave has half as
  // many of them: 32768 slots of 128 experts, 1536 x 2048, 277 to 269 us; 16384 219 to 205; 5184 of 223, 360 x 448, 33
  // to 27; full tiles as before, where a branch around each block's ops took a tenth of their time.  (Each has its sums
  // to itself: where the two forms' steps met before the results, sums were copied and spilled.)
  auto is_short = [&](const ResultTile& t) __attribute__((always_inline)) { return H::kShort && t.hi - t.m0 <= MT / 2; };
  int prow0 = 0;  // this wave's first
  auto prow = [&](int m) __attribute__((always_inline)) { return prow0 + m * 32; };
  auto set_rows = [&](const ResultTile& t) __attribute__((always_inline)) { prow0 = wm * (is_short(t) ? H::MB / 2 : H::MB) * 32; };
  const int qrow = wn * 64;
  auto by_rows = [&](const char* st, int row0, int j) __attribute__((always_inline)) {
    const int r = row0 + r32;
    return *reinterpret_cast<const bf16x8*>(st + r * 128 + chunk_slot(r, 2 * j + half) * 16);
  };
  auto by_cols = [&](const char* st, int col0, int j, int cols) __attribute__((always_inline)) {
    // rows 16 j + 8 half + 4 i + (lane % 16) / 4, columns from 16 ((lane / 16) % 2) + 4 (lane % 4) on
    const int col = col0 + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    s16x4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = 16 * j + 8 * half + 4 * i + ((lane & 15) >> 2);
      v[i] = read_transposed(st + r * (cols * 2) + (((col >> 3) ^ (4 * (r & 3))) << 4) + (col & 7) * 2);
    }
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto read_q = [&](Part& f, int j, const char* st, int tile) __attribute__((always_inline)) {
    const char* q = MX ? smem + H::oTiles + tile * H::kQStage : st + H::kPStage;
#pragma unroll
    for (int n = 0; n < H::NB; ++n)
      if constexpr (H::kQCols)
        f.q[n] = by_cols(q, qrow + 32 * n, j, H::QT);
      else
        f.q[n] = by_rows(q, qrow + 32 * n, j);
  };
  auto read_p = [&](Part& f, int m, int j, const char* st) __attribute__((always_inline)) {
    if constexpr (H::kPCols)
      f.p[m] = by_cols(st, prow(m), j, MT);
    else
      f.p[m] = by_rows(st, prow(m), j);
  };
  f32x16 acc[H::NB][H::MB];
  auto clear = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < H::NB; ++i)
#pragma unroll
      for (int j = 0; j < H::MB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
  };
  // The ops of a part, with the reads of the parts of `reads` and `between(m)` after a block's ops.
  // (Blocks of 32 slots that lie past a tile's end are multiplied all the same.)
  auto multiply = [&](auto blocks, const Part& f, const char* st, int tile, auto between, auto... reads) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < decltype(blocks)::value; ++m) {
#pragma unroll
      for (int n = 0; n < H::NB; ++n) {
        acc[n][m] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.q[n], f.p[m], acc[n][m], 0, 0, 0);
        if (m == 0 && n == 0) (read_q(*reads.part, reads.j, st, tile), ...);
        if (n == H::NB - 1) (read_p(*reads.part, m, reads.j, st), ...);
        __builtin_amdgcn_sched_barrier(0);
      }
      between(m);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  const auto nothing = [](int) {};

  load_rows(cur, 0);
  wait_loads<0>();
  aim(cur, 0);
  ld = cur;
  steps_to = steps_of(cur);
  if constexpr (FORM == kWeights) {
    if (a.rows) {
      ask_rows(cur, 0, 0);
      if (l + step_l < end) ask_rows(later, 0, 1);
      if (8 < steps_to) ask_rows(cur, 1, 4);
    }
    wait_own(std::integral_constant<int, 0>{});
  }
#pragma unroll
  for (int i = 0; i < H::NX; ++i) {
    cut(entries_left());
    if constexpr (FORM == kWeights) take_rows();
    if constexpr (MX) {
      issue_codes();
      if (i == 0) {
        wait_own(std::integral_constant<int, 0>{});
#pragma unroll
        for (int j = 0; j < 4; ++j) widen(j, 0);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
    }
    issue();
  }
  if constexpr (MX)
    wait_loads<0>();
  else
    wait_loads<(H::NX - 1) * H::kLoads>();
  find_next();
  const char* st = smem;
  int tile = 0;
  // (a tile's first fragments: those that the step before it read may be of other rows)
  auto read_first = [&](Part& f, const char* st, int tile) __attribute__((always_inline)) {
    read_q(f, 0, st, tile);
#pragma unroll
    for (int m = 0; m < H::MB; ++m) read_p(f, m, 0, st);
  };
  set_rows(cur);
  // Waits for the next stage and the workgroup; N loads are younger than it.  So are the stores of the tile before (they
  // count with the loads), in a tile's first steps: they may go on where this wave made all that there can be.
  constexpr int kStores16 = (GLU ? 1 : H::NB) * H::MB * 2, kStores32 = 2 * kStores16;
  int stored = 0;
  int pending = 0;  // the last third of a stage's loads is to go out yet
  // Loads [from, to) of a stage, those of the m-th of `turns`.
  auto loads = [&](int from, int to, int m, int turns) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < H::kLoads; ++k)
      if (k >= from && k < to && (k - from) * turns / (to - from) == m) load(k);
  };
  auto wait_step = [&](auto n, bool first) __attribute__((always_inline)) {
    if (!first || !stored)
      wait_loads<decltype(n)::value>();
    else if (a.yf32)
      wait_loads<decltype(n)::value + kStores32>();
    else
      wait_loads<decltype(n)::value + kStores16>();
  };
  // A tile of `blocks` blocks of slots a wave.
  auto run = [&](auto blocks) __attribute__((always_inline)) {
    constexpr int kTurns = decltype(blocks)::value;
    const int steps = steps_of(cur);
    Part f0, f1, f2;
    clear();
    read_first(f0, st, tile);
    for (int i = 0; i < steps; ++i) {
      const int last = i + 1 == steps, rest = pending;
      // A stage is read to its end half a step early, and its place loaded again while the other half and the next
      // step's first part are multiplied: all at once the loads would hold up the ops behind them.
      multiply(blocks, f0, st, tile, [&](int m) __attribute__((always_inline)) {
        if (rest) loads(H::kSecond, H::kLoads, m, kTurns);
      }, Ahead{&f1, 1});
      if (rest) loaded();
      if constexpr (MX) {
        // the next stage's codes are there but for what was asked for later, two thirds of P of that stage
        constexpr int kLater = H::kLoads - H::kFirst;
        if (i > 0 || !stored)
          wait_own(std::integral_constant<int, kLater>{});
        else if (a.yf32)
          wait_own(std::integral_constant<int, kLater + kStores32>{});
        else
          wait_own(std::integral_constant<int, kLater + kStores16>{});
      }
      turn();
      multiply(blocks, f1, st, tile, [&](int m) __attribute__((always_inline)) {
        if (MX && m < 2) widen(m, tile ^ 1);
      }, Ahead{&f0, 2}, Ahead{&f2, 3});
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      multiply(blocks, f0, st, tile, [&](int m) __attribute__((always_inline)) {
        if (MX && m < 2) widen(2 + m, tile ^ 1);
        loads(0, H::kFirst, m, kTurns);
      });
      // the next stage is whole (but for what was asked for later)
      wait_step(std::integral_constant<int, (H::NX - 2) * H::kLoads + H::kFirst>{}, i < H::NX - 1);
      ++since;
      if constexpr (MX) issue_codes();  // (in the place of those that are widened)
      tile ^= 1;
      st = st + H::kStage == smem + H::oRows ? smem : st + H::kStage;
      // (what is read after a tile's last step is not used; its loads all go out before the results)
      multiply(blocks, f2, st, tile, [&](int m) __attribute__((always_inline)) {
        loads(H::kFirst, H::kSecond, m, kTurns);
        if (last) loads(H::kSecond, H::kLoads, m, kTurns);
      }, Ahead{&f0, 0});
      pending = !last;
      if (last) loaded();
    }
    const int mend = FORM == kWeights ? N : cur.hi;
    const bool whole = cur.n0 + QTO <= width && a.ldy % 8 == 0;
    const int r32 = opaque(tid) & 31, half = (opaque(tid) & 63) >> 5;
    stored = whole && cur.m0 + MT <= mend;
    const int64_t first_row = FORM == kWeights ? (static_cast<int64_t>(cur.part) * a.E + cur.e) * a.N : 0;
    auto exists = [&](int m) __attribute__((always_inline)) {  // the row of a forward result's slot
      if (FORM != kForward || !a.rows) return true;
      const int row = rowbuf[buf * H::kRows + prow(m) + r32];
      return row >= 0 && row < a.x_rows;
    };
    if (H::kTurn && !GLU && whole) {
      // A lane holds pieces of 16 bytes of one row; through LDS eight (16 in fp32: a quarter of the rows at a time, else
      // half) lanes get those of a row, so that a store writes whole cache lines, not 32 bytes of 32 rows (dW of 128
      // experts, 1536 x 2048, 32768 slots: 392 to 382 us; 2048 x 768 and 512 slots: 118 to 110).  Stores that pass the
      // caches by took 1.5 to 3 times as long.
      const int lane = opaque(tid) & 63;
      char* const turn_at = smem + (MX ? H::oTiles + (tile ^ 1) * H::kQStage + wave * 4096 : H::oTurn + wave * 2048);
#pragma unroll
      for (int m = 0; m < kTurns; ++m) {
        const bool have = exists(m);
        const int row0 = cur.m0 + prow(m);
        if (a.yf32) {
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            if ((r32 >> 3) == g) {
#pragma unroll
              for (int n = 0; n < H::NB; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  f32x4 v;
#pragma unroll
                  for (int i = 0; i < 4; ++i) v[i] = have ? acc[n][m][4 * e + i] : 0.0f;
                  *reinterpret_cast<f32x4*>(turn_at + (r32 & 7) * 256 + (((8 * n + 2 * e + half) ^ (r32 & 7)) << 4)) = v;
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int r = 4 * i + lane / 16, row = row0 + 8 * g + r;
              const f32x4 v = *reinterpret_cast<const f32x4*>(turn_at + r * 256 + (((lane & 15) ^ r) << 4));
              if (row < mend)
                *reinterpret_cast<f32x4*>(static_cast<float*>(a.y) + (first_row + row) * a.ldy + cur.n0 + qrow +
                                          4 * (lane & 15)) = v;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          }
        } else {
          uint4 v[H::NB][2];
#pragma unroll
          for (int n = 0; n < H::NB; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float u[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) u[i] = have ? acc[n][m][8 * e + i] : 0.0f;
              v[n][e] = eight_in_a_row(u);
            }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if ((r32 >> 4) == g) {
#pragma unroll
              for (int n = 0; n < H::NB; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                  *reinterpret_cast<uint4*>(turn_at + (r32 & 15) * 128 + (((4 * n + 2 * e + half) ^ (r32 & 7)) << 4)) =
                      v[n][e];
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int r = 8 * i + lane / 8, row = row0 + 16 * g + r;
              const uint4 w = *reinterpret_cast<const uint4*>(turn_at + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
              if (row < mend)
                *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.y) + (first_row + row) * a.ldy + cur.n0 + qrow +
                                          8 * (lane & 7)) = w;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          }
        }
      }
    } else {
#pragma unroll
      for (int m = 0; m < kTurns; ++m) {
        const int at = cur.m0 + prow(m) + r32;
        if (at >= mend) continue;
        const bool have = exists(m);
#pragma unroll
        for (int n = 0; n < (GLU ? 1 : H::NB); ++n) {
          float v[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            v[i] = acc[n][m][i];
            if constexpr (GLU) v[i] = silu(v[i]) * acc[1][m][i];
            if (FORM == kForward && !have) v[i] = 0.0f;
          }
          store32(a, first_row + at, cur.n0 + (GLU ? wn * 32 : qrow + 32 * n), half, whole, width, v);
        }
      }
    }
  };
  for (;;) {
    if constexpr (H::kShort) {
      if (is_short(cur))
        run(std::integral_constant<int, H::MB / 2>{});
      else
        run(std::integral_constant<int, H::MB>{});
    } else {
      run(std::integral_constant<int, H::MB>{});
    }
    if (!more) {
      wait_loads<0>();  // (LDS must not be written after the end)
      return;
    }
    cur = next;
    if (H::kShort) set_rows(cur);
    buf = after(buf);
    find_next();
  }
}

// 32 x 64 results a workgroup (glu: 32 gate and 32 up rows), the sum split over its
// four waves: wave w takes stages w, w + 4, ... of 64 entries through a ring of its
// own, with no barrier up to the end, where the four sums are joined in LDS in the
// order of the waves.  For calls of too few large tiles to fill the card: what counts
// is how fast one workgroup goes through a long sum (194 slots of 8 experts, 1024 x 4096: 18.6 us for
// 67 MB, where the tiles above take 39 to 74; 8 slots of 128 experts, 1536 x 2048, with glu: 12.7).
struct SplitShape {
  static constexpr int MT = 32, QT = 64, KS = 64, NX = 3, kWaves = 4;
  static constexpr int kPStage = MT * KS * 2, kStage = kPStage + QT * KS * 2, kRing = NX * kStage;
  static constexpr int LP = kPStage / 1024, LQ = QT * KS * 2 / 1024, kLoads = LP + LQ;
  static constexpr int kBytes = kWaves * kRing;
  static_assert(kBytes <= 163840 && 2 * kLoads < 64);
};

template <Form FORM, bool GLU>
__global__ __launch_bounds__(kThreads) void expert_split_kernel(ExpertArgs a) {
  using H = SplitShape;
  extern __shared__ __align__(16) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, half = lane >> 5;
  constexpr int QTO = GLU ? H::QT / 2 : H::QT;
  const int N = static_cast<int>(a.N), K = static_cast<int>(a.K), width = FORM == kForward ? N : K;
  Tile t;
  if (!find_tile(a.offsets, a.E, a.S, (width + QTO - 1) / QTO, H::MT, &t)) return;
  const int n0 = t.col * QTO;
  f32x16 acc[2];
#pragma unroll
  for (int n = 0; n < 2; ++n)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[n][e] = 0.0f;
  bool have = t.e < a.E;  // the row of this lane's slot exists
  if (t.e < a.E) {
    const char* const zero = reinterpret_cast<const char*>(kZeros);
    const int sum = FORM == kForward ? K : N, stages = (sum + H::KS - 1) / H::KS;
    char* const ring = smem + wave * H::kRing;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(ring));
    auto token = [&](int r) {  // (a row that does not exist: row 0, its results are replaced)
      const int s = min(t.lo + r, t.hi - 1);
      if (!a.rows) return static_cast<int64_t>(s);
      const int64_t row = a.rows[s];
      return row >= 0 && row < a.x_rows ? row : -1;
    };
    // (8 lanes a row of either operand)
    const int wchunk = (lane & 7) ^ (4 * ((lane / 8 >> 1) & 1));
    const char *pp[H::LP], *pq[H::LQ];
#pragma unroll
    for (int q = 0; q < H::LP; ++q) {
      const int r = q * 8 + lane / 8, c = chunk_slot(r, lane & 7);
      if constexpr (FORM == kForward)
        pp[q] = reinterpret_cast<const char*>(a.x + max(token(r), int64_t(0)) * a.ldx + c * 8);
      else
        pp[q] = reinterpret_cast<const char*>(a.dy + static_cast<int64_t>(min(t.lo + r, t.hi - 1)) * a.lddy + c * 8);
    }
#pragma unroll
    for (int q = 0; q < H::LQ; ++q) {
      const int r = q * 8 + lane / 8;
      if constexpr (FORM == kForward) {
        int64_t row;
        if constexpr (GLU)
          row = static_cast<int64_t>(t.e) * 2 * a.N + min(n0 + (r & 31), N - 1) + (r >> 5) * a.N;
        else
          row = static_cast<int64_t>(t.e) * a.N + min(n0 + r, N - 1);
        pq[q] = reinterpret_cast<const char*>(a.w + row * a.K + chunk_slot(r, lane & 7) * 8);
      } else {
        pq[q] = reinterpret_cast<const char*>(a.w + (static_cast<int64_t>(t.e) * a.N + r) * a.K +
                                              min(n0 + 8 * wchunk, K - 8));
      }
    }
    if constexpr (FORM == kForward) have = token(r32) >= 0;
    int to = 0;
    auto issue = [&](int stage) {  // (past the last one: zeros, so that waits go by count)
      const int rem = sum - stage * H::KS;
      const int64_t at = static_cast<int64_t>(stage) * (H::KS * 2);
#pragma unroll
      for (int q = 0; q < H::LP; ++q) {
        const int c = chunk_slot(q * 8 + lane / 8, lane & 7);
        load_lds16(8 * c < rem ? pp[q] + at : zero, lds0 + to * H::kStage + q * 1024);
      }
#pragma unroll
      for (int q = 0; q < H::LQ; ++q) {
        const int c = chunk_slot(q * 8 + lane / 8, lane & 7);
        const bool in = FORM == kForward ? 8 * c < rem : q * 8 + lane / 8 < rem;
        load_lds16(in ? pq[q] + (FORM == kForward ? at : at * a.K) : zero,
                   lds0 + to * H::kStage + H::kPStage + q * 1024);
      }
      to = to + 1 == H::NX ? 0 : to + 1;
    };
#pragma unroll
    for (int i = 0; i < H::NX; ++i) issue(wave + i * H::kWaves);
    const char* st = ring;
    for (int s = wave; s < stages; s += H::kWaves) {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((H::NX - 1) * H::kLoads) : "memory");
      bf16x8 p[4], q[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[j] = *reinterpret_cast<const bf16x8*>(st + r32 * 128 + chunk_slot(r32, 2 * j + half) * 16);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const char* w = st + H::kPStage;
          if constexpr (FORM == kForward) {
            q[j][n] = *reinterpret_cast<const bf16x8*>(w + (32 * n + r32) * 128 + chunk_slot(r32, 2 * j + half) * 16);
          } else {
            const int col = 32 * n + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
            s16x4 v[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int r = 16 * j + 8 * half + 4 * i + ((lane & 15) >> 2);
              v[i] = read_transposed(w + r * 128 + (((col >> 3) ^ (4 * ((r >> 1) & 1))) << 4) + (col & 7) * 2);
            }
            q[j][n] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7));
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      issue(s + H::NX * H::kWaves);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < 2; ++n)
          acc[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[j][n], p[j], acc[n], 0, 0, 0);
      st = st + H::kStage == ring + H::kRing ? ring : st + H::kStage;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    // [wave][n][16][64]
    float* join = reinterpret_cast<float*>(smem);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) join[((wave * 2 + n) * 16 + e) * 64 + lane] = acc[n][e];
    __syncthreads();
    if (wave >= (GLU ? 1 : 2)) return;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (!GLU && n != 0) continue;  // (wave n takes block n, into acc[0])
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < H::kWaves; ++w) v += join[((w * 2 + (GLU ? n : wave)) * 16 + e) * 64 + lane];
        acc[n][e] = v;
      }
  } else if (wave >= (GLU ? 1 : 2)) {
    return;
  }
  const int slot = t.lo + r32;
  if (slot >= t.hi) return;
  float v[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    v[e] = GLU ? silu(acc[0][e]) * acc[1][e] : acc[0][e];
    if (!have) v[e] = 0.0f;
  }
  store32(a, slot, n0 + 32 * wave, half, n0 + QTO <= width && a.ldy % 8 == 0, width, v);
}

template <Form FORM, bool GLU = false>
bitsmoe_status split(const ExpertArgs& a, unsigned grid, hipStream_t s) {
  auto* fn = expert_split_kernel<FORM, GLU>;
  static std::atomic<uint64_t> allowed{0};
  if (bitsmoe_status st = allow_lds(reinterpret_cast<const void*>(fn), SplitShape::kBytes, &allowed)) return st;
  KernelTimer timer("expert_split", s);
  fn<<<grid, kThreads, SplitShape::kBytes, s>>>(a);
  BITSMOE_LAUNCH_CHECK("expert_split_kernel");
  return ok();
}

// One workgroup a compute unit, as many on every XCD.
unsigned tile_grid() {
  const int cus = device_cus();
  return static_cast<unsigned>(cus < 8 ? 8 : cus / 8 * 8);
}

template <Form FORM, int MT, bool GLU = false, bool MX = false>
bitsmoe_status tiles(const ExpertArgs& a, hipStream_t s) {
  using H = Shape<FORM, MT, MX>;
  auto* fn = expert_tile_kernel<FORM, MT, GLU, MX>;
  static std::atomic<uint64_t> allowed{0};
  if (bitsmoe_status st = allow_lds(reinterpret_cast<const void*>(fn), H::kBytes, &allowed)) return st;
  KernelTimer timer(FORM == kWeights ? "expert_weights" : MT == 32 ? "expert_tile_32" : MT == 128 ? "expert_tile_128"
                                                                                               : "expert_tile_256", s);
  fn<<<tile_grid(), H::kThreads, H::kBytes, s>>>(a);
  BITSMOE_LAUNCH_CHECK("expert_tile_kernel");
  return ok();
}

constexpr int kLargestTile = 256;

bitsmoe_status check(const char* who, const ExpertArgs& a, bitsmoe_dtype t, bitsmoe_dtype yt, int64_t cols) {
  auto bad = [who](bitsmoe_status st, const char* what) { return fail(st, std::string(who) + what); };
  if (a.E <= 0 || a.N <= 0 || a.K <= 0 || a.S < 0 || a.x_rows < 0) return bad(BITSMOE_ERR_ARG, ": non-positive size");
  if (t != BITSMOE_BF16) return bad(BITSMOE_ERR_DTYPE, ": weights and rows must be bf16");
  if (yt != BITSMOE_F32 && yt != BITSMOE_BF16) return bad(BITSMOE_ERR_DTYPE, ": results are fp32 or bf16");
  // (slots are ints, and so is what lies a tile behind one; farther ahead only slot_range.hpp's rules look)
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
  if (ld < cols || ld % 8 != 0 || ld > 0x7FFFFFFF)
    return fail(BITSMOE_ERR_SHAPE,
                std::string(who) + ": rows must not overlap, and lie a multiple of 16 bytes and below 2^31 entries apart");
  return BITSMOE_OK;
}

// Workgroups for tiles of `tile` slots and `per` workgroups each.
bool grid_of(const ExpertArgs& a, int64_t tile, int64_t per, unsigned* grid) {
  const int64_t tiles = a.S / tile + (a.E + 2 < a.S ? a.E + 2 : a.S);  // (every run's last one may be part)
  if (tiles > ((int64_t(1) << 23) - 1) / per) return false;
  *grid = static_cast<unsigned>(tiles * per);
  return true;
}

// Which kernel takes a product.  The counts of an expert's slots are on the device;
// the host goes by S and E alone: about
//     tiles(m) = max(active, S / m + active / 2),  active = E (1 - exp(-S / E))
// tiles of m slots (as of slots that choose by chance), of which active / 2 hold at most half their slots (all of
// them do where active experts have as few) and take three tenths less.  The constants (us; L entries of
// the sum, `wide` rows of weights or columns of results) fit timings of every kernel at
// 53 shapes in three forms, E 1 .. 238, S / E 0.03 .. 4100, sums of 64 .. 14336 entries: there the choice
// is 3 % off the best kernel on average and 1.72 times it at worst, where the worst kernel is 3.2 times it on average;
// at 54 other shapes, timed afterwards, 2 % off and 1.41 times it at worst
// (194 slots of 8 experts, 1024 x 4096: 38 us by rows, 18.6 split, 39, 41 and 62 in tiles of 32, 128 and 256 slots;
// 32768 slots of 128 experts, 1536 x 2048: 3136, 953, 503, 280 and 274; 512 slots of 128 experts, 2048 x 768: 141,
// 119, 71, 72 and 85).
enum Kernel { kByRows, kSplit, kTiles32, kTiles128, kTiles256 };

Kernel product_kernel(const ExpertArgs& a, Form form, int64_t wide, bool glu) {
  const double E = a.E, S = static_cast<double>(a.S), active = E * (1.0 - std::exp(-S / E));
  const double L = static_cast<double>(form == kForward ? a.K : a.N);
  const double bytes = active * static_cast<double>(a.N * (glu ? 2 : 1)) * static_cast<double>(a.K) * 2e-6;
  auto tiles = [&](double m, int64_t cols) {
    const double t = S / m + active / 2;
    return (t > active ? t : active) * static_cast<double>((wide + cols - 1) / cols);
  };
  // workgroups that stay, one a compute unit, between their rounds' number and their share
  auto rounds = [&](double t) {
    const double share = t / device_cus();
    return 0.5 * (std::ceil(share) + (share > 1.0 ? share : 1.0));
  };
  auto large = [&](double m, double most, double each) {  // tiles of m slots, some of them short
    const double t = tiles(m, 256), all = t / static_cast<double>((wide + 255) / 256);
    const double brief = S > active * m / 2 ? active / 2 / all : 1.0;
    return rounds(t) * (most + L * each * (1.0 - 0.3 * brief));
  };
  auto with_bytes = [&](double us, double rate) { return us > bytes / rate ? us : bytes / rate; };
  const double chain = L * 0.001, each = tiles(16, 16) * (L * 5.3e-6 + 0.0023);
  const double cost[5] = {with_bytes(5.6 + (chain > each ? chain : each), 4.6),
                          with_bytes(1.6 + rounds(tiles(32, 64)) * (4.5 + L * 0.0024), 4.2),
                          with_bytes(2.2 + rounds(tiles(32, 256)) * (4.0 + L * 0.0071), 5.0),
                          with_bytes(large(128, 6.3, 0.0116), 5.0),
                          with_bytes(large(256, 7.0, 0.0190), 5.0)};
  int best = form == kForward ? kByRows : kSplit;  // (there is no kernel by rows for W by its rows)
  for (int k = best + 1; k <= kTiles256; ++k)
    if (cost[k] < cost[best]) best = k;
  return static_cast<Kernel>(best);
}

template <Form FORM, bool GLU>
bitsmoe_status product(const ExpertArgs& a, hipStream_t s) {
  constexpr int kPer = GLU ? 2 : 1;
  const int64_t results = FORM == kForward ? a.N : a.K;
  Kernel kernel = product_kernel(a, FORM, results * kPer, GLU);
  unsigned grid = 0;
  // (a call of more tiles than a launch takes goes to workgroups that stay)
  if ((kernel == kByRows && !grid_of(a, 16, (results + 15) / 16, &grid)) ||
      (kernel == kSplit && !grid_of(a, SplitShape::MT, (results * kPer + SplitShape::QT - 1) / SplitShape::QT, &grid)))
    kernel = kTiles32;
  if constexpr (FORM == kForward) {
    if (kernel == kByRows) {
      KernelTimer timer("expert_rows", s);
      expert_rows_kernel<GLU><<<grid, 64 * kRowWaves, 0, s>>>(a);
      BITSMOE_LAUNCH_CHECK("expert_rows_kernel");
      return ok();
    }
  }
  switch (kernel) {
    case kSplit:
      return split<FORM, GLU>(a, grid, s);
    case kTiles32:
      return tiles<FORM, 32, GLU>(a, s);
    case kTiles128:
      return tiles<FORM, 128, GLU>(a, s);
    default:
      return tiles<FORM, 256, GLU>(a, s);
  }
}

int clip(int64_t E) { return static_cast<int>(E < 0x7FFFFFFF ? E : 0x7FFFFFFF); }

// The weights' gradient from its parts' sums, in their order (bound by bytes: 64 MB of sums 12 us).
template <bool BF16>
__global__ __launch_bounds__(kThreads) void expert_join_kernel(const float* part, int parts, int64_t n, void* y) {
  for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < n; i += int64_t(gridDim.x) * kThreads) {
    Eight<BF16> sum;
    Eight<false> v;
    v.load(part, i);
#pragma unroll
    for (int q = 0; q < 8; ++q) sum.v[q] = v.v[q];
    for (int p = 1; p < parts; ++p) {
      v.load(part + p * n * 8, i);
#pragma unroll
      for (int q = 0; q < 8; ++q) sum.v[q] += v.v[q];
    }
    sum.store(y, i);
  }
}

// Parts of the weights' gradient's sum: where its tiles are too few to fill the card, as many as do, but of four
// stages at least, and with at most 64 MB of sums, whose join takes 12 us.  (128 x 2048 of 4096 tokens, a router's:
// 97 us in one part, 29 in 16; of 32768: 713 and 58; 1024 x 2048 of 16384: 367 and 94; 8 experts of 256 x 512, 8192
// slots: 31 and 30 in 4.)
int weight_parts(int64_t E, int64_t N, int64_t K, int64_t S) {
  const int64_t tiles = E * ((N + 255) / 256) * ((K + 255) / 256), cus = device_cus();
  if (tiles * 2 > cus) return 1;
  const int64_t fill = cus / tiles, stages = S / (64 * E) / 4, room = (int64_t(64) << 20) / (E * N * K * 4);
  const int64_t parts = fill < stages ? fill : stages;
  return static_cast<int>(parts < room ? (parts < 1 ? 1 : parts) : room < 1 ? 1 : room);
}

bitsmoe_status weight_grad(const char* who, ExpertArgs a, void* work, int64_t work_bytes, hipStream_t s) {
  const int64_t tiles_ = (a.N + 255) / 256 * ((a.K + 255) / 256);
  if (tiles_ > (int64_t(1) << 30) || tiles_ > (int64_t(1) << 40) / a.E) return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": too many weights");
  if (!aligned16({work}))
    return fail(BITSMOE_ERR_ARG, std::string(who) + ": device pointers must be 16-byte aligned");
  const int parts = work ? weight_parts(a.E, a.N, a.K, a.S) : 1;
  void* const y = a.y;
  const bool bf16 = !a.yf32;
  if (parts > 1) {
    if (work_bytes < parts * a.E * a.N * a.K * 4)
      return fail(BITSMOE_ERR_ARG, std::string(who) + ": the workspace is too small");
    a.parts = parts;
    a.y = work;
    a.yf32 = 1;
  }
  if (bitsmoe_status st = a.xcodes ? tiles<kWeights, 256, false, true>(a, s) : tiles<kWeights, 256>(a, s)) return st;
  if (parts > 1) {
    const int64_t n = a.E * a.N * a.K / 8, blocks = (n + kThreads - 1) / kThreads;
    auto* fn = bf16 ? expert_join_kernel<true> : expert_join_kernel<false>;
    fn<<<static_cast<unsigned>(blocks < 4096 ? blocks : 4096), kThreads, 0, s>>>(static_cast<const float*>(work), parts, n,
                                                                                 y);
    BITSMOE_LAUNCH_CHECK("expert_join_kernel");
  }
  return ok();
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" bitsmoe_status bitsmoe_expert_product(const void* W_dev, bitsmoe_dtype t, int64_t E, int64_t N, int64_t K,
                                                 const void* X_dev, int64_t x_rows, int64_t ldx,
                                                 const int32_t* offsets_dev, const int32_t* rows_dev, int64_t S,
                                                 int glu, void* Y_dev, bitsmoe_dtype yt, int64_t ldy, void* stream) {
  ExpertArgs a{static_cast<const uint16_t*>(W_dev), clip(E), N, K, static_cast<const uint16_t*>(X_dev),
                     nullptr, nullptr, x_rows, ldx, nullptr, 0, offsets_dev, rows_dev, S, Y_dev, ldy,
                     yt == BITSMOE_F32, 1};
  if (bitsmoe_status st = check("expert_product", a, t, yt, N)) return st;
  if (bitsmoe_status st = check_stride("expert_product", K, ldx)) return st;
  if (S == 0) return ok();
  if (!W_dev || !Y_dev || (x_rows > 0 && !X_dev)) return fail(BITSMOE_ERR_ARG, "expert_product: null pointer");
  if (x_rows == 0) {  // (the kernels read a first row for slots whose own does not exist, and give them 0)
    a.x = a.w;
    a.ldx = 0;
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  return glu ? product<kForward, true>(a, s) : product<kForward, false>(a, s);
}

extern "C" bitsmoe_status bitsmoe_expert_product_grad(const void* W_dev, bitsmoe_dtype t, int64_t E, int64_t N,
                                                      int64_t K, const void* dY_dev, int64_t lddy,
                                                      const int32_t* offsets_dev, int64_t S, void* dX_dev,
                                                      bitsmoe_dtype xt, int64_t ldx, void* stream) {
  const ExpertArgs a{static_cast<const uint16_t*>(W_dev), clip(E), N, K, nullptr, nullptr, nullptr, S, 0,
                     static_cast<const uint16_t*>(dY_dev), lddy, offsets_dev, nullptr, S, dX_dev, ldx,
                     xt == BITSMOE_F32, 1};
  if (bitsmoe_status st = check("expert_product_grad", a, t, xt, K)) return st;
  if (N % 8 != 0) return fail(BITSMOE_ERR_SHAPE, "expert_product_grad: needs N % 8 == 0");
  if (bitsmoe_status st = check_stride("expert_product_grad", N, lddy)) return st;
  if (S == 0) return ok();
  if (!W_dev || !dY_dev || !dX_dev) return fail(BITSMOE_ERR_ARG, "expert_product_grad: null pointer");
  return product<kTokens, false>(a, static_cast<hipStream_t>(stream));
}

extern "C" int64_t bitsmoe_expert_weight_grad_workspace(int64_t E, int64_t N, int64_t K, int64_t S) {
  if (E <= 0 || N <= 0 || K <= 0 || S <= 0 || E > 65535 || N > (1 << 24) || K > (1 << 24)) return 0;
  const int parts = weight_parts(E, N, K, S);
  return parts > 1 ? parts * E * N * K * 4 : 0;
}

extern "C" bitsmoe_status bitsmoe_expert_weight_grad(const void* dY_dev, bitsmoe_dtype t, int64_t lddy, int64_t E,
                                                     int64_t N, int64_t K, const void* X_dev, int64_t x_rows,
                                                     int64_t ldx, const int32_t* offsets_dev, const int32_t* rows_dev,
                                                     int64_t S, void* dW_dev, bitsmoe_dtype wt, void* work_dev,
                                                     int64_t work_bytes, void* stream) {
  const ExpertArgs a{nullptr, clip(E), N, K, static_cast<const uint16_t*>(X_dev), nullptr, nullptr, x_rows, ldx,
                     static_cast<const uint16_t*>(dY_dev), lddy, offsets_dev, rows_dev, S, dW_dev, K,
                     wt == BITSMOE_F32, 1};
  if (bitsmoe_status st = check("expert_weight_grad", a, t, wt, K)) return st;
  if (N % 8 != 0) return fail(BITSMOE_ERR_SHAPE, "expert_weight_grad: needs N % 8 == 0");
  if (bitsmoe_status st = check_stride("expert_weight_grad", N, lddy)) return st;
  if (bitsmoe_status st = check_stride("expert_weight_grad", K, ldx)) return st;
  if (!dW_dev || (S > 0 && (!dY_dev || (x_rows > 0 && !X_dev))))
    return fail(BITSMOE_ERR_ARG, "expert_weight_grad: null pointer");
  return weight_grad("expert_weight_grad", a, work_dev, work_bytes, static_cast<hipStream_t>(stream));
}

extern "C" bitsmoe_status bitsmoe_expert_weight_grad_q(const void* dY_dev, bitsmoe_dtype t, int64_t lddy, int64_t E,
                                                       int64_t N, int64_t K, const uint8_t* xcodes_dev,
                                                       const uint8_t* xscales_dev, int64_t x_rows,
                                                       const int32_t* offsets_dev, const int32_t* rows_dev, int64_t S,
                                                       void* dW_dev, bitsmoe_dtype wt, void* work_dev, int64_t work_bytes,
                                                       void* stream) {
  const ExpertArgs a{nullptr, clip(E), N, K, nullptr, xcodes_dev, xscales_dev, x_rows, K,
                     static_cast<const uint16_t*>(dY_dev), lddy, offsets_dev, rows_dev, S, dW_dev, K,
                     wt == BITSMOE_F32, 1};
  if (bitsmoe_status st = check("expert_weight_grad_q", a, t, wt, K)) return st;
  if (N % 8 != 0 || K % kMx8Block != 0)
    return fail(BITSMOE_ERR_SHAPE, "expert_weight_grad_q: needs N % 8 == 0 and K % 32 == 0");
  if (bitsmoe_status st = check_stride("expert_weight_grad_q", N, lddy)) return st;
  if (!dW_dev || (S > 0 && (!dY_dev || (x_rows > 0 && (!xcodes_dev || !xscales_dev)))))
    return fail(BITSMOE_ERR_ARG, "expert_weight_grad_q: null pointer");
  return weight_grad("expert_weight_grad_q", a, work_dev, work_bytes, static_cast<hipStream_t>(stream));
}
