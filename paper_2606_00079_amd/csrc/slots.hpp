// What the experts' products share: which tile of slots and outputs a workgroup
// takes, direct loads into LDS, and the storing of results.
#pragma once

#include "mx4.hpp"

namespace bitsmoe {

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
// holds the slots of no expert past the last expert's, and e = E + 1 those
// before the first one's: their results are zero.
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
  // (both loads at once whatever e is: a chain of two would lengthen every search)
  const int first = offsets ? offsets[min(e, E)] : 0, end = offsets ? offsets[e < E ? e + 1 : 0] : 0;
  if (!offsets) {
    *lo = e == 1 ? S : 0;  // (E = 1)
    return e == 0 ? S : 0;
  }
  *lo = e > E ? 0 : min(max(first, 0), S);
  return (e == E ? S : min(max(end, *lo), S)) - *lo;
}
__device__ __forceinline__ bool find_tile(const int32_t* offsets, int E, int64_t S, int cols, int tile, Tile* out) {
  const int s = static_cast<int>(S), lane = threadIdx.x & 63;
  const int per = (E + 1) / 64 + 1;  // experts a lane, of E + 2
  int lo, tiles = 0;
  for (int i = 0; i < per; ++i) {
    const int e = lane * per + i;
    if (e <= E + 1) tiles += (slots_of(offsets, E, s, e, &lo) + tile - 1) / tile;
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
  for (;; e += 64) {  // (one pass up to 4094 experts)
    const int f = e + lane;
    const int have = f <= E + 1 && f < (run + 1) * per ? slots_of(offsets, E, s, f, &lo) : 0;
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

// (A 64-bit division takes as long as a step of a tile's sum; only calls of more than 2^32 tiles need one.)
__device__ __forceinline__ int64_t quotient(int64_t a, uint32_t b) {
  return a >> 32 ? a / static_cast<int64_t>(b) : static_cast<int64_t>(static_cast<uint32_t>(a) / b);
}

// The same order of tiles for a workgroup that stays and takes one tile after
// another (without those of no expert): it goes on from expert to expert with
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
    const int g = static_cast<int>(quotient(l, static_cast<uint32_t>(cols)));
    while (g >= before + tiles()) {
      before += tiles();
      ++e;
      load();
    }
    return true;
  }
  __device__ __forceinline__ void get(Tile* out) const {
    const int64_t in = l - static_cast<int64_t>(before) * cols;
    const int group = static_cast<int>(quotient(in, 8u * static_cast<uint32_t>(cols)));
    const int rest = static_cast<int>(in - group * 8 * static_cast<int64_t>(cols));
    const int high = min(8, tiles() - 8 * group), row = 8 * group + rest % high;
    out->e = e;
    out->col = rest / high;
    out->lo = first + row * tile;
    out->hi = min(first + count, out->lo + tile);
  }
  // The first tile of this workgroup; slots below *head and from *none on have no expert.
  __device__ __forceinline__ bool start(const int32_t* off, int E_, int64_t S_, int cols_, int tile_, int* head,
                                        int* none) {
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
    *head = offsets ? min(max(offsets[0], 0), S) : 0;
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

// v / (1 + exp(-v)) by the hardware's exponential and reciprocal: within 2^-21 of
// itself, with a fifth of the instructions of the library's exponential and an
// exact division (below v = -87.3, where it is smaller than 88 2^-126, it is 0).
__device__ __forceinline__ float silu(float v) {
  return v * __builtin_amdgcn_rcpf(1.0f + exp_hw(__builtin_amdgcn_fmed3f(-v, -150.0f, 88.0f)));
}

// Four consecutive results n .. n + 3 of slot s (A: y, its row stride ldy, and yf32).
template <class A>
__device__ __forceinline__ void store4(const A& a, int64_t s, int64_t n, int64_t N, bool wide, f32x4 v) {
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

// Eight results in a row as bf16, from two runs of four of a 32 x 32 accumulator: those at
// 16 e + 4 half + i (i < 4) and 16 e + 8 + 4 half + i; the two half-waves exchange words, and
// a lane gets those from 16 e + 8 half on.
__device__ __forceinline__ uint4 eight_in_a_row(const float (&v)[8]) {
  uint32_t w[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bf16x2 b = {static_cast<__bf16>(v[4 * i + 2 * h]), static_cast<__bf16>(v[4 * i + 2 * h + 1])};
      w[i][h] = __builtin_bit_cast(uint32_t, b);
    }
  const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
  const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
  return make_uint4(x[0], y[0], x[1], y[1]);
}

// A lane's part of the 32 results n .. n + 31 (of N) of slot s: v[i] is that of
// n + 8 (i / 4) + 4 half + i % 4, as a 32 x 32 accumulator lies.
template <class A>
__device__ __forceinline__ void store32(const A& a, int64_t s, int64_t n, int half, bool whole, int64_t N,
                                        const float (&v)[16]) {
  if (!whole) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int64_t at = n + 8 * e + 4 * half;
      if (at < N) store4(a, s, at, N, a.ldy % 4 == 0, f32x4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]});
    }
  } else if (a.yf32) {
    float* p = static_cast<float*>(a.y) + s * a.ldy + n + 4 * half;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      *reinterpret_cast<f32x4*>(p + 8 * e) = f32x4{v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]};
  } else {
    uint16_t* p = static_cast<uint16_t*>(a.y) + s * a.ldy + n + 8 * half;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float u[8] = {v[8 * e],     v[8 * e + 1], v[8 * e + 2], v[8 * e + 3],
                          v[8 * e + 4], v[8 * e + 5], v[8 * e + 6], v[8 * e + 7]};
      *reinterpret_cast<uint4*>(p + 16 * e) = eight_in_a_row(u);
    }
  }
}

// One wave-wide direct load: lane l's 16 bytes (word, byte) at p go to lds + 16 l
// (lds + 4 l, a byte as a word).  `lds` is wave-uniform.  The compiler does not
// track it: callers wait by count (wait_loads) and synchronize before the data
// is read.
__device__ __forceinline__ void load_lds16(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(p),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory");
}
__device__ __forceinline__ void load_lds4(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(p),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory");
}
__device__ __forceinline__ void load_lds1(const void* p, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ubyte %0, off" ::"v"(p),
               "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory");
}
// Waits until at most N of this wave's loads, and none of its LDS reads, are
// under way, and for the workgroup.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64);
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// Place of 16-byte chunk c of row r in a stage of 128-byte rows: sixteen rows
// read at the same chunk (what the LDS serves together) then lie in different
// banks.
__device__ __forceinline__ int chunk_slot(int r, int c) { return c ^ ((r >> 1) & 7); }
typedef __attribute__((ext_vector_type(4))) short s16x4;
__device__ __forceinline__ s16x4 read_transposed(const char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(reinterpret_cast<uintptr_t>(p)));
}

}  // namespace bitsmoe
