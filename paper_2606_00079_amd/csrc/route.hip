// The router of an MoE layer: softmax, the k largest experts of every token,
// their weights, the slots in expert order, and the losses that keep the
// experts evenly used; and the gradient of its logits.
//
// Forward, for a counted row t (valid, with a logit above -inf):
//     p_te = exp(l_te - lse_t),  S_t = the k largest logits (ties: lowest e),
//     w_tj = p_tj / sum_{S_t} p  (or p_tj as it is),
//     c_e = number of slots of e,  P_e = sum_t p_te,  n = counted rows,
//     balance = E / (k n^2) sum_e c_e P_e,   z = 1/n sum_t lse_t^2.
// Backward, with a_e = E c_e / (k n^2) (the counts carry no gradient):
//     dl_te = gb p_te (a_e - sum_f p_tf a_f) + 2 gz / n lse_t p_te + gate term.
//
// A row lies on LPT lanes, V consecutive logits a lane (V = 8 up to 512
// experts), so that up to 64 rows share a wave and every reduction is a few
// lane exchanges.  Workgroups take runs of consecutive rows: a first launch
// writes each run's expert counts and probability sums, a second one sums them
// up over the runs (integers, and fp32 in the order of the runs: results do not
// depend on timing), and a third places the slots.  A single run does it all in
// one launch.
//
// The largest calls are bound by the logits' bytes and a row's chain of lane
// exchanges, the others by their launches: 16384 rows of 256 fp32 logits, k = 8
// (17 MB), take 18 us (rows), 4 (sums), 7 (places) and 16 for the gradient (34 MB);
// one row of 128, 7.8 us in its one launch, the chain of k rounds, barriers and
// placement.
#include <atomic>
#include <cstdint>
#include <string>
#include <type_traits>

#include "common.hpp"
#include "internal.hpp"

namespace bitsmoe {
namespace {

constexpr int kThreads = 1024;      // of a workgroup with eight logits a lane (256 with more)
constexpr int kGradThreads = 256;
constexpr int kMaxExperts = 4096;
constexpr int kMaxRuns = 256;       // workgroups of the first launch, unless a run gets too long
constexpr int kMinRun = 16;         // rows of the shortest run
constexpr int kMaxRun = 128;        // and of the longest
constexpr int kOneRun = 128;        // rows that one workgroup does alone, up to 512 experts
constexpr int kMostLds = 163840;

// fp32 as an unsigned integer of the same order, and back; 0 is below -inf.
__device__ __forceinline__ uint32_t order_bits(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);  // (-0 counts as 0)
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

// A row's lanes exchange values inside the VALU: by lane permutations within
// sixteen lanes (neighbour, pair, then mirrored halves, whose lanes already
// agree), and by swapping rows of lanes beyond.
template <int LPT, typename T, typename F>
__device__ __forceinline__ T row_reduce(T v, F f) {
  static_assert(sizeof(T) == 4);
  auto dpp = [&](auto ctrl) {
    const int x = __builtin_bit_cast(int, v);
    v = f(v, __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xF, 0xF, false)));
  };
  if constexpr (LPT > 1) dpp(std::integral_constant<int, 0xB1>());
  if constexpr (LPT > 2) dpp(std::integral_constant<int, 0x4E>());
  if constexpr (LPT > 4) dpp(std::integral_constant<int, 0x141>());
  if constexpr (LPT > 8) dpp(std::integral_constant<int, 0x140>());
  if constexpr (LPT > 16) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t p = s[0], q = s[1];  // (a bit cast of a vector's element takes the first)
    v = f(__builtin_bit_cast(T, p), __builtin_bit_cast(T, q));
  }
  if constexpr (LPT > 32) {
    const uint32_t x = __builtin_bit_cast(uint32_t, v);
    const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const uint32_t p = s[0], q = s[1];  // (a bit cast of a vector's element takes the first)
    v = f(__builtin_bit_cast(T, p), __builtin_bit_cast(T, q));
  }
  return v;
}
// exp(d) for d <= 0 (or NaN).
__device__ __forceinline__ float exp_neg(float d) {
  return exp_hw(d < -150.0f ? -150.0f : d);  // (0 in fp32; -inf would give a NaN)
}

template <int LPT>
__device__ __forceinline__ float row_sum(float v) {
  return row_reduce<LPT>(v, [](float a, float b) { return a + b; });
}
template <int LPT>
__device__ __forceinline__ float row_max(float v) {
  return row_reduce<LPT>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <int LPT>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
  return row_reduce<LPT>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// LDS operations of this wave before it are done, for its other lanes too.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The V logits first .. first + V - 1 of a row (experts past E: -inf).
template <bool BF16, int V>
__device__ __forceinline__ void load_logits(const void* row, int first, int E, bool wide, float* x) {
  if (wide && first + V <= E) {
    if constexpr (BF16 && V % 8 == 0) {
#pragma unroll
      for (int q = 0; q < V / 8; ++q) {
        const uint4 v = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(row) + first)[q];
        const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[8 * q + 2 * i] = __uint_as_float(d[i] << 16);
          x[8 * q + 2 * i + 1] = __uint_as_float(d[i] & 0xFFFF0000u);
        }
      }
      return;
    }
    if constexpr (!BF16) {
#pragma unroll
      for (int q = 0; q < V / 4; ++q) {
        const f32x4 v = reinterpret_cast<const f32x4*>(static_cast<const float*>(row) + first)[q];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[4 * q + i] = v[i];
      }
      return;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int e = first + i;
    float v = -INFINITY;
    if (e < E)
      v = BF16 ? bf16_to_f32(static_cast<const uint16_t*>(row)[e]) : static_cast<const float*>(row)[e];
    x[i] = v;
  }
}

struct RouteArgs {
  const void* logits;
  int64_t ld;
  int64_t T;
  int E, k, renorm, wide;
  int run, runs;  // rows of a run, and how many runs
  const uint8_t* valid;
  int32_t* experts;
  float* weights;
  int32_t* counts;   // [E + 1]: slots of every expert, then the counted rows
  int32_t* offsets;  // [E + 1]
  int32_t* rows;
  int32_t* slots;
  float* lse;
  float* losses;
  // of every run: slots of every expert [E], probability sums [E], z and counted rows
  int32_t* run_counts;
  float* run_probs;
  float* run_z;
  int32_t* run_n;
};

// Exclusive sums over v[0 .. n) in LDS (n <= kMaxExperts + 1), in place, by NT
// threads; `tmp` holds a value a wave.  Ends with a barrier.
template <int NT>
__device__ __forceinline__ void exclusive_scan(int32_t* v, int n, int32_t* tmp) {
  const int per = (n + NT - 1) / NT, tid = threadIdx.x;
  const int lo = min(n, tid * per), hi = min(n, lo + per);
  int s = 0;
  for (int i = lo; i < hi; ++i) s += v[i];
  int inc = s;  // inclusive over the wave
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(inc, o, 64);
    if ((tid & 63) >= o) inc += u;
  }
  if ((tid & 63) == 63) tmp[tid >> 6] = inc;
  __syncthreads();
  int base = inc - s;
  for (int w = 0; w < (tid >> 6); ++w) base += tmp[w];
  for (int i = lo; i < hi; ++i) {
    const int c = v[i];
    v[i] = base;
    base += c;
  }
  __syncthreads();
}

// Places the slots of a run of `rows` rows from row0 on, experts[i] being the
// expert of its slot i: next[e] is where the run's first slot of expert e goes
// (e = E: no expert).  A slot's place among its expert's is the number of rows
// before it that have the expert too, by a bit a row in mask [E][words]; an
// expert is in a row once.  Slots without an expert are a row's last ones: what
// comes before them is all slots before less those with an expert, taken
// [rows + 1] and tmp (a value a wave).
template <int NT>
__device__ __forceinline__ void place_slots(const RouteArgs& a, const int32_t* next, const int32_t* experts,
                                            int64_t row0, int rows, uint32_t* mask, int32_t* taken, int32_t* tmp) {
  const int words = (rows + 31) / 32, n = rows * a.k, tid = threadIdx.x;
  for (int i = tid; i < a.E * words; i += NT) mask[i] = 0;
  for (int i = tid; i <= rows; i += NT) taken[i] = 0;
  __syncthreads();
  const uint64_t inv = (uint64_t(1) << 32) / a.k + 1;  // i / k = i inv / 2^32 for i < 2^16, k <= 64
  for (int i = tid; i < n; i += NT) {
    const int e = experts[i], r = static_cast<int>((static_cast<uint32_t>(i) * inv) >> 32);
    if (e < 0) continue;
    atomicOr(&mask[e * words + (r >> 5)], 1u << (r & 31));
    atomicAdd(&taken[r], 1);
  }
  __syncthreads();
  exclusive_scan<NT>(taken, rows + 1, tmp);
  for (int i = tid; i < n; i += NT) {
    const int e = experts[i], r = static_cast<int>((static_cast<uint32_t>(i) * inv) >> 32);
    int pos;
    if (e >= 0) {
      pos = next[e] + __popc(mask[e * words + (r >> 5)] & ((1u << (r & 31)) - 1));
      for (int w = 0; w < (r >> 5); ++w) pos += __popc(mask[e * words + w]);
    } else {
      pos = next[a.E] + i - taken[r + 1];
    }
    a.rows[pos] = static_cast<int32_t>(row0) + r;
    a.slots[row0 * a.k + i] = pos;
  }
}

__device__ __forceinline__ void write_losses(const RouteArgs& a, float balance, float z, int rows) {
  const float n = static_cast<float>(rows);
  a.losses[0] = rows > 0 ? balance * (static_cast<float>(a.E) / (static_cast<float>(a.k) * n * n)) : 0.0f;
  a.losses[1] = rows > 0 ? z / n : 0.0f;
  a.counts[a.E] = rows;
}

// Sum over the workgroup in a fixed order, valid in thread 0.
template <int NT, typename T>
__device__ __forceinline__ T block_sum(T v, void* lds) {
  T* tmp = static_cast<T*>(lds);
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
  __syncthreads();
  T s = 0;
  for (int w = 0; w < NT / 64; ++w) s += tmp[w];
  return s;
}

// First launch: the rows of one run, bound by the k rounds of lane exchanges
// (1 TB/s at 16384 rows of 256 logits).
template <bool BF16, int V, int LPT, int NT>
__global__ __launch_bounds__(NT) void route_rows_kernel(RouteArgs a) {
  constexpr int G = NT / LPT;  // rows at a time
  extern __shared__ __align__(16) char smem[];
  float* probs = reinterpret_cast<float*>(smem);                  // [G][LPT * V]
  int32_t* cnt = reinterpret_cast<int32_t*>(probs + NT * V);  // [E + 1]
  float* chosen = reinterpret_cast<float*>(cnt + a.E + 1);        // [G][k]
  float* tmp = chosen + G * a.k;                                  // [NT / 64]
  // one run only: the experts of its slots, and what place_slots takes
  int32_t* list = reinterpret_cast<int32_t*>(tmp + NT / 64);  // [run][k]
  int32_t* taken = list + a.run * a.k;                        // [run + 1]
  uint32_t* mask = reinterpret_cast<uint32_t*>(taken + a.run + 1);  // [E][words]
  const int tid = threadIdx.x, lane = tid % LPT, grp = tid / LPT;
  const bool one = a.runs == 1;
  const int64_t t0 = static_cast<int64_t>(blockIdx.x) * a.run;
  const int nrows = static_cast<int>(min(static_cast<int64_t>(a.run), a.T - t0));
  for (int e = tid; e <= a.E; e += NT) cnt[e] = 0;
  __syncthreads();
  const int first = lane * V;
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.0f;
  float zsum = 0.0f;
  int nsum = 0;
  for (int r = grp; r < nrows; r += G) {
    const int64_t t = t0 + r;
    const char* row = static_cast<const char*>(a.logits) + t * a.ld * (BF16 ? 2 : 4);
    float x[V];
    load_logits<BF16, V>(row, first, a.E, a.wide != 0, x);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < V; ++i) m = fmaxf(m, x[i]);
    m = row_max<LPT>(m);
    m = m == -INFINITY ? 0.0f : m;
    float ex[V], total = 0.0f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      ex[i] = exp_neg(x[i] - m);  // (NaN for a NaN, and in a row with an infinity)
      total += ex[i];
    }
    total = row_sum<LPT>(total);
    const bool broken = !(total == total);
    const bool live = (a.valid == nullptr || a.valid[t] != 0) && (broken || total > 0.0f);
    const float inv = 1.0f / total;
    const float lse = live ? m + logf(total) : -INFINITY;
    if (live) {
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += ex[i] * inv;
      ++nsum;
      zsum += lse * lse;
    }
    if (lane == 0) a.lse[t] = lse;
    // The k largest, one after another: the largest logit over the row's lanes, and of the lanes that have it the
    // lowest one, whose logits have the lowest indices.
    uint32_t key[V];
#pragma unroll
    for (int i = 0; i < V; ++i) key[i] = live && !broken && x[i] > -INFINITY ? order_bits(x[i]) : 0;
    for (int j = 0; j < a.k; ++j) {
      uint32_t mine = key[0];
#pragma unroll
      for (int i = 1; i < V; ++i) mine = key[i] > mine ? key[i] : mine;
      const uint32_t best = row_max<LPT>(mine);
      const uint64_t have = __ballot(mine == best) >> ((threadIdx.x & 63) / LPT * LPT);
      const bool winner = lane == (LPT == 64 ? __builtin_ctzll(have) : __builtin_ctz(static_cast<uint32_t>(have)));
      if (winner) {
        int e = -1;
        if (best != 0) {
#pragma unroll
          for (int i = V - 1; i >= 0; --i) e = key[i] == best ? first + i : e;
#pragma unroll
          for (int i = 0; i < V; ++i) key[i] = first + i == e ? 0 : key[i];
        }
        a.experts[t * a.k + j] = e;
        chosen[grp * a.k + j] = best != 0 ? order_value(best) : -INFINITY;
        const int bucket = e < 0 ? a.E : e;
        atomicAdd(&cnt[bucket], 1);
        if (one) list[r * a.k + j] = e;
      }
    }
    // their weights, a slot a lane (the row's lanes are of one wave, which wrote what is read here)
    wave_fence();
    float total_w = 0.0f;
    for (int j = lane; j < a.k; j += LPT) {
      float p = exp_neg(chosen[grp * a.k + j] - m) * inv;
      p = live && broken ? __uint_as_float(0x7FC00000u) : live ? p : 0.0f;
      chosen[grp * a.k + j] = p;
      total_w += p;
    }
    total_w = row_sum<LPT>(total_w);
    const float scale = a.renorm && total_w != 0.0f ? 1.0f / total_w : 1.0f;
    for (int j = lane; j < a.k; j += LPT) a.weights[t * a.k + j] = chosen[grp * a.k + j] * scale;
    wave_fence();  // (the next row's winners write where other lanes have read)
  }
#pragma unroll
  for (int i = 0; i < V; ++i) probs[grp * LPT * V + first + i] = sum[i];
  // z and n of the run: from one lane of every row, the rows in a fixed order
  const float z = block_sum<NT>(lane == 0 ? zsum : 0.0f, tmp);
  const int n = block_sum<NT>(lane == 0 ? nsum : 0, tmp);
  __syncthreads();
  if (!one) {
    for (int e = tid; e < a.E; e += NT) a.run_counts[int64_t(blockIdx.x) * a.E + e] = cnt[e];
    for (int e = tid; e < a.E; e += NT) {
      float s = 0.0f;
      for (int g = 0; g < G; ++g) s += probs[g * LPT * V + e];
      a.run_probs[int64_t(blockIdx.x) * a.E + e] = s;
    }
    if (tid == 0) {
      a.run_z[blockIdx.x] = z;
      a.run_n[blockIdx.x] = n;
    }
    return;
  }
  float balance = 0.0f;
  for (int e = tid; e < a.E; e += NT) {
    float s = 0.0f;
    for (int g = 0; g < G; ++g) s += probs[g * LPT * V + e];
    balance += s * static_cast<float>(cnt[e]);
    a.counts[e] = cnt[e];
  }
  balance = block_sum<NT>(balance, tmp);
  if (tid == 0) write_losses(a, balance, z, n);
  __syncthreads();
  exclusive_scan<NT>(cnt, a.E + 1, reinterpret_cast<int32_t*>(tmp));
  for (int e = tid; e <= a.E; e += NT) a.offsets[e] = cnt[e];
  place_slots<NT>(a, cnt, list, 0, nrows, mask, taken, reinterpret_cast<int32_t*>(tmp));
}

// Second launch: 32 experts a workgroup, 32 threads an expert.  Every run's
// count becomes the sum of those before it; the totals follow the last run's.
// With few instructions on purpose, as are the others: a launch this short is
// bound by fetching them.
__global__ __launch_bounds__(1024) void route_sum_kernel(RouteArgs a) {
  __shared__ int32_t part[32][33];
  __shared__ float ppart[32][33];
  const int col = threadIdx.x & 31, s = threadIdx.x >> 5, e = blockIdx.x * 32 + col;
  const int each = (a.runs + 31) / 32, lo = min(a.runs, s * each), hi = min(a.runs, lo + each);
  int sum = 0;
  float p = 0.0f;
  if (e < a.E) {
    const int32_t* c = a.run_counts + static_cast<int64_t>(lo) * a.E + e;
    const float* f = a.run_probs + static_cast<int64_t>(lo) * a.E + e;
#pragma unroll 8
    for (int q = lo; q < hi; ++q) {
      sum += *c;
      p += *f;
      c += a.E;
      f += a.E;
    }
  }
  part[s][col] = sum;
  ppart[s][col] = p;
  __syncthreads();
  if (e >= a.E) return;
  int before = 0;
  for (int u = 0; u < s; ++u) before += part[u][col];
  int32_t* c = a.run_counts + static_cast<int64_t>(lo) * a.E + e;
#pragma unroll 8
  for (int q = lo; q < hi; ++q) {
    const int v = *c;
    *c = before;
    before += v;
    c += a.E;
  }
  if (s == 31) {
    a.run_counts[static_cast<int64_t>(a.runs) * a.E + e] = before;
    a.counts[e] = before;
  }
  if (s == 0) {
    for (int u = 1; u < 32; ++u) p += ppart[u][col];
    a.run_probs[static_cast<int64_t>(a.runs) * a.E + e] = p;
  }
}

// Third launch: workgroup b < runs places the slots of run b; the last one
// writes the offsets and losses.
__global__ __launch_bounds__(kThreads) void route_place_kernel(RouteArgs a) {
  extern __shared__ __align__(16) char smem[];
  int32_t* next = reinterpret_cast<int32_t*>(smem);  // [E + 1]
  int32_t* tmp = next + a.E + 1;                     // [kThreads / 64]
  int32_t* taken = tmp + kThreads / 64;              // [run + 1]
  uint32_t* mask = reinterpret_cast<uint32_t*>(taken + a.run + 1);  // [E][words]
  const int tid = threadIdx.x, b = blockIdx.x;
  const bool last = b == a.runs;
  const int64_t row0 = static_cast<int64_t>(b) * a.run;
  const int32_t* total = a.run_counts + static_cast<int64_t>(a.runs) * a.E;
  for (int e = tid; e < a.E; e += kThreads) next[e] = total[e];
  if (tid == 0) next[a.E] = 0;
  __syncthreads();
  if (last) {
    float balance = 0.0f, z = 0.0f;
    int rows = 0;
    for (int e = tid; e < a.E; e += kThreads)
      balance += static_cast<float>(next[e]) * a.run_probs[static_cast<int64_t>(a.runs) * a.E + e];
    for (int q = tid; q < a.runs; q += kThreads) {
      z += a.run_z[q];
      rows += a.run_n[q];
    }
    balance = block_sum<kThreads>(balance, tmp);
    z = block_sum<kThreads>(z, tmp);
    rows = block_sum<kThreads>(rows, tmp);
    if (tid == 0) write_losses(a, balance, z, rows);
    __syncthreads();
  }
  exclusive_scan<kThreads>(next, a.E + 1, tmp);
  if (last) {
    for (int e = tid; e <= a.E; e += kThreads) a.offsets[e] = next[e];
    return;
  }
  // the slots of the runs before: of every expert, and (what those leave) of none
  int before = 0;
  for (int e = tid; e < a.E; e += kThreads) {
    const int c = a.run_counts[static_cast<int64_t>(b) * a.E + e];
    next[e] += c;
    before += c;
  }
  before = block_sum<kThreads>(before, tmp);
  if (tid == 0) next[a.E] += static_cast<int32_t>(row0 * a.k - before);
  place_slots<kThreads>(a, next, a.experts + row0 * a.k, row0,
                        static_cast<int>(min(static_cast<int64_t>(a.run), a.T - row0)), mask, taken, tmp);
}

// No rows at all.
__global__ void route_none_kernel(int E, int32_t* counts, int32_t* offsets, float* losses) {
  for (int e = threadIdx.x; e <= E; e += blockDim.x) counts[e] = offsets[e] = 0;
  if (threadIdx.x < 2) losses[threadIdx.x] = 0.0f;
}

struct GradArgs {
  const void* logits;
  int64_t ld, T;
  int E, k, renorm, wide;
  const int32_t* experts;
  const float* weights;
  const int32_t* counts;
  const float* lse;
  const float* dweights;
  const float* dlosses;
  void* dlogits;
};

// A row on LPT lanes as in the forward form; a row's slots lie on its lanes too, and
// their gate terms reach the lanes of their experts through LDS (by shuffles and
// compares the kernel took 18 us, with it 15.6).  Read and written once: 16384 rows
// of 256 fp32 logits (34 MB) at 2.2 TB/s, bound by the instructions of a row's
// exponentials and sums and by its chain of loads.
template <bool BF16, int V, int LPT>
__global__ __launch_bounds__(kGradThreads) void route_grad_kernel(GradArgs a) {
  constexpr int G = kGradThreads / LPT;
  __shared__ __align__(16) float gates[kGradThreads * V];  // a row's gate terms by expert; zero between rows
  const int lane = threadIdx.x % LPT, grp = threadIdx.x / LPT, first = lane * V;
  float* gate = gates + grp * (LPT * V);
#pragma unroll
  for (int i = 0; i < V; ++i) gate[first + i] = 0.0f;
  const float n = static_cast<float>(a.counts[a.E]);
  const float gb =
      a.dlosses && n > 0.0f ? a.dlosses[0] * (static_cast<float>(a.E) / (static_cast<float>(a.k) * n * n)) : 0.0f;
  const float gz = a.dlosses && n > 0.0f ? a.dlosses[1] * 2.0f / n : 0.0f;
  float share[V];  // gb E c_e / (k n^2)
#pragma unroll
  for (int i = 0; i < V; ++i) share[i] = first + i < a.E ? gb * static_cast<float>(a.counts[first + i]) : 0.0f;
  for (int64_t t = static_cast<int64_t>(blockIdx.x) * G + grp; t < a.T;
       t += static_cast<int64_t>(gridDim.x) * G) {
    // (all that a row needs is asked for at once)
    float p[V], d[V];
    load_logits<BF16, V>(static_cast<const char*>(a.logits) + t * a.ld * (BF16 ? 2 : 4), first, a.E, a.wide != 0, p);
    const float lse = a.lse[t];
    // a slot a lane: its expert, and weight x gradient
    int e0 = -1;
    float w0 = 0.0f, dw0 = 0.0f, wd = 0.0f;
    if (a.dweights) {
      if (lane < a.k) {
        e0 = a.experts[t * a.k + lane];
        w0 = a.weights[t * a.k + lane];
        dw0 = a.dweights[t * a.k + lane];
        wd = e0 >= 0 ? w0 * dw0 : 0.0f;
      }
      for (int j = lane + LPT; j < a.k; j += LPT)  // (more slots than lanes)
        if (a.experts[t * a.k + j] >= 0) wd += a.weights[t * a.k + j] * a.dweights[t * a.k + j];
    }
    if (lse == -INFINITY) {  // a row that does not count
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = 0.0f;
    } else {
      // p anew from the row: from lse alone a large lse would cost it its digits
      float m = -INFINITY, total = 0.0f, s = 0.0f;
#pragma unroll
      for (int i = 0; i < V; ++i) m = fmaxf(m, p[i]);
      m = row_max<LPT>(m);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        p[i] = exp_neg(p[i] - m);
        total += p[i];
      }
      const float inv = 1.0f / row_sum<LPT>(total);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        p[i] *= inv;
        s += p[i] * share[i];
      }
      s = row_sum<LPT>(s);
      wd = row_sum<LPT>(wd);
      const float all = gz * lse - s - (a.renorm ? 0.0f : wd);
#pragma unroll
      for (int i = 0; i < V; ++i) d[i] = p[i] * (share[i] + all);
      if (a.dweights) {
        const float mean = a.renorm ? wd : 0.0f;
        auto put = [&](int e, float g) {
          if (e >= 0 && e < a.E) atomicAdd(gate + e, g);  // (one slot an expert)
        };
        if (lane < a.k) put(e0, w0 * (dw0 - mean));
        for (int j = lane + LPT; j < a.k; j += LPT)
          put(a.experts[t * a.k + j], a.weights[t * a.k + j] * (a.dweights[t * a.k + j] - mean));
        wave_fence();  // (a row's lanes are of one wave)
#pragma unroll
        for (int i = 0; i < V; ++i) d[i] += gate[first + i];
#pragma unroll
        for (int i = 0; i < V; ++i) gate[first + i] = 0.0f;
        wave_fence();
      }
    }
    if constexpr (BF16) {
      uint16_t* out = static_cast<uint16_t*>(a.dlogits) + t * a.E + first;
      if (V % 8 == 0 && a.E % 8 == 0 && first + V <= a.E) {
#pragma unroll
        for (int q = 0; q < V / 8; ++q) {
          bf16x8 v;
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] = static_cast<__bf16>(d[8 * q + i]);
          reinterpret_cast<bf16x8*>(out)[q] = v;
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (first + i < a.E) out[i] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(d[i]));
      }
    } else {
      float* out = static_cast<float*>(a.dlogits) + t * a.E + first;
      if (a.E % 4 == 0 && first + V <= a.E) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
          f32x4 v;
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = d[4 * q + i];
          reinterpret_cast<f32x4*>(out)[q] = v;
        }
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (first + i < a.E) out[i] = d[i];
      }
    }
  }
}

// Calls f(V, LPT) as integral constants for rows of E logits.
template <typename F>
void with_layout(int64_t E, F f) {
  using I8 = std::integral_constant<int, 8>;
  using I64 = std::integral_constant<int, 64>;
  if (E <= 8) f(I8(), std::integral_constant<int, 1>());
  else if (E <= 16) f(I8(), std::integral_constant<int, 2>());
  else if (E <= 32) f(I8(), std::integral_constant<int, 4>());
  else if (E <= 64) f(I8(), std::integral_constant<int, 8>());
  else if (E <= 128) f(I8(), std::integral_constant<int, 16>());
  else if (E <= 256) f(I8(), std::integral_constant<int, 32>());
  else if (E <= 512) f(I8(), I64());
  else if (E <= 1024) f(std::integral_constant<int, 16>(), I64());
  else if (E <= 2048) f(std::integral_constant<int, 32>(), I64());
  else f(I64(), I64());
}

bitsmoe_status check(const char* who, const void* logits, bitsmoe_dtype lt, int64_t T, int64_t E, int64_t ld,
                     int64_t k) {
  if (T < 0 || E <= 0 || k <= 0 || (T > 0 && logits == nullptr))
    return fail(BITSMOE_ERR_ARG, std::string(who) + ": null pointer or non-positive size");
  if (lt != BITSMOE_F32 && lt != BITSMOE_BF16)
    return fail(BITSMOE_ERR_DTYPE, std::string(who) + ": logits must be fp32 or bf16");
  if (E > kMaxExperts || k > E || k > BITSMOE_ROUTE_MAX_K)
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": needs E <= 4096 and k <= min(E, 64)");
  if (ld < E || T > (int64_t(1) << 31) / k - 1 || ld > (int64_t(1) << 40))
    return fail(BITSMOE_ERR_SHAPE, std::string(who) + ": needs ld >= E and T * k < 2^31");
  return BITSMOE_OK;
}

bool wide_rows(const void* p, bitsmoe_dtype lt, int64_t E, int64_t ld) {
  const int64_t size = lt == BITSMOE_BF16 ? 2 : 4;
  return aligned16({p}) && ld * size % 16 == 0 && E % 8 == 0;
}

// How a call's rows are cut into runs, and the bytes that more than one run takes for each one's sums (and the
// totals after them).
struct Runs {
  int64_t run, runs;
  size_t table, bytes;  // of counts (as of probabilities), in all
};
Runs runs_of(int64_t T, int64_t E) {
  int64_t run = (T + kMaxRuns - 1) / kMaxRuns;
  if (run < kMinRun) run = kMinRun;
  if (run > kMaxRun) run = kMaxRun;
  // (three launches take longer than one workgroup's few rounds)
  if (T <= kOneRun && E <= 512) run = T;
  Runs r{run, run > 0 ? (T + run - 1) / run : 0, 0, 0};
  if (r.runs > 1) {
    r.table = (size_t(r.runs + 1) * E * 4 + 255) & ~size_t(255);
    r.bytes = 2 * r.table + size_t(r.runs) * 8;
  }
  return r;
}

// Room for the runs' sums out of the library's scratch.
void* run_scratch(size_t bytes, void* stream, bitsmoe_status* st) {
  // A graph would keep the address, which a later, larger call of any operator that uses this scratch frees.
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  const hipError_t e = hipStreamIsCapturing(static_cast<hipStream_t>(stream), &capture);
  if (e != hipSuccess) {
    *st = device_error("route: hipStreamIsCapturing", e);
    return nullptr;
  }
  if (capture != hipStreamCaptureStatusNone) {
    *st = fail(BITSMOE_ERR_ARG, "route: under graph capture this many rows need bitsmoe_route_ws");
    return nullptr;
  }
  return scratch(kScratchMisc, bytes, stream, st);
}

// Both forms of the call: with a workspace, or (`own`) out of the library's scratch.
bitsmoe_status run_route(const char* who, const void* logits_dev, bitsmoe_dtype lt, int64_t T, int64_t E, int64_t ld,
                         int64_t k, const uint8_t* valid_dev, int renorm, int32_t* experts_dev, float* weights_dev,
                         int32_t* counts_dev, int32_t* offsets_dev, int32_t* rows_dev, int32_t* slots_dev,
                         float* lse_dev, float* losses_dev, bool own, void* work_dev, int64_t work_bytes,
                         void* stream) {
  if (bitsmoe_status st = check(who, logits_dev, lt, T, E, ld, k)) return st;
  if (!counts_dev || !offsets_dev || !losses_dev ||
      (T > 0 && (!experts_dev || !weights_dev || !rows_dev || !slots_dev || !lse_dev)))
    return fail(BITSMOE_ERR_ARG, std::string(who) + ": null pointer");
  if (!aligned16({logits_dev, experts_dev, weights_dev, counts_dev, offsets_dev, rows_dev, slots_dev, lse_dev,
                  losses_dev}))
    return fail(BITSMOE_ERR_ARG, std::string(who) + ": device pointers must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (T == 0) {
    route_none_kernel<<<1, 256, 0, s>>>(static_cast<int>(E), counts_dev, offsets_dev, losses_dev);
    BITSMOE_LAUNCH_CHECK("route_none_kernel");
    return ok();
  }
  RouteArgs a{};
  a.logits = logits_dev;
  a.ld = ld;
  a.T = T;
  a.E = static_cast<int>(E);
  a.k = static_cast<int>(k);
  a.renorm = renorm != 0;
  a.wide = wide_rows(logits_dev, lt, E, ld);
  a.valid = valid_dev;
  a.experts = experts_dev;
  a.weights = weights_dev;
  a.counts = counts_dev;
  a.offsets = offsets_dev;
  a.rows = rows_dev;
  a.slots = slots_dev;
  a.lse = lse_dev;
  a.losses = losses_dev;
  const Runs cut = runs_of(T, E);
  const int64_t run = cut.run, runs = cut.runs;
  a.run = static_cast<int>(run);
  a.runs = static_cast<int>(runs);
  if (runs > 1) {
    bitsmoe_status st = BITSMOE_OK;
    char* p = static_cast<char*>(own ? run_scratch(cut.bytes, stream, &st) : work_dev);
    if (st) return st;
    if (!own && (!p || work_bytes < static_cast<int64_t>(cut.bytes) || !aligned16({p})))
      return fail(BITSMOE_ERR_ARG, std::string(who) + ": the workspace is missing, too small or misaligned");
    a.run_counts = reinterpret_cast<int32_t*>(p);
    a.run_probs = reinterpret_cast<float*>(p + cut.table);
    a.run_z = reinterpret_cast<float*>(p + 2 * cut.table);
    a.run_n = reinterpret_cast<int32_t*>(a.run_z + runs);
  }
  bitsmoe_status st = BITSMOE_OK;
  with_layout(E, [&](auto v, auto l) {
    constexpr int V = decltype(v)::value, LPT = decltype(l)::value;
    constexpr int MANY = V == 8 ? kThreads : 256;
    const bool small = T <= kMinRun;  // (a workgroup that is launched sooner)
    const int nt = small ? 256 : MANY;
    const size_t lds = size_t(nt) * V * 4 + (E + 1) * 4 + size_t(nt / LPT) * k * 4 + nt / 64 * 4 +
                       (runs == 1 ? size_t(run * k + run + 1 + E * ((run + 31) / 32)) * 4 : 0);
    auto* fn = lt == BITSMOE_BF16
                   ? (small ? route_rows_kernel<true, V, LPT, 256> : route_rows_kernel<true, V, LPT, MANY>)
                   : (small ? route_rows_kernel<false, V, LPT, 256> : route_rows_kernel<false, V, LPT, MANY>);
    if (lds > 65536) {
      static std::atomic<uint64_t> allowed[4];
      st = allow_lds(reinterpret_cast<const void*>(fn), kMostLds, &allowed[2 * (lt == BITSMOE_BF16) + small]);
      if (st) return;
    }
    fn<<<static_cast<unsigned>(runs), nt, lds, s>>>(a);
  });
  if (st) return st;
  BITSMOE_LAUNCH_CHECK("route_rows_kernel");
  if (runs > 1) {
    route_sum_kernel<<<static_cast<unsigned>((E + 31) / 32), 1024, 0, s>>>(a);
    BITSMOE_LAUNCH_CHECK("route_sum_kernel");
    const size_t lds = size_t(E + 1 + kThreads / 64 + run + 1 + E * ((run + 31) / 32)) * 4;
    if (lds > 65536) {
      static std::atomic<uint64_t> allowed{0};
      st = allow_lds(reinterpret_cast<const void*>(route_place_kernel), kMostLds, &allowed);
      if (st) return st;
    }
    route_place_kernel<<<static_cast<unsigned>(runs + 1), kThreads, lds, s>>>(a);
    BITSMOE_LAUNCH_CHECK("route_place_kernel");
  }
  return ok();
}

}  // namespace
}  // namespace bitsmoe

using namespace bitsmoe;

extern "C" int64_t bitsmoe_route_workspace(int64_t T, int64_t E) {
  if (T <= 0 || T >= (int64_t(1) << 31) || E <= 0 || E > kMaxExperts) return 0;
  return static_cast<int64_t>(runs_of(T, E).bytes);
}

extern "C" bitsmoe_status bitsmoe_route_ws(const void* logits_dev, bitsmoe_dtype lt, int64_t T, int64_t E, int64_t ld,
                                           int64_t k, const uint8_t* valid_dev, int renorm, int32_t* experts_dev,
                                           float* weights_dev, int32_t* counts_dev, int32_t* offsets_dev,
                                           int32_t* rows_dev, int32_t* slots_dev, float* lse_dev, float* losses_dev,
                                           void* work_dev, int64_t work_bytes, void* stream) {
  return run_route("route_ws", logits_dev, lt, T, E, ld, k, valid_dev, renorm, experts_dev, weights_dev, counts_dev,
                   offsets_dev, rows_dev, slots_dev, lse_dev, losses_dev, false, work_dev, work_bytes, stream);
}

extern "C" bitsmoe_status bitsmoe_route(const void* logits_dev, bitsmoe_dtype lt, int64_t T, int64_t E,
                                        int64_t ld, int64_t k, const uint8_t* valid_dev, int renorm,
                                        int32_t* experts_dev, float* weights_dev, int32_t* counts_dev,
                                        int32_t* offsets_dev, int32_t* rows_dev, int32_t* slots_dev,
                                        float* lse_dev, float* losses_dev, void* stream) {
  return run_route("route", logits_dev, lt, T, E, ld, k, valid_dev, renorm, experts_dev, weights_dev, counts_dev,
                   offsets_dev, rows_dev, slots_dev, lse_dev, losses_dev, true, nullptr, 0, stream);
}

extern "C" bitsmoe_status bitsmoe_route_grad(const void* logits_dev, bitsmoe_dtype lt, int64_t T, int64_t E,
                                             int64_t ld, int64_t k, int renorm, const int32_t* experts_dev,
                                             const float* weights_dev, const int32_t* counts_dev,
                                             const float* lse_dev, const float* dweights_dev,
                                             const float* dlosses_dev, void* dlogits_dev, void* stream) {
  if (bitsmoe_status st = check("route_grad", logits_dev, lt, T, E, ld, k)) return st;
  if (T == 0) return ok();
  if (!experts_dev || !weights_dev || !counts_dev || !lse_dev || !dlogits_dev)
    return fail(BITSMOE_ERR_ARG, "route_grad: null pointer");
  if (!aligned16({logits_dev, experts_dev, weights_dev, counts_dev, lse_dev, dweights_dev, dlosses_dev, dlogits_dev}))
    return fail(BITSMOE_ERR_ARG, "route_grad: device pointers must be 16-byte aligned");
  GradArgs a{};
  a.logits = logits_dev;
  a.ld = ld;
  a.T = T;
  a.E = static_cast<int>(E);
  a.k = static_cast<int>(k);
  a.renorm = renorm != 0;
  a.wide = wide_rows(logits_dev, lt, E, ld);
  a.experts = experts_dev;
  a.weights = weights_dev;
  a.counts = counts_dev;
  a.lse = lse_dev;
  a.dweights = dweights_dev;
  a.dlosses = dlosses_dev;
  a.dlogits = dlogits_dev;
  with_layout(E, [&](auto v, auto l) {
    constexpr int V = decltype(v)::value, LPT = decltype(l)::value;
    const int64_t groups = (T + kGradThreads / LPT - 1) / (kGradThreads / LPT);
    const unsigned grid = static_cast<unsigned>(groups < 8192 ? groups : 8192);
    auto* fn = lt == BITSMOE_BF16 ? route_grad_kernel<true, V, LPT> : route_grad_kernel<false, V, LPT>;
    fn<<<grid, kGradThreads, 0, static_cast<hipStream_t>(stream)>>>(a);
  });
  BITSMOE_LAUNCH_CHECK("route_grad_kernel");
  return ok();
}
