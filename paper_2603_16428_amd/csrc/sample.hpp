// A token for each row of logits, from a given random number: temperature, top-k, top-p, min-p.
//
// Weights exp((z - max) / T) are computed in 64 bits and added as 64-bit integers (fixed point: V logits have a unit of 2^-44 of the
// largest weight up to 2^18, 2^-50 up to 2^12; above 2^18 the unit follows from the row's logits, 2^-53 of their sum or 2^-50). A running
// sum is then off by less than 2^-25 of the kept weights together, half of the finest step of a number below 1: V half units, at most
// 2^-27, V 2^-50 for the tables' own rounding, and V 2^-45.8 for weights past the tables' end. Integer sums do not depend on their order, so counts and weights are gathered by
// LDS atomics, and everything that is looked for (the k-th largest, where top-p ends, which of several equal ones are still in,
// the token whose running sum passes u Z) is found the same way: 2048 bins over the range in question, a prefix sum, the bin
// where the target is reached, and again inside that bin until it is one value. Nothing is sorted.
//
// Two launches: parts of a row in parallel (the maximum of each group of 64 logits, sums of weights where the whole row's
// is needed), then a workgroup per row. Its settings and the groups' maxima give a bound that no kept logit is below: only
// groups above it are read again, and, where few logits pass, they are listed in LDS. Where top-p (or a top-k beyond the number of
// groups) may keep very many, each part also leaves a table of counts and weights by cells of T / 4: the cell where the target is
// reached is then known without reading the row, and only that cell's logits are listed.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops_row.hpp"

namespace lce {

constexpr int kSampleCells = 128;  // of a quarter of T: the last one's weights are 2^-46
constexpr int kSampleParts = 64, kPartGroups = 64, kMostGroups = kSampleParts * kPartGroups;
constexpr double kCellUnits = 0x1p49;  // of a table's weights: a part's 2^14 logits at most stay below 2^64

struct SampleArgs {
  const void* logits;
  int64_t ld;  // elements
  const float* u;
  float temperature, top_p, min_p;
  int top_k;
  const float *temperatures, *top_ps, *min_ps;  // of each row, or null
  const int32_t* top_ks;
  int64_t* tokens;
  float* logprobs;
  float *group_max, *part_max;  // [N][groups], [N][parts]
  double* part_sum;             // [N][parts], relative to the part's maximum
  uint64_t* cell_weight;        // [N][parts][cells], relative to the part's maximum (rows for which cells() is true)
  uint32_t* cell_count;
  int V, groups, parts, bits;   // bits: a weight of 1 is 2^bits
};

struct SampleRow {
  double rate;  // 256 log2(e) / T
  float T, p, least;
  int k;  // 0: all
  // cells: so many may be kept that their weights and counts are tabled.
  bool greedy, by_k, by_p, by_least, cells;
  __device__ __forceinline__ bool whole() const { return !by_k && !by_p && !by_least; }
  // Whether the sum of the whole row's weights is needed.
  __device__ __forceinline__ bool sums() const { return !greedy && (cells || (!by_k && (by_p || whole()))); }
};
__device__ __forceinline__ SampleRow sample_row(const SampleArgs& a, int64_t i) {
  SampleRow r;
  r.T = a.temperatures ? a.temperatures[i] : a.temperature;
  r.T = r.T > 1e30f ? 1e30f : r.T;  // (all weights are equal then, and no product below is 0 times infinity)
  r.p = a.top_ps ? a.top_ps[i] : a.top_p;
  r.least = fminf(a.min_ps ? a.min_ps[i] : a.min_p, 1.f);  // the largest is always kept
  r.k = a.top_ks ? a.top_ks[i] : a.top_k;
  r.greedy = !(r.T > 0.f);
  r.by_k = r.k > 0 && r.k < a.V;
  r.by_p = r.p < 1.f;
  r.by_least = r.least > 0.f;
  r.cells = !r.greedy && !r.by_least && (r.by_k ? r.k > a.groups : r.by_p);
  r.rate = 256.0 * 1.4426950408889634074 / (double)r.T;
  return r;
}

// exp from its argument times 256 log2(e): 2^(n / 256) from a table and the rest's series, whose next term is below 4e-17.
// (Far below the smallest weight that counts, so that infinities pass.)
__device__ __forceinline__ double sample_exp(double t, const double* table) {
  constexpr double c1 = 0.69314718055994530942 / 256, c2 = c1 * c1 / 2, c3 = c1 * c1 * c1 / 6, c4 = c1 * c1 * c1 * c1 / 24;
  t = fmax(t, -65536.0);
  const double n = rint(t), f = t - n;
  const int i = (int)n;
  return __builtin_ldexp(table[i & 255] * fma(f, fma(f, fma(f, fma(f, c4, c3), c2), c1), 1.0), i >> 8);
}
__device__ __forceinline__ void sample_table(double* table) {
  if (threadIdx.x < 256) table[threadIdx.x] = exp2((double)threadIdx.x / 256.0);
}
// The weight of z relative to `top`, 1 where they are equal (infinities too).
__device__ __forceinline__ double sample_weight(float z, float top, double rate, const double* table) {
  const double w = sample_exp(((double)z - (double)top) * rate, table);
  return z == top ? 1.0 : w;
}

// How many cells below the larger `top` z is, up to kSampleCells. Cells lie at multiples of T / 4, the same for every part.
__device__ __forceinline__ int sample_cell(float z, float top, double rate) {
  const double c = rate * (4.0 / (256.0 * 1.4426950408889634074));  // 4 / T
  const double d = floor((double)top * c) - floor((double)z * c);
  return z == top ? 0 : d < (double)kSampleCells ? (int)d : kSampleCells;
}

// The larger of two, and NaN if one is.
__device__ __forceinline__ float max_or_nan(float a, float b) { return (a >= b || a != a) ? a : b; }

// A workgroup for each part (64 groups): eight lanes a group, REP pieces of 8 logits each. 256 x 152064 in fp32, an eighth of the rows with
// tables and another with sums: 38 us (156 MB, 4.1 TB/s); one row of 128256 in bf16 3.4.
template <typename T, int REP, RowEnd END>
__global__ __launch_bounds__(256) void sample_parts_kernel(const SampleArgs a) {
  constexpr int kGroup = 64 * REP, kRounds = kPartGroups / 32;
  __shared__ double table[256], sums[4];
  __shared__ float tops[4];
  __shared__ unsigned long long cell_weight[kSampleCells];
  __shared__ uint32_t cell_count[kSampleCells];
  const int64_t i = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  const T* row = (const T*)a.logits + i * a.ld;
  const SampleRow set = sample_row(a, i);
  const bool summed = set.sums();
  RawRow<T> raw[kRounds][REP];
#pragma unroll
  for (int g = 0; g < kRounds; ++g)
#pragma unroll
    for (int r = 0; r < REP; ++r) {
      const int at = (part * kPartGroups + g * 32 + (int)threadIdx.x / 8) * kGroup + r * 64 + (threadIdx.x % 8) * kNormVec;
      raw[g][r].clear();
      load_raw<END>(row + at, a.V - at, raw[g][r]);
    }
  if (summed) sample_table(table);
  if (threadIdx.x < kSampleCells) cell_weight[threadIdx.x] = cell_count[threadIdx.x] = 0;
  float top = -INFINITY;
  auto count_of = [&](int g, int r) {  // logits of this piece
    return a.V - ((part * kPartGroups + g * 32 + (int)threadIdx.x / 8) * kGroup + r * 64 + ((int)threadIdx.x % 8) * kNormVec);
  };
#pragma unroll
  for (int g = 0; g < kRounds; ++g) {
    float m = -INFINITY;
#pragma unroll
    for (int r = 0; r < REP; ++r) {
      const int n = count_of(g, r);
      align_end<END>(n, raw[g][r]);
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) m = e < n ? max_or_nan(raw[g][r].at(e), m) : m;
    }
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) m = max_or_nan(__shfl_xor(m, o), m);
    const int group = part * kPartGroups + g * 32 + (int)threadIdx.x / 8;
    if (threadIdx.x % 8 == 0 && group < a.groups) a.group_max[i * a.groups + group] = m;
    top = max_or_nan(m, top);
  }
  if (!summed) return;
#pragma unroll
  for (int o = 8; o < 64; o <<= 1) top = max_or_nan(__shfl_xor(top, o), top);
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  top = max_or_nan(max_or_nan(tops[0], tops[1]), max_or_nan(tops[2], tops[3]));
  double sum = 0.0;
  if (top > -INFINITY) {
#pragma unroll
    for (int g = 0; g < kRounds; ++g)
#pragma unroll
      for (int r = 0; r < REP; ++r)
#pragma unroll
        for (int e = 0; e < kNormVec; ++e)
          if (e < count_of(g, r)) {
            const float z = raw[g][r].at(e);
            const double w = sample_weight(z, top, set.rate, table);
            sum += w;
            if (set.cells) {
              const int cell = sample_cell(z, top, set.rate);
              if (cell < kSampleCells) {
                atomicAdd(&cell_weight[cell], (unsigned long long)(uint64_t)fma(w, kCellUnits, 0.5));
                atomicAdd(&cell_count[cell], 1u);
              }
            }
          }
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    a.part_max[i * a.parts + part] = top;
    a.part_sum[i * a.parts + part] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  }
  if (set.cells && threadIdx.x < kSampleCells) {
    a.cell_weight[(i * a.parts + part) * kSampleCells + threadIdx.x] = cell_weight[threadIdx.x];
    a.cell_count[(i * a.parts + part) * kSampleCells + threadIdx.x] = cell_count[threadIdx.x];
  }
}

// ---- a row's token ----

// An order of the logits by integers, and back. 16-bit types use the bits that they have.
template <typename T>
struct SampleKey {
  static constexpr int kShift = sizeof(T) == 4 ? 0 : std::is_same_v<T, bf16> ? 16 : 13;
  static __device__ __forceinline__ uint32_t of(float z) {
    const uint32_t b = __builtin_bit_cast(uint32_t, z + 0.f);  // (-0 is 0)
    return (b >> 31 ? ~b : b | 0x80000000u) >> kShift;
  }
  static __device__ __forceinline__ float value(uint32_t key) {
    const uint32_t b = key << kShift;
    return __builtin_bit_cast(float, b >> 31 ? b & 0x7fffffffu : ~(b | ((1u << kShift) - 1u)));
  }
};

constexpr int kSampleThreads = 1024, kSampleBins = 2 * kSampleThreads, kSampleList = 8192, kSampleFew = 256;

struct SampleFound {
  int bin;  // -1: the target is not reached
  uint32_t before, count;
  uint64_t weight_before, weight, weight_all;
};
struct SampleLds {
  double table[256];
  unsigned long long weight[kSampleBins];
  uint32_t count[kSampleBins];
  uint32_t list_key[kSampleList], list_at[kSampleList];
  uint16_t active[kMostGroups];
  uint64_t wave_weight[16];
  uint32_t wave_count[16];
  float wave_max[16], wave_least[16];
  uint32_t actives, listed, lowest;
  unsigned long long kept, all;
  SampleFound found;
};

// Sums over a wave's lanes up to and with each one, by lane moves within the vector unit (a shuffle through LDS is ten times as long, and
// what one row waits for is the chain of these).
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <typename F>
__device__ __forceinline__ void for_row_steps(F f) {
  using std::integral_constant;
  f(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // row_shr:1, 2, 4, 8: within 16 lanes
  f(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  f(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  f(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
}
template <typename F>
__device__ __forceinline__ void for_scan_steps(F f) {
  using std::integral_constant;
  for_row_steps(f);
  f(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // row_bcast:15, 31: the rows before
  f(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t moved(uint64_t v) {
  return (uint64_t)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v);
}
template <typename V>
__device__ __forceinline__ V wave_scan(V v) {
  for_scan_steps([&](auto c, auto r) { v += moved<decltype(c)::value, decltype(r)::value>(v); });
  return v;
}
template <typename V>
__device__ __forceinline__ V row_scan(V v) {
  for_row_steps([&](auto c, auto r) { v += moved<decltype(c)::value, decltype(r)::value>(v); });
  return v;
}
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ uint64_t lane_of(uint64_t v, int lane) { return (uint64_t)lane_of((uint32_t)(v >> 32), lane) << 32 | lane_of((uint32_t)v, lane); }
// The wave's largest (a NaN if there is one), for all lanes.
__device__ __forceinline__ float wave_max(float v) {
  for_scan_steps([&](auto c, auto r) {
    const int b = __builtin_bit_cast(int, v);  // (lanes without a partner take their own)
    v = max_or_nan(__builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, decltype(c)::value, decltype(r)::value, 0xf, false)), v);
  });
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

__device__ __forceinline__ void sample_clear(SampleLds& s) {
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    s.weight[threadIdx.x + k * kSampleThreads] = 0;
    s.count[threadIdx.x + k * kSampleThreads] = 0;
  }
  __syncthreads();
}

// The first bin with which the counts reach `count` or the weights `weight` (u >= 0: the first whose running weight is above u
// times the whole). All threads, after their additions to the bins.
__device__ __forceinline__ SampleFound sample_find(SampleLds& s, uint32_t count, uint64_t weight, double u = -1.0) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), b = 2 * threadIdx.x;
  __syncthreads();
  if (threadIdx.x == 0) s.found.bin = -1;
  const uint32_t c0 = s.count[b], c1 = s.count[b + 1];
  const uint64_t w0 = s.weight[b], w1 = s.weight[b + 1];
  uint32_t c = wave_scan(c0 + c1);
  uint64_t w = wave_scan(w0 + w1);
  if (lane == 63) {
    s.wave_count[wave] = c;
    s.wave_weight[wave] = w;
  }
  __syncthreads();
  // The sums of the waves before, and of all, from 16 lanes' scan.
  const uint32_t upto_c = row_scan(s.wave_count[lane & 15]);
  const uint64_t upto_w = row_scan(s.wave_weight[lane & 15]);
  const uint64_t all_w = lane_of(upto_w, 15);
  if (wave > 0) {
    c += lane_of(upto_c, wave - 1);
    w += lane_of(upto_w, wave - 1);
  }
  if (u >= 0.0) {
    weight = (uint64_t)(fmin(u, 1.0) * (double)all_w) + 1;
    weight = weight > all_w ? all_w : weight;
  }
  c -= c0 + c1;
  w -= w0 + w1;
  auto reached = [&](uint32_t cc, uint64_t ww) { return cc >= count || ww >= weight; };
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const uint32_t ck = k ? c1 : c0;
    const uint64_t wk = k ? w1 : w0;
    if (!reached(c, w) && reached(c + ck, w + wk)) s.found = {b + k, c, ck, w, wk, all_w};
    c += ck;
    w += wk;
  }
  __syncthreads();
  SampleFound f = s.found;
  f.weight_all = all_w;
  return f;
}

// Bits by which a span of values is shifted to fall into the bins.
__device__ __forceinline__ int sample_shift(uint32_t span) { return span < (uint32_t)kSampleBins ? 0 : 21 - __builtin_clz(span); }
static_assert(kSampleBins == 1 << 11, "sample_shift");

// A workgroup a row. All paths share the 128 registers that 1024 threads leave a lane, and 200 to 300 bytes of each lane's are spilled; how
// much of a row's time that is, beside its chain of searches (a barrier or two and a read of cold code each), was not measured. The largest logit 3.4 us,
// top-k 50 with top-p 17, the whole distribution 11, top-p alone 29 (128256 logits in bf16); 256 rows of 152064 with settings of their own 47,
// the slowest of them. (Each search in one place and loops over logits rolled up: 40 KB of code; 125 KB unrolled took 30 us
// for top-k and 70 for the 256 rows.)
template <typename T, int REP, RowEnd END>
__global__ __launch_bounds__(kSampleThreads) void sample_row_kernel(const SampleArgs a) {
  using Key = SampleKey<T>;
  constexpr int kGroup = 64 * REP, kEach = kMostGroups / kSampleThreads;
  __shared__ SampleLds s;
  const int tid = threadIdx.x;
  const int64_t i = blockIdx.x;
  const T* row = (const T*)a.logits + i * a.ld;
  const SampleRow set = sample_row(a, i);
  const float u = a.u[i];
  float maxima[kEach];
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int g = tid + k * kSampleThreads;
    maxima[k] = g < a.groups ? a.group_max[i * a.groups + g] : -INFINITY;
  }
  sample_table(s.table);
  if (tid == 0) {
    s.actives = s.listed = 0;
    s.lowest = ~0u;
  }
  // The largest, and the least above -inf.
  float top = -INFINITY, least = INFINITY;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    top = max_or_nan(maxima[k], top);
    if (maxima[k] > -INFINITY) least = fminf(least, maxima[k]);
  }
  top = wave_max(top);
  least = -wave_max(-least);
  if ((tid & 63) == 0) {
    s.wave_max[tid >> 6] = top;
    s.wave_least[tid >> 6] = least;
  }
  __syncthreads();
  top = wave_max(s.wave_max[tid & 15]);
  least = -wave_max(-s.wave_least[tid & 15]);
  auto answer = [&](int64_t token, float logprob) {
    if (tid == 0) {
      a.tokens[i] = token;
      if (a.logprobs != nullptr) a.logprobs[i] = logprob;
    }
  };
  // A NaN among the logits or for u, or nothing above -inf.
  if (!(top > -INFINITY) || u != u) return answer(-1, __builtin_nanf(""));

  // The logits of a range of places, by single loads, four requested at once.
  constexpr uint32_t kAtOnce = 4;
  auto range = [&](uint32_t lo, uint32_t n, auto f) {
    for (uint32_t k = tid; k < n; k += kAtOnce * kSampleThreads) {
      float z[kAtOnce];
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) z[q] = to_f32(row[min(lo + k + q * kSampleThreads, (uint32_t)a.V - 1)]);
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q)
        if (k + q * kSampleThreads < n && lo + k + q * kSampleThreads < (uint32_t)a.V) f(Key::of(z[q]), z[q], lo + k + q * kSampleThreads);
    }
  };

  if (set.greedy) {
    uint32_t g0 = ~0u;
#pragma unroll
    for (int k = kEach - 1; k >= 0; --k)
      if (maxima[k] == top) g0 = tid + k * kSampleThreads;
    if (g0 != ~0u) atomicMin(&s.lowest, g0);
    __syncthreads();
    g0 = s.lowest;
    __syncthreads();
    if (tid == 0) s.lowest = ~0u;
    __syncthreads();
    range(g0 * kGroup, kGroup, [&](uint32_t, float z, uint32_t at) {
      if (z == top) atomicMin(&s.lowest, at);
    });
    __syncthreads();
    return answer(s.lowest, 0.f);
  }

  // The unit of the weights: all of them together stay below 2^63, one below 2^51.
  int bits = a.bits;
  if constexpr (REP > 1) {
    // For very many logits the worst case's unit (all are equal) is too coarse for a tail below few large ones (2^20 weights of a
    // 2^43rd each are 2^-23 of the large one): the groups' maxima say how large the sum can be, to a factor of the groups' length.
    uint64_t most = 0;  // 2^-20ths
#pragma unroll
    for (int k = 0; k < kEach; ++k) most += (uint64_t)(sample_weight(maxima[k], top, set.rate, s.table) * (kGroup * 0x1p20)) + 1;
    most = wave_scan(most);
    if ((tid & 63) == 63) s.wave_weight[tid >> 6] = most;
    __syncthreads();
    most = lane_of(row_scan(s.wave_weight[tid & 15]), 15);
    bits = min(50, 82 - (64 - __builtin_clzll(most)));
  }
  const double one = __builtin_ldexp(1.0, bits);
  // A weight in fixed point: below 2^52, so that adding 2^52 rounds it to an integer in the low bits.
  auto in_units = [](double w, double n) { return __builtin_bit_cast(uint64_t, fma(w, n, 0x1p52)) - __builtin_bit_cast(uint64_t, 0x1p52); };
  auto fixed = [&](double w) { return in_units(w, one); };
  auto logprob = [&](uint32_t at, double sum) {
    const float z = to_f32(row[at]);
    return (float)((z == top ? 0.0 : ((double)z - (double)top) / (double)set.T) - log(sum));
  };
  const double chance = u > 0.f ? (double)u : 0.0;

  // Falling logits, equal ones by their places: place and key in one number. Kept are those from `cut` on.
  auto rank = [](uint32_t key, uint32_t at) { return (uint64_t)key << 32 | (0xffffffffu - at); };
  uint64_t cut = 0;
  int cell = -1;  // the listed logits' cell, the last of which some are kept (-1: no cell)
  // Where the token is known to lie: the part in which the parts' running weight passes `chance`.
  SampleFound part;
  part.bin = -1;
  // The whole row's weight from its parts'.
  double sum = 0.0;
  if (set.sums()) {
    sample_clear(s);
    if (tid < a.parts) {
      const double w = a.part_sum[i * a.parts + tid] * sample_weight(a.part_max[i * a.parts + tid], top, set.rate, s.table);
      s.weight[tid] = (uint64_t)(w * one + 0.5);
    }
    part = sample_find(s, ~0u, 0, chance);
    sum = (double)part.weight_all / one;
    if (!set.whole()) part.bin = -1;
  }

  auto weight = [&](float z) { return sample_weight(z, top, set.rate, s.table); };
  // No kept logit that is looked for is below `bound`.
  float bound = -INFINITY;
  int actives = 0;
  uint32_t listed = 0;
  // The logits of the active groups that are not below the bound: eight lanes a group, four groups requested at once.
  auto stream = [&](auto f) {
    constexpr int kAhead = 4, kGroups = kSampleThreads / 8;
    for (int k0 = tid / 8; k0 < actives; k0 += kAhead * kGroups) {
#pragma unroll
      for (int r = 0; r < REP; ++r) {
        RawRow<T> raw[kAhead];
        int at[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
          at[q] = (int)s.active[min(k0 + q * kGroups, actives - 1)] * kGroup + r * 64 + (tid % 8) * kNormVec;
          raw[q].clear();
          load_raw<END>(row + at[q], a.V - at[q], raw[q]);
        }
#pragma unroll
        for (int q = 0; q < kAhead; ++q) align_end<END>(a.V - at[q], raw[q]);
        // One after the other out of the registers' front: unrolled, these loops are 100 KB of code that a single row
        // waits for.
#pragma nounroll
        for (int e = 0; e < kNormVec; ++e) {
#pragma unroll
          for (int q = 0; q < kAhead; ++q) {
            const float z = raw[q].at(0);
            if (k0 + q * kGroups < actives && at[q] + e < a.V && z >= bound) f(Key::of(z), z, (uint32_t)(at[q] + e));
            raw[q].drop(1);
          }
        }
      }
    }
  };
  // Lists the logits that are not below the bound (those of the cell alone).
  auto list = [&]() {
    __syncthreads();
    if (tid == 0) s.actives = s.listed = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (maxima[k] >= bound && tid + k * kSampleThreads < a.groups) s.active[atomicAdd(&s.actives, 1u)] = (uint16_t)(tid + k * kSampleThreads);
    __syncthreads();
    actives = (int)s.actives;
    stream([&](uint32_t key, float z, uint32_t at) {
      if (cell >= 0 && sample_cell(z, top, set.rate) != cell) return;
      const uint32_t k = atomicAdd(&s.listed, 1u);
      if (k < (uint32_t)kSampleList) {
        s.list_key[k] = key;
        s.list_at[k] = at;
      }
    });
    __syncthreads();
    listed = s.listed;
  };
  auto each = [&](auto f) {
    if (listed <= (uint32_t)kSampleList) {
      for (uint32_t k = tid; k < listed; k += kSampleThreads) f(s.list_key[k], Key::value(s.list_key[k]), s.list_at[k]);
    } else {
      stream(f);
    }
  };
  // (with room for the rounding of these bounds)
  auto below = [&](double b) { return (float)(b - 1e-6 * fabs(b) - 1e-6 * (double)set.T); };
  auto bound_of = [&](double w) { return below((double)top + (double)set.T * log(w)); };  // logits below it weigh less than w
  auto find_bound = [&]() {
    bound = -INFINITY;
    if (set.by_k && set.k <= a.groups && top < INFINITY) {
      // The k-th largest of the groups' maxima: k logits at least are as large. It is no smaller than the end of its bin.
      const float inv = top > least ? (float)(kSampleBins - 1) / (top - least) : 0.f;
      if (inv < INFINITY && top - least < INFINITY) {
        sample_clear(s);
#pragma unroll
        for (int k = 0; k < kEach; ++k)
          if (maxima[k] > -INFINITY) atomicAdd(&s.count[min((int)((top - maxima[k]) * inv), kSampleBins - 1)], 1u);
        const SampleFound f = sample_find(s, (uint32_t)set.k, ~0ull);
        if (f.bin >= 0) bound = inv > 0.f ? top - ((float)(f.bin + 1) / inv * (1.f + 0x1p-20f) + fabsf(top) * 0x1p-22f) : top;
      }
    }
    if (set.by_least && !(set.by_k && set.by_p)) bound = fmaxf(bound, bound_of((double)set.least));
    // Those below (1 - p) Z / V together weigh less than (1 - p) Z.
    if (set.by_p && set.p <= 0.f) bound = top;
    else if (set.by_p && !set.by_k) bound = fmaxf(bound, bound_of((1.0 - (double)set.p) * sum / (double)a.V));
  };
  auto share_of = [&](double whole) {  // top-p's weight
    const double target = ceil((double)set.p * whole);
    return target >= 1.0 ? (uint64_t)target : (uint64_t)1;
  };

  // Few logits: every one looks at all others, whose number is shared out among as many threads as there are.
  auto few = [&]() {
    int slots = 64;
    while (slots < (int)listed) slots *= 2;
    const int me = tid % slots, segment = tid / slots, segments = kSampleThreads / slots;
    const bool mine = me < (int)listed;
    unsigned long long *w_of = s.weight, *before_of = w_of + kSampleFew, *kept_of = before_of + kSampleFew, *up_to_of = kept_of + kSampleFew;
    const uint32_t key = mine ? s.list_key[me] : 0u, at = mine ? s.list_at[me] : ~0u;
    const double share = mine ? weight(Key::value(key)) : 0.0;
    const uint64_t w = fixed(share), order = rank(key, at);
    if (segment == 0) {
      w_of[me] = mine ? w : 0;
      before_of[me] = up_to_of[me] = 0;
      s.count[me] = 0;
    }
    if (tid == 0) s.kept = s.all = 0;
    __syncthreads();
    uint64_t before = 0;
    uint32_t ahead = 0;
    for (int k = segment; k < (int)listed; k += segments) {
      const bool first = rank(s.list_key[k], s.list_at[k]) > order;
      before += first ? w_of[k] : 0;
      ahead += first;
    }
    if (mine) {
      atomicAdd(&before_of[me], (unsigned long long)before);
      atomicAdd(&s.count[me], ahead);
    }
    __syncthreads();
    bool kept = mine && (!set.by_k || s.count[me] < (uint32_t)set.k);
    if (kept && segment == 0) atomicAdd(&s.kept, (unsigned long long)w);
    __syncthreads();
    if (set.by_p) kept = kept && before_of[me] < share_of(set.by_k ? (double)s.kept : sum * one);
    if (set.by_least) kept = kept && share >= (double)set.least;
    if (segment == 0) {
      kept_of[me] = kept ? w : 0;
      if (kept) atomicAdd(&s.all, (unsigned long long)w);
    }
    __syncthreads();
    uint64_t up_to = 0;
    for (int k = segment; k < (int)listed; k += segments) up_to += s.list_at[k] <= at ? kept_of[k] : 0;
    if (kept) atomicAdd(&up_to_of[me], (unsigned long long)up_to);
    __syncthreads();
    const uint64_t all = s.all;
    uint64_t target = (uint64_t)(fmin(chance, 1.0) * (double)all) + 1;
    target = target > all ? all : target;
    if (kept && segment == 0 && up_to_of[me] >= target && up_to_of[me] - w < target) {
      a.tokens[i] = at;
      if (a.logprobs != nullptr) a.logprobs[i] = logprob(at, (double)all / one);
    }
  };

  // Makes the cut at the smallest beginning of that order with `count` logits or a weight of `target`, of which `before` and
  // `weight_before` are not among those listed; returns its weight.
  auto keep = [&](uint32_t count, uint64_t target, uint32_t before, uint64_t weight_before) {
    const bool weighed = target != ~0ull || set.by_p;
    uint32_t hi = Key::of(top), lo = Key::of(bound), equal = 0;
    for (bool first = true;; first = false) {
      const int shift = sample_shift(hi - lo);
      sample_clear(s);
      each([&](uint32_t key, float z, uint32_t at) {
        if (key < lo || key > hi || rank(key, at) < cut) return;
        // Lanes with the first one's logit add as one: many equal logits would queue up at their bin (128256 of them 640 us).
        const uint64_t same = __ballot(key == (uint32_t)__builtin_amdgcn_readfirstlane((int)key));
        const bool alike = (same >> (tid & 63)) & 1;
        const uint32_t first_of = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
        if (alike && first_of != 0) return;
        const uint32_t times = alike ? (uint32_t)__popcll(same) : 1u;
        atomicAdd(&s.count[(hi - key) >> shift], times);
        if (weighed) {
          const uint64_t w = fixed(weight(z)) * times;
          if (w != 0) atomicAdd(&s.weight[(hi - key) >> shift], (unsigned long long)w);
        }
      });
      const SampleFound f = sample_find(s, count == ~0u ? ~0u : count - before, target == ~0ull ? ~0ull : target - weight_before);
      if (f.bin < 0) return weight_before + f.weight_all;  // (the first time alone: all are kept)
      before += f.before;
      weight_before += f.weight_before;
      equal = f.count;
      hi -= (uint32_t)f.bin << shift;
      if (shift == 0) break;
      lo = max(lo, hi - ((1u << shift) - 1u));
    }
    const uint64_t w = fixed(weight(Key::value(hi)));
    uint64_t of_equal = count != ~0u ? count - before : (target - weight_before + w - 1) / w;
    uint32_t last = 0xffffffffu;  // place of the last of the equal ones that is kept
    if (of_equal < equal) {
      uint32_t from = 0, n = (uint32_t)a.V, left = (uint32_t)of_equal;
      for (;;) {
        const int shift = sample_shift(n - 1);
        sample_clear(s);
        each([&](uint32_t key, float, uint32_t at) {
          if (key == hi && at - from < n && rank(key, at) >= cut) atomicAdd(&s.count[(at - from) >> shift], 1u);
        });
        const SampleFound f = sample_find(s, left, ~0ull);
        left -= f.before;
        from += (uint32_t)f.bin << shift;
        n = min(n - ((uint32_t)f.bin << shift), 1u << shift);
        if (shift == 0) break;
      }
      last = from;
    } else {
      of_equal = equal;
    }
    const uint64_t from_here = rank(hi, last);
    cut = cut > from_here ? cut : from_here;  // (all of the equal ones that an earlier cut left)
    return weight_before + of_equal * w;
  };
  // The parts' tables: f(part, the row's cell, count, weight).
  auto tables = [&](auto f) {
    for (int k = tid; k < a.parts * kSampleCells; k += kSampleThreads) {
      const int part = k / kSampleCells;
      const int64_t at = (i * a.parts + part) * kSampleCells + k % kSampleCells;
      const uint32_t n = a.cell_count[at];
      const uint64_t w = a.cell_weight[at];
      const float of = a.part_max[i * a.parts + part];
      const int c = sample_cell(of, top, set.rate) + k % kSampleCells;
      if (n != 0 && c < kSampleCells) f(part, c, n, (uint64_t)((double)w * (1.0 / kCellUnits) * weight(of) * one + 0.5));
    }
  };
  bool by_cells = set.cells, ready = false;
  const double of_row = sum;
#pragma nounroll
  for (int what = set.whole() ? 2 : 0; what < 2; ++what) {  // top-k, then top-p
    const bool wanted = what == 0 ? set.by_k : set.by_p;
    if (!wanted && (by_cells || ready)) continue;
    const uint32_t count = what == 0 ? (uint32_t)set.k : ~0u;
    const uint64_t target = what == 0 ? ~0ull : share_of(sum * one);
    uint32_t before = 0;
    uint64_t weight_before = 0;
    if (by_cells) {
      sample_clear(s);
      tables([&](int, int c, uint32_t n, uint64_t w) {
        atomicAdd(&s.count[c], n);
        atomicAdd(&s.weight[c], (unsigned long long)w);
      });
      const SampleFound f = sample_find(s, count, target);
      if (f.bin < 0) continue;  // all weights that count are kept
      before = f.before;
      weight_before = f.weight_before;
      cell = f.bin;
      const double c = set.rate * (4.0 / (256.0 * 1.4426950408889634074));
      bound = top < INFINITY ? below((floor((double)top * c) - cell) / c) : top;
    } else if (!ready) {
      find_bound();
    }
    if (by_cells || !ready) list();
    if (by_cells && listed > (uint32_t)kSampleList) {  // too many logits in one cell: the long way
      by_cells = false;
      cell = -1;
      cut = 0;
      sum = of_row;
      what = -1;
      continue;
    }
    if (!by_cells && !ready && listed <= (uint32_t)kSampleFew) return few();
    ready = true;
    if (!wanted) continue;
    const uint64_t kept = keep(count, target, before, weight_before);
    if (what == 0) sum = (double)kept / one;
  }
  if (by_cells) {
    sample_clear(s);
    tables([&](int of, int c, uint32_t, uint64_t w) {
      if (cell < 0 || c < cell) atomicAdd(&s.weight[of], (unsigned long long)w);
    });
    if (cell >= 0)
      for (uint32_t k = tid; k < listed; k += kSampleThreads)
        if (rank(s.list_key[k], s.list_at[k]) >= cut)
          atomicAdd(&s.weight[s.list_at[k] / (kPartGroups * kGroup)], (unsigned long long)fixed(weight(Key::value(s.list_key[k]))));
    part = sample_find(s, ~0u, 0, chance);
  }

  // The token of all kept ones, or of a part's (in weights relative to the part's own maximum): where the running weight by places passes
  // `share` times the whole; again inside the bin that it lies in, until that is one place.
  const bool inside = part.bin >= 0;
  const float of = inside ? a.part_max[i * a.parts + part.bin] : top;
  uint32_t lo = inside ? (uint32_t)part.bin * kPartGroups * kGroup : 0u;
  uint32_t n = inside ? min((uint32_t)(kPartGroups * kGroup), (uint32_t)a.V - lo) : (uint32_t)a.V;
  double share = fmin(chance, 1.0);
  if (inside) share = fmin(fmax((share * (double)part.weight_all - (double)part.weight_before) / (double)part.weight, 0.0), 1.0);
  // (a part's logits, each at most its largest, may have a finer unit than the row's, and must have room in theirs)
  constexpr double kInside = REP == 4 ? 0x1p48 : 0x1p49;
  const double unit = REP > 1 && inside ? kInside : one;
  uint64_t target = 0, whole = part.weight_all;
  bool first = true;
#pragma nounroll
  for (int shift = 1; shift > 0; first = false) {
    shift = sample_shift(n - 1);
    sample_clear(s);
    auto add = [&](uint32_t key, float z, uint32_t place) {
      if (place - lo >= n || z < bound || rank(key, place) < cut || (cell >= 0 && sample_cell(z, top, set.rate) > cell)) return;
      if (set.by_least && weight(z) < (double)set.least) return;
      const uint64_t w = in_units(sample_weight(z, of, set.rate, s.table), unit);
      if (w != 0) atomicAdd(&s.weight[(place - lo) >> shift], (unsigned long long)w);
    };
    if (first && !inside) each(add);
    else range(lo, n, add);
    const SampleFound f = sample_find(s, ~0u, target, first ? share : -1.0);
    if (first) {
      target = (uint64_t)(share * (double)f.weight_all) + 1;
      target = target > f.weight_all ? f.weight_all : target;
      if (!inside) whole = f.weight_all;
    }
    if (f.bin < 0) break;  // (no weight at all, which the kept ones' largest rules out)
    target -= f.weight_before;
    lo += (uint32_t)f.bin << shift;
    n = min(n - ((uint32_t)f.bin << shift), 1u << shift);
  }
  answer(lo, logprob(lo, (double)whole / one));
}

}  // namespace lce
