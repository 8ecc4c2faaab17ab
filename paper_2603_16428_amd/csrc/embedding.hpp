// Rows of a V x H matrix by token, and the gradient: for each token the sum of its rows of the upstream gradient.
//
// The gradient's sums run over the tokens' positions in order. The positions are sorted by token (stably, so a
// token's stay in order): tiles of 4096 in LDS, then up to 16 sorted runs at a time merged by rank. The sorted list is cut into
// chunks of a fixed length, whatever the tokens are: a frequent token's rows are spread over many workgroups and rare
// ones share one. A token whose positions lie in one chunk is written at once; one that goes on into other chunks
// leaves fp32 sums, which a last kernel adds in order. No atomics: the order of every sum is fixed by the tokens.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ops_row.hpp"

namespace lce {

__device__ __forceinline__ int64_t token_at(const void* tokens, int wide, int64_t i) {
  return wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

struct EmbedArgs {
  const void *tokens, *weight;
  void* out;
  int64_t weight_ld, out_ld;  // elements
  int64_t N, V;
  int H, wide;
  float scale;
};

// TPR threads a row, two pieces of 8 values requested at once by each.
template <typename T, int TPR, RowEnd END>
__global__ __launch_bounds__(256) void embedding_kernel(const EmbedArgs a) {
  constexpr int kRows = 256 / TPR, kAhead = 2;
  const int t = threadIdx.x % TPR;
  for (int64_t i = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; i < a.N; i += (int64_t)gridDim.x * kRows) {
    const int64_t v = token_at(a.tokens, a.wide, i);
    const bool known = v >= 0 && v < a.V;
    const T* p = (const T*)a.weight + (known ? v : 0) * a.weight_ld;
    T* q = (T*)a.out + i * a.out_ld;
    const float scale = known ? a.scale : __builtin_nanf("");
    for (int c0 = t * kNormVec; c0 < a.H; c0 += kAhead * TPR * kNormVec) {
      RawRow<T> raw[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        raw[u].clear();
        load_raw<END>(p + c0 + u * TPR * kNormVec, a.H - c0 - u * TPR * kNormVec, raw[u]);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int c = c0 + u * TPR * kNormVec, n = a.H - c;
        align_end<END>(n, raw[u]);
        float y[kNormVec];
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) y[e] = raw[u].at(e) * scale;
        store_row<END>(q + c, n, y);
      }
    }
  }
}

// ---- the positions sorted by token ----

constexpr int kSortThreads = 1024, kSortEach = 4, kSortTile = kSortThreads * kSortEach, kSortWaves = kSortThreads / 64;
constexpr int kSortBits = 6, kSortBins = 1 << kSortBits;
static_assert(kSortBins * kSortWaves == kSortThreads, "one count per thread");

// Memory that the call fills with zeros: `rows` pieces of `row` bytes, the last of `last` bytes.
struct FillArgs {
  char* p;
  int64_t pitch, row, last, rows;
};

struct SortArgs {
  const void* tokens;
  uint32_t *key, *at;  // sorted tokens (V: none that counts) and their positions
  int64_t N, V, padding;
  int wide, bits, tiles;
};

// A wave's own LDS values, written by some of its lanes and read by others.
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Exclusive prefix sum over the workgroup's threads, in their order. Two barriers: one before the first use of lds's
// other readers ends it, one inside.
__device__ __forceinline__ uint32_t sort_scan(uint32_t v, uint32_t* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t sum = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t below = __shfl_up(sum, o);
    if (lane >= o) sum += below;
  }
  if (lane == 63) lds[wave] = sum;
  __syncthreads();
  uint32_t before = 0;
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) before += w < wave ? lds[w] : 0u;
  return before + sum - v;
}

struct SortLds {
  uint32_t key[kSortTile];
  uint16_t at[kSortTile];
  uint32_t count[kSortThreads];  // [bin][wave]
  uint32_t sums[kSortWaves];
};

// One tile, stably, by 6 bits a pass: a lane's place among the wave's equal digits is the number of lower lanes in
// the ballots' match and the wave's count so far, so no count is shared by two waves before the scan over
// [bin][wave]. 4096 keys of 18 bits take about 8 us, nearly all of it the ballots: tiles of a fourth of what LDS
// holds spread that over four times as many CUs.
__device__ __forceinline__ void sort_tile(const SortArgs& a, int tile, SortLds& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t first = (int64_t)tile * kSortTile;
  uint32_t key[kSortEach], at[kSortEach];
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    at[r] = wave * 64 * kSortEach + r * 64 + lane;
    int64_t v = first + at[r] < a.N ? token_at(a.tokens, a.wide, first + at[r]) : a.V;
    if (v < 0 || v >= a.V || v == a.padding) v = a.V;
    key[r] = (uint32_t)v;
  }
  for (int shift = 0; shift < a.bits; shift += kSortBits) {
    s.count[lane * kSortWaves + wave] = 0;
    wave_lds_order();
    uint32_t place[kSortEach];
#pragma unroll
    for (int r = 0; r < kSortEach; ++r) {
      const uint32_t digit = (key[r] >> shift) & (kSortBins - 1);
      uint64_t match = ~0ull;
#pragma unroll
      for (int b = 0; b < kSortBits; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        match &= (digit >> b) & 1 ? set : ~set;
      }
      const uint32_t lower = __builtin_amdgcn_mbcnt_hi((uint32_t)(match >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)match, 0));
      uint32_t* count = &s.count[digit * kSortWaves + wave];
      const uint32_t before = *count;
      wave_lds_order();
      if (lower == 0) *count = before + (uint32_t)__popcll(match);
      wave_lds_order();
      place[r] = before + lower;
    }
    __syncthreads();
    const uint32_t before = sort_scan(s.count[threadIdx.x], s.sums);
    s.count[threadIdx.x] = before;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortEach; ++r) {
      const uint32_t digit = (key[r] >> shift) & (kSortBins - 1);
      const uint32_t to = s.count[digit * kSortWaves + wave] + place[r];
      s.key[to] = key[r];
      s.at[to] = (uint16_t)at[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortEach; ++r) {
      const int from = wave * 64 * kSortEach + r * 64 + lane;
      key[r] = s.key[from];
      at[r] = s.at[from];
    }
  }
  // Places past the last position were sorted behind all others.
#pragma unroll
  for (int r = 0; r < kSortEach; ++r) {
    const int64_t p = first + wave * 64 * kSortEach + r * 64 + lane;
    if (p < a.N) {
      a.key[p] = key[r];
      a.at[p] = (uint32_t)first + at[r];
    }
  }
}

__device__ __forceinline__ void fill_zeros(const FillArgs& f, int64_t block, int64_t blocks) {
  const u32x4 zero = {};
  for (int64_t r = block; r < f.rows; r += blocks) {
    char* p = f.p + r * f.pitch;
    const int64_t n = r + 1 == f.rows ? f.last : f.row;
    for (int64_t c = (int64_t)threadIdx.x * 16; c + 16 <= n; c += kSortThreads * 16) __builtin_memcpy(p + c, &zero, 16);
    // (rows are whole elements of 2 or 4 bytes)
    const int64_t c = n / 16 * 16 + 2 * (int64_t)threadIdx.x;
    if (c < n) *(uint16_t*)(p + c) = 0;
  }
}

// The first blocks sort a tile each, the others write the gradient's zeros meanwhile (rows that tokens name are
// written again by later launches).
__global__ __launch_bounds__(kSortThreads) void embedding_sort_kernel(const SortArgs a, const FillArgs f) {
  __shared__ SortLds s;
  if ((int)blockIdx.x < a.tiles) sort_tile(a, blockIdx.x, s);
  else fill_zeros(f, (int)blockIdx.x - a.tiles, (int)gridDim.x - a.tiles);
}

constexpr int kMergeRuns = 16;

// Up to 16 runs of `length` (a power of two) become one: an element's place is its own and, in each other run, the
// number of elements that come before it, found in all runs at once.
__global__ __launch_bounds__(256) void embedding_merge_kernel(const uint32_t* __restrict__ key, const uint32_t* __restrict__ at,
                                                              uint32_t* __restrict__ key_out, uint32_t* __restrict__ at_out,
                                                              int64_t N, int64_t length) {
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (p >= N) return;
  const int64_t group = p / (length * kMergeRuns) * (length * kMergeRuns);
  const int own = (int)((p - group) / length);
  const uint32_t k = key[p];
  int64_t lo[kMergeRuns], len[kMergeRuns];
#pragma unroll
  for (int b = 0; b < kMergeRuns; ++b) {
    lo[b] = 0;
    const int64_t left = N - group - b * length;
    len[b] = b == own || left < 0 ? 0 : left < length ? left : length;
  }
  for (int64_t step = length; step > 0; step >>= 1) {
#pragma unroll
    for (int b = 0; b < kMergeRuns; ++b) {
      const int64_t next = lo[b] + step;
      if (next <= len[b]) {
        const uint32_t other = key[group + b * length + next - 1];
        if (b < own ? other <= k : other < k) lo[b] = next;
      }
    }
  }
  int64_t to = p - own * length;
#pragma unroll
  for (int b = 0; b < kMergeRuns; ++b) to += lo[b];
  key_out[to] = k;
  at_out[to] = at[p];
}

// ---- the sums ----

struct EmbedSumArgs {
  const void* grad;
  void* out;
  const uint32_t *key, *at;
  float* part;  // [chunks][2][part_ld]: sums of a chunk's first run, where it began earlier, and of its last, where it goes on
  int64_t grad_ld, out_ld, part_ld;
  int64_t N;
  uint32_t V;
  int H, chunk, accumulate;
  float scale;
};

template <RowEnd END, typename T>
__device__ __forceinline__ void write_sum(const EmbedSumArgs& a, uint32_t v, int c, const float (&sum)[kNormVec]) {
  T* p = (T*)a.out + (int64_t)v * a.out_ld + c;
  const int n = a.H - c;
  RawRow<T> old;
  old.clear();
  if (a.accumulate) {
    load_raw<END>(p, n, old);
    align_end<END>(n, old);
  }
  float y[kNormVec];
#pragma unroll
  for (int e = 0; e < kNormVec; ++e) y[e] = fmaf(sum[e], a.scale, old.at(e));
  store_row<END>(p, n, y);
}

// TPR threads walk along a chunk of the sorted positions, 8 columns each, eight rows requested at once.
template <typename T, int TPR, RowEnd END>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbedSumArgs a) {
  constexpr int kAhead = 8;
  int64_t b = (int64_t)blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
  const int64_t first = b * a.chunk;
  if (first >= a.N) return;
  const int n = (int)(a.N - first < a.chunk ? a.N - first : a.chunk);
  const int c = (blockIdx.y * TPR + threadIdx.x % TPR) * kNormVec;
  if (c >= a.H) return;
  float acc[kNormVec] = {};
  uint32_t now = a.key[first];
  // Whether the run at hand began in an earlier chunk.
  bool begun = first > 0 && a.key[first - 1] == now;
  auto leave = [&](int slot) {
    float* p = a.part + (b * 2 + slot) * a.part_ld + c;
    __builtin_memcpy(p, acc, sizeof(acc));
  };
  for (int j0 = 0; j0 < n; j0 += kAhead) {
    uint32_t k[kAhead];
    RawRow<T> g[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) k[u] = j0 + u < n ? a.key[first + j0 + u] : a.V;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      g[u].clear();
      if (k[u] < a.V) load_raw<END>((const T*)a.grad + (int64_t)a.at[first + j0 + u] * a.grad_ld + c, a.H - c, g[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (j0 + u >= n) break;
      if (k[u] != now) {
        if (begun) leave(0);
        else write_sum<END, T>(a, now, c, acc);
        begun = false;
        now = k[u];
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) acc[e] = 0.f;
      }
      if (now >= a.V) return;  // sorted last: nothing that counts follows
      align_end<END>(a.H - c, g[u]);
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) acc[e] += g[u].at(e);
    }
  }
  if (begun) leave(0);
  else if (first + n < a.N && a.key[first + n] == now) leave(1);
  else write_sum<END, T>(a, now, c, acc);
}

// A workgroup for each chunk that a run begins in and leaves: the run's sums from its chunks, in their order.
template <typename T, RowEnd END>
__global__ __launch_bounds__(256) void embedding_join_kernel(const EmbedSumArgs a) {
  const int64_t b = blockIdx.x, first = b * a.chunk, next = first + a.chunk;
  if (next >= a.N) return;
  const uint32_t v = a.key[next - 1];
  if (v >= a.V || a.key[next] != v || (first > 0 && a.key[first - 1] == v)) return;
  const int64_t chunks = (a.N + a.chunk - 1) / a.chunk;
  int64_t end = b + 1;  // the run's last chunk is end - 1
  for (bool on = true; on;) {
    const int64_t k = end + (threadIdx.x & 63);
    const uint64_t goes = __ballot(k < chunks && a.key[(k < chunks ? k : 0) * a.chunk] == v);
    const int more = __builtin_ctzll(~goes | (1ull << 63));
    end += more + (goes == ~0ull ? 1 : 0);
    on = goes == ~0ull;
  }
  const int c = (blockIdx.y * 256 + threadIdx.x) * kNormVec;
  if (c >= a.H) return;
  // A frequent token's sums are thousands: each addition's rounding error is kept and added at the end.
  constexpr int kAhead = 4;
  float acc[kNormVec], lost[kNormVec] = {};
  __builtin_memcpy(acc, a.part + (b * 2 + 1) * a.part_ld + c, sizeof(acc));
  for (int64_t k0 = b + 1; k0 < end; k0 += kAhead) {
    float p[kAhead][kNormVec];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t k = k0 + u < end ? k0 + u : b + 1;
      __builtin_memcpy(p[u], a.part + k * 2 * a.part_ld + c, sizeof(p[u]));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (k0 + u >= end) break;
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) {
        const float x = p[u][e], sum = acc[e] + x, y = sum - acc[e];
        const float off = (acc[e] - (sum - y)) + (x - y);
        lost[e] += fabsf(sum) < INFINITY ? off : 0.f;
        acc[e] = sum;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kNormVec; ++e) acc[e] += lost[e];
  write_sum<END, T>(a, v, c, acc);
}

}  // namespace lce
