// Rows of a V x H matrix by token, and the gradient: for each token the sum of its rows of the upstream gradient.
//
// The gradient's sums run over the tokens' positions in order. The positions are sorted by token (stably, so a
// token's stay in order): tiles of 2048 in LDS, then up to 16 sorted runs at a time merged by rank. The sorted list is cut into
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

// TPR threads a row, two pieces of 8 values requested at once by each. Bound by HBM's writes: 8192 x 4096 in bf16 19.4 us (99 MB,
// 5.1 TB/s, as a large copy); one row 1.9 us.
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

constexpr int kSortThreads = 1024, kSortEach = 2, kSortTile = kSortThreads * kSortEach, kSortWaves = kSortThreads / 64;
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

// Exclusive prefix sum over the workgroup's threads, in their order. (The caller's barriers keep one use of lds from the next.)
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
// [bin][wave]. Bound by the ballots' instructions: small tiles spread them over more CUs, but leave more runs to merge (8192
// positions of 17 bits: tiles of 1024 6.6 us and 14 for the merge, of 2048 8.4 and 7.0, of 4096 12.5 and 11 in memory).
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
// written again by later launches). 128256 x 4096 in bf16: 168 us (1.05 GB, 6.3 TB/s; torch's fill of 1 GB 6.8).
__global__ __launch_bounds__(kSortThreads) void embedding_sort_kernel(const SortArgs a, const FillArgs f) {
  __shared__ SortLds s;
  if ((int)blockIdx.x < a.tiles) sort_tile(a, blockIdx.x, s);
  else fill_zeros(f, (int)blockIdx.x - a.tiles, (int)gridDim.x - a.tiles);
}

constexpr int kMergeRuns = 16;

// Up to RUNS tiles become one run: an element's place is its own and, in each other tile, the number of elements that come
// before it, found in all tiles at once in a copy of their keys in LDS (8192 positions: 21 us searched in memory).
template <int RUNS>
__global__ __launch_bounds__(256) void embedding_merge_tiles_kernel(const uint32_t* __restrict__ key, const uint32_t* __restrict__ at,
                                                                    uint32_t* __restrict__ key_out, uint32_t* __restrict__ at_out,
                                                                    int64_t N) {
  constexpr int kKeys = RUNS * kSortTile, kLoads = kKeys / 1024;
  __shared__ uint32_t keys[kKeys];
  const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x, group = (int64_t)blockIdx.x * 256 / kKeys * kKeys;
  const int left = (int)(N - group < kKeys ? N - group : kKeys);
  u32x4 k4[kLoads];  // (the arrays' lengths are multiples of 64)
#pragma unroll
  for (int u = 0; u < kLoads; ++u) __builtin_memcpy(&k4[u], key + group + min(u * 1024 + (int)threadIdx.x * 4, (left - 1) / 4 * 4), 16);
#pragma unroll
  for (int u = 0; u < kLoads; ++u) *(u32x4*)&keys[u * 1024 + threadIdx.x * 4] = k4[u];
  const uint32_t place = at[p < N ? p : N - 1];
  __syncthreads();
  if (p >= N) return;
  const int self = (int)(p - group), own = self / kSortTile;
  const uint32_t k = keys[self];
  int lo[RUNS];
#pragma unroll
  for (int b = 0; b < RUNS; ++b) lo[b] = b * kSortTile;
  // Without a branch, so that a step is one read's latency.
  for (int step = kSortTile; step > 0; step >>= 1) {
    uint32_t other[RUNS];
#pragma unroll
    for (int b = 0; b < RUNS; ++b) {
      const int next = lo[b] + step;
      other[b] = keys[next <= min(left, (b + 1) * kSortTile) ? next - 1 : self];
    }
#pragma unroll
    for (int b = 0; b < RUNS; ++b) {
      const int next = lo[b] + step;
      if (next <= min(left, (b + 1) * kSortTile) && (b < own ? other[b] <= k : other[b] < k)) lo[b] = next;
    }
  }
  int to = self % kSortTile;
#pragma unroll
  for (int b = 0; b < RUNS; ++b)
    if (b != own) to += lo[b] - b * kSortTile;
  key_out[group + to] = k;
  at_out[group + to] = place;
}

// The same for up to 16 longer runs, of `length` (a power of two), in memory.
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
  // Three of a run's elements a step, those of all runs requested together without a branch (a place past the run's
  // end reads another and counts for nothing): a step is a load's latency.
  for (int64_t step = __builtin_ctzll(length) % 2 == 0 ? length : length / 2; step > 0; step >>= 2) {  // powers of four
    uint32_t other[kMergeRuns][3];
#pragma unroll
    for (int b = 0; b < kMergeRuns; ++b)
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        const int64_t next = lo[b] + (q + 1) * step;
        other[b][q] = key[next <= len[b] ? group + b * length + next - 1 : p];
      }
#pragma unroll
    for (int b = 0; b < kMergeRuns; ++b) {
      int more = 0;
#pragma unroll
      for (int q = 0; q < 3; ++q)
        more += lo[b] + (q + 1) * step <= len[b] && (b < own ? other[b][q] <= k : other[b][q] < k);
      lo[b] += more * step;
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
  int H, chunk;
  float scale;
};

template <RowEnd END, bool ADD, typename T>
__device__ __forceinline__ void write_sum(const EmbedSumArgs& a, uint32_t v, int c, const float (&sum)[kNormVec], RawRow<T>& old) {
  const int n = a.H - c;
  float y[kNormVec];
  if constexpr (ADD) {
    align_end<END>(n, old);
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) y[e] = fmaf(sum[e], a.scale, old.at(e));
  } else {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) y[e] = sum[e] * a.scale;
  }
  store_row<END>((T*)a.out + (int64_t)v * a.out_ld + c, n, y);
}

constexpr int kMostChunk = 64;

// TPR threads walk along a chunk of the sorted positions, 8 columns each. Bound by the loads' latency unless many are on
// the way: the chunk's tokens and positions come first, all at once, and then eight rows are requested ahead
// (with the token's earlier row where it is added to; 16 ahead are no faster, 30 us against 27.5). 8192 x 4096 in bf16, added to the rows of
// 1800 tokens: 27.5 us for 104 MB (51 with the requests behind branches); into new memory 38, while the zeros are still on their
// way from the caches to HBM. Chunks of 16 positions: 28.6 here and 14 instead of 8 for the join.
template <typename T, int TPR, RowEnd END, bool ADD>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const EmbedSumArgs a) {
  constexpr int kAhead = 8, kChunks = 256 / TPR;
  __shared__ uint32_t keys[kChunks][kMostChunk + 1], places[kChunks][kMostChunk];
  const int64_t b0 = (int64_t)blockIdx.x * kChunks;
  for (int k = threadIdx.x; k < kChunks * (a.chunk + 1); k += 256) {
    const int of = k / (a.chunk + 1), j = k % (a.chunk + 1);
    const int64_t p = (b0 + of) * a.chunk + j;
    keys[of][j] = p < a.N ? a.key[p] : a.V;
    if (j < a.chunk) places[of][j] = p < a.N ? a.at[p] : 0u;
  }
  __syncthreads();
  int group = threadIdx.x / TPR;
  if constexpr (TPR >= 64) group = __builtin_amdgcn_readfirstlane(group);  // (what a wave shares is a scalar)
  const int64_t b = b0 + group, first = b * a.chunk;
  const int c = (blockIdx.y * TPR + threadIdx.x % TPR) * kNormVec;
  if (first >= a.N || c >= a.H) return;
  const int n = (int)(a.N - first < a.chunk ? a.N - first : a.chunk);
  auto scalar = [](uint32_t v) { return TPR >= 64 ? (uint32_t)__builtin_amdgcn_readfirstlane((int)v) : v; };
  auto key = [&](int j) { return scalar(keys[group][j]); };
  RawRow<T> g[kAhead], old[kAhead];
  // No branch stands around a request (of places past the chunk the last row is read again): behind one, the compiler
  // waits for all that is on the way.
  auto request = [&](int j, RawRow<T>& row, RawRow<T>& before) {
    j = j < n ? j : n - 1;
    load_raw<END>((const T*)a.grad + (int64_t)scalar(places[group][j]) * a.grad_ld + c, a.H - c, row);
    if constexpr (ADD) {
      const uint32_t v = key(j);
      load_raw<END>((const T*)a.out + (int64_t)(v < a.V ? v : 0u) * a.out_ld + c, a.H - c, before);
    }
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) request(u, g[u], old[u]);
  float acc[kNormVec] = {};
  // Whether the run at hand began in an earlier chunk.
  bool begun = first > 0 && a.key[first - 1] == key(0);
  auto leave = [&](int slot) { __builtin_memcpy(a.part + (b * 2 + slot) * a.part_ld + c, acc, sizeof(acc)); };
  for (int j0 = 0; j0 < n; j0 += kAhead) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u;
      if (j < n) {
        align_end<END>(a.H - c, g[u]);
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) acc[e] += g[u].at(e);
        const uint32_t v = key(j);
        const bool goes_on = key(j + 1) == v;
        if (!goes_on || j + 1 == n) {
          // (a.V is no token: rows that count for nothing, sorted last)
          if (v < a.V) {
            if (begun) leave(0);
            else if (goes_on) leave(1);
            else write_sum<END, ADD, T>(a, v, c, acc, old[u]);
          }
          begun = false;
#pragma unroll
          for (int e = 0; e < kNormVec; ++e) acc[e] = 0.f;
        }
      }
      request(j + kAhead, g[u], old[u]);
    }
  }
}

// A workgroup for each chunk that a run begins in and leaves: the run's sums from its chunks, in their order.
template <typename T, RowEnd END, bool ADD>
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
  RawRow<T> old;
  if constexpr (ADD) load_raw<END>((const T*)a.out + (int64_t)v * a.out_ld + c, a.H - c, old);
  write_sum<END, ADD, T>(a, v, c, acc, old);
}

}  // namespace lce
