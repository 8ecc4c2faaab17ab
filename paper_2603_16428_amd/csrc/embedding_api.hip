// C ABI of the embedding lookup and its gradient (lce_vocab.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "embedding.hpp"
#include "lce_vocab.h"
#include "ops_check.hpp"

namespace lce {
namespace {

lce_status_t check_embedding(int token_bytes, int64_t N, int64_t V, int64_t H, int dtype, float scale) {
  if (N < 0 || V < 1 || H < 1 || !dtype_ok(dtype) || (token_bytes != 4 && token_bytes != 8) || !std::isfinite(scale)) return LCE_ERR_INVALID_ARGUMENT;
  return N > kMaxRows || V > kMaxRows || H > LCE_EMBEDDING_MAX_H ? LCE_ERR_UNSUPPORTED : LCE_OK;
}

// Threads that share a row: 16 up to 128 values, a wave up to 1024 (in two steps), a workgroup above, so that few
// threads have no piece of it. f(threads, how rows end).
template <typename F>
void by_row(int64_t H, F f) {
  using std::integral_constant;
  using Whole = integral_constant<RowEnd, WHOLE>;
  using Part = integral_constant<RowEnd, PART>;
  const bool whole = H % kNormVec == 0;
  auto with = [&](auto tpr) { whole ? f(tpr, Whole{}) : f(tpr, Part{}); };
  if (H < kNormVec) f(integral_constant<int, 16>{}, integral_constant<RowEnd, TINY>{});
  else if (H <= 16 * kNormVec) with(integral_constant<int, 16>{});
  else if (H <= 128 * kNormVec) with(integral_constant<int, 64>{});
  else with(integral_constant<int, 256>{});
}

// Positions of a chunk of the sorted list.
constexpr int64_t kChunk = 32, kLongChunk = 64, kLongFrom = 32768;
int64_t chunk_of(int64_t N) { return N > kLongFrom ? kLongChunk : kChunk; }
// The most chunks that N positions or fewer make (a workspace for N serves any smaller number).
int64_t most_chunks(int64_t N) { return std::max(cdiv(N, chunk_of(N)), cdiv(std::min(N, kLongFrom), kChunk)); }

int64_t padded(int64_t n) { return cdiv(n, 64) * 64; }

struct EmbedSpace {
  uint32_t *key[2], *at[2];
  float* part;
};
EmbedSpace embed_space(void* workspace, int64_t N) {
  EmbedSpace w;
  uint32_t* p = (uint32_t*)workspace;
  for (int k = 0; k < 2; ++k) {
    w.key[k] = p + 2 * k * padded(N);
    w.at[k] = p + (2 * k + 1) * padded(N);
  }
  w.part = (float*)(p + 4 * padded(N));
  return w;
}

FillArgs fill_of(void* p, int64_t ld, int64_t V, int64_t H, int64_t size) {
  constexpr int64_t kPiece = 64 * 1024;
  if (ld != H) return {(char*)p, ld * size, H * size, H * size, V};
  const int64_t bytes = V * H * size, pieces = cdiv(bytes, kPiece);
  return {(char*)p, kPiece, kPiece, bytes - (pieces - 1) * kPiece, pieces};
}

template <typename T, bool ADD>
lce_status_t run_embedding_backward(const SortArgs& sort0, const FillArgs& fill, const EmbedSumArgs& sum0, const EmbedSpace& w, hipStream_t s) {
  SortArgs sort = sort0;
  EmbedSumArgs sum = sum0;
  sort.key = w.key[0];
  sort.at = w.at[0];
  // 512 workgroups of 1024 threads fill the chip's 256 CUs.
  const int64_t fills = std::min<int64_t>(fill.rows, 512);
  if (sort.tiles + fills > 0)
    hipLaunchKernelGGL(embedding_sort_kernel, dim3((unsigned)(sort.tiles + fills)), dim3(kSortThreads), 0, s, sort, fill);
  if (sort.N == 0) return launched();
  int now = 0;
  const dim3 each((unsigned)cdiv(sort.N, 256));
  for (int64_t length = kSortTile; length < sort.N; length *= kMergeRuns, now ^= 1) {
    if (length > kSortTile) {
      hipLaunchKernelGGL(embedding_merge_kernel, each, dim3(256), 0, s, w.key[now], w.at[now], w.key[now ^ 1], w.at[now ^ 1], sort.N, length);
      continue;
    }
    // As few tiles' keys in LDS, and searches in them, as there are.
    auto kernel = sort.tiles <= 2 ? embedding_merge_tiles_kernel<2> : sort.tiles <= 4 ? embedding_merge_tiles_kernel<4>
                : sort.tiles <= 8 ? embedding_merge_tiles_kernel<8> : embedding_merge_tiles_kernel<kMergeRuns>;
    hipLaunchKernelGGL(kernel, each, dim3(256), 0, s, w.key[now], w.at[now], w.key[now ^ 1], w.at[now ^ 1], sort.N);
  }
  sum.key = w.key[now];
  sum.at = w.at[now];
  const int64_t chunks = cdiv(sum.N, sum.chunk);
  by_row(sum.H, [&](auto tpr, auto end) {
    constexpr int kTpr = decltype(tpr)::value;
    constexpr RowEnd kEnd = decltype(end)::value;
    const dim3 grid((unsigned)cdiv(chunks, 256 / kTpr), (unsigned)cdiv(sum.H, kTpr * kNormVec));
    hipLaunchKernelGGL((embedding_sum_kernel<T, kTpr, kEnd, ADD>), grid, dim3(256), 0, s, sum);
    if (chunks > 1)
      hipLaunchKernelGGL((embedding_join_kernel<T, kEnd, ADD>), dim3((unsigned)(chunks - 1), (unsigned)cdiv(sum.H, 256 * kNormVec)), dim3(256), 0, s, sum);
  });
  return launched();
}

}  // namespace
}  // namespace lce

extern "C" {

lce_status_t lce_embedding_forward(const void* tokens, int token_bytes, int64_t N, const void* weight, int64_t weight_ld,
                                   int64_t V, int64_t H, int dtype, float scale, void* out, int64_t out_ld, void* stream) {
  using namespace lce;
  lce_status_t st = check_embedding(token_bytes, N, V, H, dtype, scale);
  if (st != LCE_OK || N == 0) return st;
  if (!tokens || !weight || !out) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype);
  for (const lce_status_t e : {check_pitch(tokens, 1, 1, token_bytes), check_pitch(weight, weight_ld, 0, z), check_pitch(out, out_ld, H, z)})
    if (e != LCE_OK) return e;
  st = check_overlaps({{{out, out_ld * z, H * z, N}, false}},
                      {{tokens, token_bytes, token_bytes, N}, {weight, weight_ld * z, H * z, V}}, {});
  if (st != LCE_OK) return st;
  const EmbedArgs a{tokens, weight, out, weight_ld, out_ld, N, V, (int)H, token_bytes == 8, scale};
  return by_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    by_row(H, [&](auto tpr, auto end) {
      constexpr int kTpr = decltype(tpr)::value;
      const int64_t blocks = std::min(cdiv(N, 256 / kTpr), kRowBlocks);
      hipLaunchKernelGGL((embedding_kernel<T, kTpr, decltype(end)::value>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, a);
    });
    return launched();
  });
}

size_t lce_embedding_workspace_size(int64_t N, int64_t H) {
  using namespace lce;
  if (check_embedding(8, N, 1, H, LCE_DTYPE_FP32, 1.f) != LCE_OK || N > LCE_EMBEDDING_MAX_N) return 0;
  const int64_t n = std::max<int64_t>(N, 1);
  return (size_t)(4 * padded(n) * 4 + most_chunks(n) * 2 * cdiv(H, kNormVec) * kNormVec * 4 + 255) / 256 * 256;
}

lce_status_t lce_embedding_backward(const void* grad, int64_t grad_ld, const void* tokens, int token_bytes, int64_t N,
                                    int64_t V, int64_t H, int dtype, float scale, int64_t padding_idx, void* grad_weight,
                                    int64_t grad_weight_ld, int accumulate, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  using namespace lce;
  lce_status_t st = check_embedding(token_bytes, N, V, H, dtype, scale);
  if (st != LCE_OK) return st;
  if (padding_idx < -1 || padding_idx >= V) return LCE_ERR_INVALID_ARGUMENT;
  if (N > LCE_EMBEDDING_MAX_N) return LCE_ERR_UNSUPPORTED;
  if (N == 0 && accumulate) return LCE_OK;
  if (!grad_weight || (N > 0 && (!grad || !tokens))) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype), need = (int64_t)lce_embedding_workspace_size(N, H);
  for (const lce_status_t e : {check_pitch(N > 0 ? tokens : nullptr, 1, 1, token_bytes), check_pitch(N > 0 ? grad : nullptr, grad_ld, 0, z),
                               check_pitch(grad_weight, grad_weight_ld, H, z)})
    if (e != LCE_OK) return e;
  if (N > 0) {
    if (!workspace || workspace_bytes < (size_t)need) return LCE_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace % 256 != 0) return LCE_ERR_INVALID_ARGUMENT;
    st = check_overlaps({{{grad_weight, grad_weight_ld * z, H * z, V}, false}, {{workspace, need, need, 1}, false}},
                        {{grad, grad_ld * z, H * z, N}, {tokens, token_bytes, token_bytes, N}}, {});
    if (st != LCE_OK) return st;
  }
  const SortArgs sort{tokens, nullptr, nullptr, N, V, padding_idx, token_bytes == 8, 64 - __builtin_clzll((unsigned long long)V), (int)cdiv(N, kSortTile)};
  const EmbedSpace w = embed_space(workspace, N);
  const EmbedSumArgs sum{grad, grad_weight, nullptr, nullptr, w.part, grad_ld, grad_weight_ld, cdiv(H, kNormVec) * kNormVec, N,
                         (uint32_t)V, (int)H, (int)chunk_of(N), scale};
  const FillArgs fill = accumulate ? FillArgs{} : fill_of(grad_weight, grad_weight_ld, V, H, z);
  return by_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    return accumulate ? run_embedding_backward<T, true>(sort, fill, sum, w, (hipStream_t)stream)
                      : run_embedding_backward<T, false>(sort, fill, sum, w, (hipStream_t)stream);
  });
}

}  // extern "C"
