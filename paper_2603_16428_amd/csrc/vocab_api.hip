// C ABI of the operators on the vocabulary's matrix and logits (lce_vocab.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "embedding.hpp"
#include "lce_vocab.h"
#include "mxfp4.hpp"
#include "ops_check.hpp"
#include "sample.hpp"

namespace lce {
namespace {

// Calls f with a value of the element type.
template <typename F>
lce_status_t by_type(int dtype, F f) {
  if (dtype == LCE_DTYPE_BF16) return f(bf16{});
  if (dtype == LCE_DTYPE_FP16) return f(f16{});
  return f(float{});
}

// ---- embedding ----

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

constexpr int64_t kEmbedBlocks = int64_t(1) << 20;

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

// ---- 4 bits ----

lce_status_t check_mxfp4(int64_t N, int64_t H, int dtype) {
  if (N < 0 || H < kMxGroup || H % kMxGroup != 0 || !dtype_ok(dtype)) return LCE_ERR_INVALID_ARGUMENT;
  return N > kMaxRows || H > LCE_MXFP4_MAX_H ? LCE_ERR_UNSUPPORTED : LCE_OK;
}

Rows codes_of(const void* p, int64_t N, int64_t H) { return {p, H / 2, H / 2, N}; }
Rows scales_of(const void* p, int64_t N, int64_t H) { return {p, H / kMxGroup, H / kMxGroup, N}; }

// Threads that share a row, as by_row's.
template <typename F>
void by_row_of_groups(int64_t H, F f) {
  if (H <= 16 * kNormVec) f(std::integral_constant<int, 16>{});
  else if (H <= 128 * kNormVec) f(std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 256>{});
}

template <typename T, int BN>
lce_status_t run_mxfp4_many(MxMatmulArgs a, hipStream_t s) {
  a.tiles_m = (int)cdiv(a.M, BN);
  a.tiles_v = (int)cdiv(a.V, 256);
  const int64_t tiles = (int64_t)a.tiles_m * a.tiles_v;
  if (tiles > (1 << 22)) return LCE_ERR_UNSUPPORTED;
  auto kernel = mxfp4_many_kernel<T, BN>;
  constexpr int kSmem = mx_many_smem<BN>();
  if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kSmem) != hipSuccess) return LCE_ERR_HIP;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(512), kSmem, s, a);
  return launched();
}

template <typename T>
lce_status_t run_mxfp4_matmul(const MxMatmulArgs& a, hipStream_t s) {
  // Few rows read W straight into registers. From 49 on the tile of 128 is the faster (4096 x 128256: 48 rows 76 us, 64 rows
  // 89 us so and 85 in the tile, which takes 90 for 128).
  if (a.M > 48) return a.M <= 128 ? run_mxfp4_many<T, 128>(a, s) : run_mxfp4_many<T, 256>(a, s);
  // 64 rows of W a workgroup read x half as often as 32 (4096 x 128256: 32 rows 68 us against 79, one 51 against 48), if they
  // still leave each CU a workgroup.
  const bool wide = a.M > 4 && a.V >= 64 * 256;
  auto go = [&](auto kernel, int rows) { hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv(a.V, rows)), dim3(256), 0, s, a); };
  if (a.M <= 16) wide ? go(mxfp4_few_kernel<T, 1, 4>, 64) : go(mxfp4_few_kernel<T, 1, 2>, 32);
  else if (a.M <= 32) wide ? go(mxfp4_few_kernel<T, 2, 4>, 64) : go(mxfp4_few_kernel<T, 2, 2>, 32);
  else wide ? go(mxfp4_few_kernel<T, 3, 4>, 64) : go(mxfp4_few_kernel<T, 3, 2>, 32);
  return launched();
}

// ---- sampling ----

lce_status_t check_sample(int64_t N, int64_t V) {
  if (N < 0 || V < 1) return LCE_ERR_INVALID_ARGUMENT;
  return N > LCE_SAMPLE_MAX_N || V > LCE_SAMPLE_MAX_V ? LCE_ERR_UNSUPPORTED : LCE_OK;
}
// Pieces of 64 logits that make a group: as few as keep the groups' number.
int sample_rep(int64_t V) { return V <= 64 * kMostGroups ? 1 : V <= 128 * kMostGroups ? 2 : 4; }
static_assert(LCE_SAMPLE_MAX_V == 256 * kMostGroups, "sample_rep");

template <typename T, int REP, RowEnd END>
lce_status_t run_sample(const SampleArgs& a, int64_t N, hipStream_t s) {
  hipLaunchKernelGGL((sample_parts_kernel<T, REP, END>), dim3((unsigned)(N * a.parts)), dim3(256), 0, s, a);
  hipLaunchKernelGGL((sample_row_kernel<T, REP, END>), dim3((unsigned)N), dim3(kSampleThreads), 0, s, a);
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
      const int64_t blocks = std::min(cdiv(N, 256 / kTpr), kEmbedBlocks);
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

lce_status_t lce_mxfp4_quantize(const void* x, int64_t x_ld, int64_t N, int64_t H, int dtype, void* codes, void* scales, void* stream) {
  using namespace lce;
  lce_status_t st = check_mxfp4(N, H, dtype);
  if (st != LCE_OK || N == 0) return st;
  if (!x || !codes || !scales || (uintptr_t)codes % 16 != 0) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype);
  if ((st = check_pitch(x, x_ld, 0, z)) != LCE_OK) return st;
  st = check_overlaps({{codes_of(codes, N, H), false}, {scales_of(scales, N, H), false}}, {{x, x_ld * z, H * z, N}}, {});
  if (st != LCE_OK) return st;
  const MxRowsArgs a{x, nullptr, (uint8_t*)codes, (uint8_t*)scales, x_ld, N, (int)H};
  return by_type(dtype, [&](auto zero) {
    by_row_of_groups(H, [&](auto tpr) {
      constexpr int kTpr = decltype(tpr)::value;
      hipLaunchKernelGGL((mxfp4_quantize_kernel<decltype(zero), kTpr>), dim3((unsigned)std::min(cdiv(N, 256 / kTpr), kEmbedBlocks)), dim3(256), 0,
                         (hipStream_t)stream, a);
    });
    return launched();
  });
}

lce_status_t lce_mxfp4_dequantize(const void* codes, const void* scales, int64_t N, int64_t H, int dtype, void* y, int64_t y_ld,
                                  void* stream) {
  using namespace lce;
  lce_status_t st = check_mxfp4(N, H, dtype);
  if (st != LCE_OK || N == 0) return st;
  if (!y || !codes || !scales || (uintptr_t)codes % 16 != 0) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype);
  if ((st = check_pitch(y, y_ld, H, z)) != LCE_OK) return st;
  st = check_overlaps({{{y, y_ld * z, H * z, N}, false}}, {codes_of(codes, N, H), scales_of(scales, N, H)}, {});
  if (st != LCE_OK) return st;
  const MxRowsArgs a{nullptr, y, (uint8_t*)codes, (uint8_t*)scales, y_ld, N, (int)H};
  return by_type(dtype, [&](auto zero) {
    by_row_of_groups(H, [&](auto tpr) {
      constexpr int kTpr = decltype(tpr)::value;
      hipLaunchKernelGGL((mxfp4_dequantize_kernel<decltype(zero), kTpr>), dim3((unsigned)std::min(cdiv(N, 256 / kTpr), kEmbedBlocks)), dim3(256), 0,
                         (hipStream_t)stream, a);
    });
    return launched();
  });
}

lce_status_t lce_mxfp4_matmul(const void* x_codes, const void* x_scales, int64_t M, const void* w_codes, const void* w_scales,
                              int64_t V, int64_t H, int dtype, void* out, int64_t out_ld, void* stream) {
  using namespace lce;
  lce_status_t st = check_mxfp4(M, H, dtype);
  if (st == LCE_OK) st = check_mxfp4(V, H, dtype);
  if (st != LCE_OK || M == 0 || V == 0) return st;
  if (!x_codes || !x_scales || !w_codes || !w_scales || !out || ((uintptr_t)x_codes | (uintptr_t)w_codes) % 16 != 0) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype);
  if (out_ld < V || (uintptr_t)out % z != 0) return LCE_ERR_INVALID_ARGUMENT;
  st = check_overlaps({{{out, out_ld * z, V * z, M}, false}},
                      {codes_of(x_codes, M, H), scales_of(x_scales, M, H), codes_of(w_codes, V, H), scales_of(w_scales, V, H)}, {});
  if (st != LCE_OK) return st;
  const MxMatmulArgs a{(const uint8_t*)x_codes, (const uint8_t*)x_scales, (const uint8_t*)w_codes, (const uint8_t*)w_scales, out, out_ld, M, V, (int)H, 0, 0};
  return by_type(dtype, [&](auto zero) { return run_mxfp4_matmul<decltype(zero)>(a, (hipStream_t)stream); });
}

size_t lce_sample_workspace_size(int64_t N, int64_t V) {
  using namespace lce;
  if (check_sample(N, V) != LCE_OK) return 0;
  const int64_t groups = cdiv(V, 64 * sample_rep(V)), parts = cdiv(groups, kPartGroups), n = std::max<int64_t>(N, 1);
  return (size_t)cdiv(n * (parts * 12 + groups * 4), 256) * 256;
}

lce_status_t lce_sample(const void* logits, int64_t logits_ld, int64_t N, int64_t V, int dtype, const float* uniforms,
                        const lce_sample_t* settings, int64_t* tokens, float* logprobs, void* workspace, size_t workspace_bytes,
                        void* stream) {
  using namespace lce;
  lce_status_t st = dtype_ok(dtype) ? check_sample(N, V) : LCE_ERR_INVALID_ARGUMENT;
  if (st != LCE_OK) return st;
  if (!settings) return LCE_ERR_INVALID_ARGUMENT;
  const lce_sample_t c = *settings;
  // (a NaN fails the comparisons)
  if ((!c.temperatures && !(c.temperature >= 0.f)) || (!c.top_ps && !(c.top_p >= 0.f)) || (!c.min_ps && !(c.min_p >= 0.f && c.min_p <= 1.f)) ||
      (!c.top_ks && c.top_k < 0))
    return LCE_ERR_INVALID_ARGUMENT;
  if (N == 0) return LCE_OK;
  if (!logits || !uniforms || !tokens) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype), need = (int64_t)lce_sample_workspace_size(N, V);
  for (const lce_status_t e : {check_pitch(logits, logits_ld, 0, z), check_pitch(uniforms, 1, 1, 4), check_pitch(tokens, 1, 1, 8), check_pitch(logprobs, 1, 1, 4),
                               check_pitch(c.temperatures, 1, 1, 4), check_pitch(c.top_ps, 1, 1, 4), check_pitch(c.min_ps, 1, 1, 4), check_pitch(c.top_ks, 1, 1, 4)})
    if (e != LCE_OK) return e;
  if (!workspace || workspace_bytes < (size_t)need) return LCE_ERR_WORKSPACE_TOO_SMALL;
  if ((uintptr_t)workspace % 256 != 0) return LCE_ERR_INVALID_ARGUMENT;
  st = check_overlaps({{{tokens, 8, 8, N}, false}, {{logprobs, 4, 4, N}, false}, {{workspace, need, need, 1}, false}},
                      {{logits, logits_ld * z, V * z, N}, {uniforms, 4, 4, N}, {c.temperatures, 4, 4, N}, {c.top_ps, 4, 4, N}, {c.min_ps, 4, 4, N}, {c.top_ks, 4, 4, N}}, {});
  if (st != LCE_OK) return st;
  const int rep = sample_rep(V), groups = (int)cdiv(V, 64 * rep), parts = (int)cdiv(groups, kPartGroups);
  double* sums = (double*)workspace;
  float* part_max = (float*)(sums + N * parts);
  // All weights together stay below 2^63, one below 2^51.
  const int bits = std::min(50, 62 - (V > 1 ? 32 - __builtin_clz((unsigned)(V - 1)) : 0));
  const SampleArgs a{logits, logits_ld, uniforms, c.temperature, c.top_p, c.min_p, c.top_k, c.temperatures, c.top_ps, c.min_ps, c.top_ks, tokens, logprobs,
                     part_max + N * parts, part_max, sums, (int)V, groups, parts, bits};
  hipStream_t s = (hipStream_t)stream;
  return by_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    if (V < kNormVec) return run_sample<T, 1, TINY>(a, N, s);
    return rep == 1 ? run_sample<T, 1, PART>(a, N, s) : rep == 2 ? run_sample<T, 2, PART>(a, N, s) : run_sample<T, 4, PART>(a, N, s);
  });
}

}  // extern "C"
