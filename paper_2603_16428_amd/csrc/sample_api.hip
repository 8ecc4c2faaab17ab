// C ABI of the choice of a token from logits (lce_vocab.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "lce_vocab.h"
#include "ops_check.hpp"
#include "sample.hpp"

namespace lce {
namespace {

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

size_t lce_sample_workspace_size(int64_t N, int64_t V) {
  using namespace lce;
  if (check_sample(N, V) != LCE_OK) return 0;
  const int64_t groups = cdiv(V, 64 * sample_rep(V)), parts = cdiv(groups, kPartGroups), n = std::max<int64_t>(N, 1);
  return (size_t)cdiv(n * (parts * (12 + 12 * kSampleCells) + groups * 4), 256) * 256;
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
  uint64_t* cell_weight = (uint64_t*)(sums + N * parts);
  uint32_t* cell_count = (uint32_t*)(cell_weight + N * parts * kSampleCells);
  float* part_max = (float*)(cell_count + N * parts * kSampleCells);
  // All weights together stay below 2^63, one below 2^51 (for groups of more than 64 the kernel takes it from the row).
  const int bits = std::min(50, 62 - (V > 1 ? 32 - __builtin_clz((unsigned)(V - 1)) : 0));
  const SampleArgs a{logits, logits_ld, uniforms, c.temperature, c.top_p, c.min_p, c.top_k, c.temperatures, c.top_ps, c.min_ps, c.top_ks, tokens, logprobs,
                     part_max + N * parts, part_max, sums, cell_weight, cell_count, (int)V, groups, parts, bits};
  hipStream_t s = (hipStream_t)stream;
  return by_type(dtype, [&](auto zero) {
    using T = decltype(zero);
    if (V < kNormVec) return run_sample<T, 1, TINY>(a, N, s);
    return rep == 1 ? run_sample<T, 1, PART>(a, N, s) : rep == 2 ? run_sample<T, 2, PART>(a, N, s) : run_sample<T, 4, PART>(a, N, s);
  });
}

}  // extern "C"
