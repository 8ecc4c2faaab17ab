// C ABI of rows and weights in 4 bits and their product (lce_vocab.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "lce_vocab.h"
#include "mxfp4.hpp"
#include "ops_check.hpp"

namespace lce {
namespace {

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
  if (tiles > LCE_MXFP4_MAX_TILES) return LCE_ERR_UNSUPPORTED;
  constexpr int kWaves = BN / 32;
  auto kernel = mxfp4_many_kernel<T, BN, kWaves>;
  constexpr int kSmem = mx_many_smem<BN>();
  if (hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kSmem) != hipSuccess) return LCE_ERR_HIP;
  hipLaunchKernelGGL(kernel, dim3((unsigned)tiles), dim3(64 * kWaves), kSmem, s, a);
  return launched();
}

template <typename T>
lce_status_t run_mxfp4_matmul(const MxMatmulArgs& a, hipStream_t s) {
  // Few rows read W straight into registers. From 49 on the tile of 128 is the faster (4096 x 128256: 48 rows 76 us, 64 rows
  // 89 us so and 86 in the tile, which takes 89 for 128). The rule does not look at V, and loses where a workgroup for 256 rows of W
  // leaves CUs idle that the kernel for few rows has work for: 48 and 49 rows take 49 and 88 us for 12288 x 32768, 13 and 47 for 8192 x 4096, 9 and
  // 26 for 4096 x 2048. (Smaller tiles of W, or K split over workgroups, are what is missing there.)
  // More rows than that take the tile of 256 (256 rows: 107 us against 152, 2048: 686 against 1168) where it leaves no more than half of
  // the 256 CUs without one (2048 x 1024 x 2048: 14 us, 11 in twice as many tiles of 128).
  if (a.M > 128 && cdiv(a.M, 256) * cdiv(a.V, 256) > 128) return run_mxfp4_many<T, 256>(a, s);
  if (a.M > 48) return run_mxfp4_many<T, 128>(a, s);
  // 64 rows of W a workgroup read x half as often as 32 (4096 x 128256: 32 rows 68 us against 79, one 51 against 48), if they
  // still leave each CU a workgroup.
  const bool wide = a.M > 4 && a.V >= 64 * 256;
  // (a launch's threads are counted in 32 bits: 2^28 rows of W at a time)
  constexpr int64_t kRowsAtOnce = int64_t(1) << 28;
  auto go = [&](auto kernel, int rows) {
    for (int64_t v = 0; v < a.V; v += kRowsAtOnce) {
      MxMatmulArgs b = a;
      b.w += v * (a.K / 2);
      b.w_scales += v * (a.K / kMxGroup);
      b.out = (T*)a.out + v;
      b.V = std::min(a.V - v, kRowsAtOnce);
      hipLaunchKernelGGL(kernel, dim3((unsigned)cdiv(b.V, rows)), dim3(256), 0, s, b);
    }
  };
  if (a.M <= 16) wide ? go(mxfp4_few_kernel<T, 1, 4>, 64) : go(mxfp4_few_kernel<T, 1, 2>, 32);
  else if (a.M <= 32) wide ? go(mxfp4_few_kernel<T, 2, 4>, 64) : go(mxfp4_few_kernel<T, 2, 2>, 32);
  else wide ? go(mxfp4_few_kernel<T, 3, 4>, 64) : go(mxfp4_few_kernel<T, 3, 2>, 32);
  return launched();
}

}  // namespace
}  // namespace lce

extern "C" {

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
      hipLaunchKernelGGL((mxfp4_quantize_kernel<decltype(zero), kTpr>), dim3((unsigned)std::min(cdiv(N, 256 / kTpr), kRowBlocks)), dim3(256), 0,
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
      hipLaunchKernelGGL((mxfp4_dequantize_kernel<decltype(zero), kTpr>), dim3((unsigned)std::min(cdiv(N, 256 / kTpr), kRowBlocks)), dim3(256), 0,
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

}  // extern "C"
