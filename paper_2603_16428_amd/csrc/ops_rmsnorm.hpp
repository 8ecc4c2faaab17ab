// The residual's addition with the RMSNorm of the sum (rows in the input type or in e4m3 with scales),
// and its backward.
//
// A row is held in the registers of the TPR threads that share it: each takes 8 consecutive values (16
// bytes of a 16-bit type) of every 8 TPR, CH times. So every tensor is read and written once, whatever is
// needed of the whole row (the mean square, the largest value, the backward's dot product) in between, and
// an output may be an input's own memory: a row's values are all in registers before any is written. Loads
// and stores are 16 bytes wide at any alignment of the element type; only the end of a row whose H is not
// a multiple of 8 goes value by value.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lce_aux.hpp"

namespace lce {

constexpr int kNormVec = 8;

// 8 values at p as fp32, of which the first n exist (the others are 0); n may be <= 0.
template <typename T>
__device__ __forceinline__ void load_row(const T* p, int n, float (&v)[kNormVec]) {
  T raw[kNormVec];
  if (n >= kNormVec) {
    __builtin_memcpy(raw, p, sizeof(raw));
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) v[e] = to_f32(raw[e]);
  } else {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) v[e] = e < n ? to_f32(p[e]) : 0.f;
  }
}

template <typename T>
__device__ __forceinline__ void store_row(T* p, int n, const float (&v)[kNormVec]) {
  if (n >= kNormVec) {
    T raw[kNormVec];
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) raw[e] = from_f32<T>(v[e]);
    __builtin_memcpy(p, raw, sizeof(raw));
  } else {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}

// 8 values in e4m3, to nearest even. All are NaN or at most 448 (up to an fp32 rounding, which goes to
// 448): nothing has to be clamped.
__device__ __forceinline__ void store_row_fp8(uint8_t* p, int n, const float (&v)[kNormVec]) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int q = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], q, true);
  }
  if (n >= kNormVec) {
    __builtin_memcpy(p, w, 8);
  } else {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e)
      if (e < n) p[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
  }
}

// The TPR threads' sum (or, of bit patterns, maximum) of a row, in a fixed order, for all of them. More
// than a wave's goes through `lds`, one entry per wave; two buffers in turn need one barrier a row.
struct AddOp {
  static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct MaxOp {
  static __device__ __forceinline__ uint32_t of(uint32_t a, uint32_t b) { return a > b ? a : b; }
};
template <int TPR, typename Op, typename V>
__device__ __forceinline__ V row_reduce(V v, V* lds) {
#pragma unroll
  for (int o = 1; o < (TPR < 64 ? TPR : 64); o <<= 1) v = Op::of(v, __shfl_xor(v, o));
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < TPR / 64; ++w) v = Op::of(v, lds[w]);
  }
  return v;
}

struct NormArgs {
  const void *x, *residual, *gamma;
  void *normed, *added;
  float *rstd, *scales;
  int64_t x_ld, residual_ld, normed_ld, added_ld;  // elements (quantised rows: bytes)
  int64_t N;
  int H, group;
  float eps;
};

constexpr float kFp8Max = 448.f;
constexpr float kScaleMin = 1.17549435e-38f;  // 2^-126, whose inverse is still finite

template <typename T, int TPR, int CH, bool QUANT>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void add_rmsnorm_kernel(const NormArgs a) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR, kWaves = TPR > 64 ? TPR / 64 : 1;
  __shared__ float sums[2][kWaves];
  __shared__ uint32_t tops[2][kWaves];
  const int t = threadIdx.x % TPR;
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.N; base += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t i = base + threadIdx.x / TPR;
    const bool live = i < a.N;
    float s[CH][kNormVec];
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
      load_row((const T*)a.x + i * a.x_ld + c, n, s[k]);
      if (a.residual != nullptr) {
        float r[kNormVec];
        load_row((const T*)a.residual + i * a.residual_ld + c, n, r);
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) s[k][e] += r[e];
      }
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) ss = fmaf(s[k][e], s[k][e], ss);
    }
    ss = row_reduce<TPR, AddOp>(ss, sums[turn]);
    const float r = 1.f / sqrtf(ss / (float)a.H + a.eps);
    if (live && t == 0 && a.rstd != nullptr) a.rstd[i] = r;
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
      if (a.added != nullptr) store_row((T*)a.added + i * a.added_ld + c, n, s[k]);
      float g[kNormVec];
      load_row((const T*)a.gamma + c, n, g);
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) s[k][e] = s[k][e] * r * g[e];
      if constexpr (!QUANT) {
        store_row((T*)a.normed + i * a.normed_ld + c, n, s[k]);
      } else {
        // The largest magnitude by its bits, among which a NaN's are above all others.
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) m = MaxOp::of(m, __builtin_bit_cast(uint32_t, s[k][e]) & 0x7fffffffu);
        if (a.group == 0) {
          top = MaxOp::of(top, m);
        } else {
          for (int o = 1; o < a.group / kNormVec; o <<= 1) m = MaxOp::of(m, (uint32_t)__shfl_xor((int)m, o));
          const float amax = __builtin_bit_cast(float, m);
          const float scale = amax / kFp8Max, inv = scale < kScaleMin ? 1.f / kScaleMin : kFp8Max / amax;
          if (n > 0 && c % a.group == 0)
            a.scales[i * ((a.H + a.group - 1) / a.group) + c / a.group] = scale < kScaleMin ? kScaleMin : scale;
#pragma unroll
          for (int e = 0; e < kNormVec; ++e) s[k][e] *= inv;
          store_row_fp8((uint8_t*)a.normed + i * a.normed_ld + c, n, s[k]);
        }
      }
    }
    if constexpr (QUANT) {
      if (a.group == 0) {
        top = row_reduce<TPR, MaxOp>(top, tops[turn]);
        const float amax = __builtin_bit_cast(float, top);
        const float scale = amax / kFp8Max, inv = scale < kScaleMin ? 1.f / kScaleMin : kFp8Max / amax;
        if (live && t == 0) a.scales[i] = scale < kScaleMin ? kScaleMin : scale;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
#pragma unroll
          for (int e = 0; e < kNormVec; ++e) s[k][e] *= inv;
          store_row_fp8((uint8_t*)a.normed + i * a.normed_ld + c, n, s[k]);
        }
      }
    }
  }
}

struct NormBackwardArgs {
  const void *dy, *ds, *x, *residual, *gamma;
  const float* rstd;
  void* dx;
  float* part;  // [gridDim.x][H], or null: no gradient of gamma
  int64_t dy_ld, ds_ld, x_ld, residual_ld, dx_ld;
  int64_t N;
  int H;
};

// A workgroup walks over rows; each thread keeps the sums of its own columns of dgamma over them, and
// the workgroup's sums go to part (summed by gamma_sum_kernel in a fixed order).
template <typename T, int TPR, int CH>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void add_rmsnorm_backward_kernel(const NormBackwardArgs a) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR, kWaves = TPR > 64 ? TPR / 64 : 1;
  constexpr int kCols = TPR * CH * kNormVec;
  __shared__ float sums[2][kWaves];
  const int t = threadIdx.x % TPR;
  float acc[CH][kNormVec], g[CH][kNormVec];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = (k * TPR + t) * kNormVec;
    load_row((const T*)a.gamma + c, a.H - c, g[k]);
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) acc[k][e] = 0.f;
  }
  const float inv_h = 1.f / (float)a.H;
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.N; base += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t i = base + threadIdx.x / TPR;
    const bool live = i < a.N;
    float dy[CH][kNormVec], s[CH][kNormVec], ds[CH][kNormVec];
    const float r = live ? a.rstd[i] : 0.f;
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
      load_row((const T*)a.dy + i * a.dy_ld + c, n, dy[k]);
      load_row((const T*)a.x + i * a.x_ld + c, n, s[k]);
      if (a.residual != nullptr) {
        float res[kNormVec];
        load_row((const T*)a.residual + i * a.residual_ld + c, n, res);
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) s[k][e] += res[e];
      }
      if (a.ds != nullptr) load_row((const T*)a.ds + i * a.ds_ld + c, n, ds[k]);
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) {
        acc[k][e] = fmaf(dy[k][e], s[k][e] * r, acc[k][e]);
        dy[k][e] *= g[k][e];
        dot = fmaf(dy[k][e], s[k][e], dot);
      }
    }
    dot = row_reduce<TPR, AddOp>(dot, sums[turn]);
    const float c1 = r * r * (dot * inv_h);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) {
        dy[k][e] = r * (dy[k][e] - s[k][e] * c1);
        if (a.ds != nullptr) dy[k][e] += ds[k][e];
      }
      store_row((T*)a.dx + i * a.dx_ld + c, n, dy[k]);
    }
  }
  if (a.part == nullptr) return;
  float* out = a.part + (size_t)blockIdx.x * a.H;
  if constexpr (kRows == 1) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec;
      store_row(out + c, a.H - c, acc[k]);
    }
  } else {
    __shared__ float cols[kRows][kCols];
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) cols[threadIdx.x / TPR][(k * TPR + t) * kNormVec + e] = acc[k][e];
    __syncthreads();
    for (int c = threadIdx.x; c < a.H; c += kThreads) {
      float v = cols[0][c];
#pragma unroll
      for (int w = 1; w < kRows; ++w) v += cols[w][c];
      out[c] = v;
    }
  }
}

// dgamma_j = sum_b part[b][j] in a fixed order: 64 columns per workgroup, every 16th row of part per
// wave (four requested ahead), then the 16 waves' sums in order.
template <typename T>
__global__ __launch_bounds__(1024) void gamma_sum_kernel(const float* __restrict__ part, int rows, int H,
                                                         T* __restrict__ dgamma) {
  constexpr int kAhead = 4, kWaves = 16;
  __shared__ float sums[kWaves][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int j = blockIdx.x * 64 + lane;
  float acc = 0.f;
  if (j < H) {
    for (int b0 = w; b0 < rows; b0 += kWaves * kAhead) {
      float v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = b0 + kWaves * u < rows ? part[(size_t)(b0 + kWaves * u) * H + j] : 0.f;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) acc += v[u];
    }
  }
  sums[w][lane] = acc;
  __syncthreads();
  if (w == 0 && j < H) {
#pragma unroll
    for (int k = 1; k < kWaves; ++k) acc += sums[k][lane];
    dgamma[j] = from_f32<T>(acc);
  }
}

}  // namespace lce
