// The global norm of many tensors, and the tensors scaled by it.
//
// The tensors are cut into pieces of 16 KB, numbered through all of them; a workgroup takes a run of
// consecutive pieces. So the tensors' number and sizes do not matter, and the sums' order is fixed by
// the tensors' sizes alone. The table of tensors comes with the kernel's arguments, or, where they are
// more than kInlineTensors, from the workspace (grad_table_kernel).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lce_aux.hpp"

namespace lce {

struct TensorEntry {
  const void* in;
  void* out;
  int64_t n;
  int32_t first;  // its first piece
  int32_t dtype;
};
constexpr int kInlineTensors = 112;    // 3584 bytes of the kernel's arguments
constexpr int kPieceBytes = 16 * 1024;
constexpr int kGradThreads = 256;
// 8 workgroups of 4 waves per CU, all resident at once. The norm of 1.05 GB of bf16 takes 191 us (5.5 TB/s), of 300
// fp32 tensors of 139 MB 37 us; with 1024 workgroups 186 and (before the last pieces' wide loads, 41 with these) 45;
// with 4096 as long, but clipping in place 196 against 192, as each workgroup joins all the shares.
constexpr int kGradBlocks = 2048;

struct TensorTable {
  TensorEntry entry[kInlineTensors];
};

static __global__ __launch_bounds__(128) void grad_table_kernel(const TensorTable t, int count, TensorEntry* __restrict__ out) {
  if ((int)threadIdx.x < count) out[threadIdx.x] = t.entry[threadIdx.x];
}

// The larger of two, and NaN if one is.
__device__ __forceinline__ double max_nan(double a, double b) { return (a >= b || a != a) ? a : b; }
template <bool INF>
__device__ __forceinline__ double join(double a, double b) { return INF ? max_nan(a, b) : a + b; }

// The workgroup's joined values, for its thread 0 (all threads call it).
template <bool INF>
__device__ __forceinline__ double block_join(double v, double* lds) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) v = join<INF>(v, __shfl_xor(v, o));
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return join<INF>(join<INF>(lds[0], lds[1]), join<INF>(lds[2], lds[3]));
}

// One piece's share of the norm: kVec values per thread and step, all four steps requested at once. A tensor's
// last piece ends with up to kVec - 1 values that go one by one.
template <typename T, bool INF>
__device__ __forceinline__ double piece_norm(const T* p, int64_t n, double acc) {
  constexpr int kVec = 16 / (int)sizeof(T), kSteps = kPieceBytes / 16 / kGradThreads, kAll = kPieceBytes / (int)sizeof(T);
  T raw[kSteps][kVec];
  double part[2] = {acc, 0.0};
  auto add = [&](T x, int to) {
    const double v = (double)to_f32(x);
    part[to] = INF ? max_nan(part[to], fabs(v)) : fma(v, v, part[to]);
  };
  if (n >= kAll) {
#pragma unroll
    for (int u = 0; u < kSteps; ++u) __builtin_memcpy(raw[u], p + (u * kGradThreads + threadIdx.x) * kVec, 16);
  } else {
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int at = (u * kGradThreads + threadIdx.x) * kVec;
      __builtin_memset(raw[u], 0, 16);
      if (at + kVec <= n) __builtin_memcpy(raw[u], p + at, 16);
    }
    const int at = (int)n / kVec * kVec + (int)threadIdx.x;
    if (at < n) add(p[at], 0);
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u)
#pragma unroll
    for (int e = 0; e < kVec; ++e) add(raw[u][e], e & 1);
  return join<INF>(part[0], part[1]);
}

// One piece scaled. The stores leave the caches to the gradients that are still to be read (non-temporal): with
// the pieces walked backwards, so that the pass meets first what the norm's pass read last, 250 MB of bf16 into
// new memory take 132 us (both passes; 160 with neither, 135 with the stores alone), 1.05 GB 591 us (628).
typedef u32x4 u32x4_any __attribute__((aligned(2)));
template <typename T>
__device__ __forceinline__ void piece_scale(const T* p, T* out, int64_t n, float f) {
  constexpr int kVec = 16 / (int)sizeof(T), kSteps = kPieceBytes / 16 / kGradThreads, kAll = kPieceBytes / (int)sizeof(T);
  T raw[kSteps][kVec];
  const bool all = n >= kAll;
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int at = (u * kGradThreads + threadIdx.x) * kVec;
    if (all || at + kVec <= n) __builtin_memcpy(raw[u], p + at, 16);
  }
#pragma unroll
  for (int u = 0; u < kSteps; ++u) {
    const int at = (u * kGradThreads + threadIdx.x) * kVec;
    if (all || at + kVec <= n) {
#pragma unroll
      for (int e = 0; e < kVec; ++e) raw[u][e] = from_f32<T>(to_f32(raw[u][e]) * f);
      u32x4 w;
      __builtin_memcpy(&w, raw[u], 16);
      __builtin_nontemporal_store(w, (u32x4_any*)(out + at));
    }
  }
  if (!all) {
    const int at = (int)n / kVec * kVec + (int)threadIdx.x;
    if (at < n) out[at] = from_f32<T>(to_f32(p[at]) * f);
  }
}

// The tensor that piece c lies in: the last whose first piece is at most c. (Empty tensors have no
// pieces: the one after them starts at the same.)
__device__ __forceinline__ int find_tensor(const TensorEntry* e, int count, int64_t c) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (e[mid].first <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct GradRun {
  int count;
  int64_t pieces;
};

// Calls f(entry, its piece) for the workgroup's run of pieces, the last one first where BACK.
template <bool BACK, typename F>
__device__ __forceinline__ void for_pieces(const TensorEntry* e, const GradRun& r, F f) {
  const int64_t c0 = r.pieces * blockIdx.x / gridDim.x, c1 = r.pieces * (blockIdx.x + 1) / gridDim.x;
  if (c0 >= c1) return;
  int k = find_tensor(e, r.count, BACK ? c1 - 1 : c0);
  for (int64_t n = 0; n < c1 - c0; ++n) {
    const int64_t c = BACK ? c1 - 1 - n : c0 + n;
    if (BACK) {
      while (e[k].first > c) --k;
    } else {
      while (k + 1 < r.count && e[k + 1].first <= c) ++k;
    }
    f(e[k], c - e[k].first);
  }
}

template <bool INF>
__device__ __forceinline__ void norm_pieces(const TensorEntry* e, const GradRun& r, double* __restrict__ part) {
  __shared__ double lds[kGradThreads / 64];
  double acc = 0.0;
  for_pieces<false>(e, r, [&](const TensorEntry& t, int64_t c) {
    if (t.dtype == 0) {
      constexpr int64_t kN = kPieceBytes / 4;
      acc = piece_norm<float, INF>((const float*)t.in + c * kN, t.n - c * kN, acc);
    } else {
      constexpr int64_t kN = kPieceBytes / 2;
      if (t.dtype == 1) acc = piece_norm<bf16, INF>((const bf16*)t.in + c * kN, t.n - c * kN, acc);
      else acc = piece_norm<f16, INF>((const f16*)t.in + c * kN, t.n - c * kN, acc);
    }
  });
  acc = block_join<INF>(acc, lds);
  if (threadIdx.x == 0) part[blockIdx.x] = acc;
}

template <bool INF>
__global__ __launch_bounds__(kGradThreads, 8) void grad_norm_kernel(const TensorTable t, const GradRun r, double* __restrict__ part) {
  norm_pieces<INF>(t.entry, r, part);
}
template <bool INF>
__global__ __launch_bounds__(kGradThreads, 8) void grad_norm_many_kernel(const TensorEntry* __restrict__ e, const GradRun r,
                                                                      double* __restrict__ part) {
  norm_pieces<INF>(e, r, part);
}

// The norm from the workgroups' shares, for every thread of a workgroup.
template <bool INF>
__device__ __forceinline__ double total_norm(const double* __restrict__ part, int parts) {
  __shared__ double lds[kGradThreads / 64];
  constexpr int kEach = kGradBlocks / kGradThreads;
  double p[kEach], v = 0.0;
#pragma unroll
  for (int u = 0; u < kEach; ++u) {  // all requested at once
    const int k = u * kGradThreads + threadIdx.x;
    p[u] = k < parts ? part[k] : 0.0;
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u) v = join<INF>(v, p[u]);
  v = block_join<INF>(v, lds);
  return INF ? v : sqrt(v);
}

template <bool INF>
__global__ __launch_bounds__(kGradThreads) void grad_norm_finish_kernel(const double* __restrict__ part, int parts,
                                                                        float* __restrict__ norm) {
  const double v = total_norm<INF>(part, parts);
  if (threadIdx.x == 0) *norm = (float)v;
}

struct ClipArgs {
  const double* part;
  int parts;
  double max_norm;
  float* norm;
  int in_place;
};

template <bool INF>
__device__ __forceinline__ void clip_pieces(const TensorEntry* e, const GradRun& r, const ClipArgs& a) {
  const double norm = total_norm<INF>(a.part, a.parts);
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  const double ratio = a.max_norm / (norm + 1e-6);
  const float f = ratio >= 1.0 || a.max_norm == INFINITY ? 1.f : (float)ratio;  // a NaN stays
  if (a.in_place && f == 1.f) return;
  for_pieces<true>(e, r, [&](const TensorEntry& t, int64_t c) {
    if (t.dtype == 0) {
      constexpr int64_t kN = kPieceBytes / 4;
      piece_scale((const float*)t.in + c * kN, (float*)t.out + c * kN, t.n - c * kN, f);
    } else {
      constexpr int64_t kN = kPieceBytes / 2;
      if (t.dtype == 1) piece_scale((const bf16*)t.in + c * kN, (bf16*)t.out + c * kN, t.n - c * kN, f);
      else piece_scale((const f16*)t.in + c * kN, (f16*)t.out + c * kN, t.n - c * kN, f);
    }
  });
}

template <bool INF>
__global__ __launch_bounds__(kGradThreads, 8) void clip_kernel(const TensorTable t, const GradRun r, const ClipArgs a) {
  clip_pieces<INF>(t.entry, r, a);
}
template <bool INF>
__global__ __launch_bounds__(kGradThreads) void clip_many_kernel(const TensorEntry* __restrict__ e, const GradRun r, const ClipArgs a) {
  clip_pieces<INF>(e, r, a);
}

}  // namespace lce
