// The residual's addition with the RMSNorm of the sum (rows in the input type or in e4m3 with scales),
// and its backward.
//
// A row is held in the registers of the TPR threads that share it: each takes 8 consecutive values (16
// bytes of a 16-bit type) of every 8 TPR, CH times. So every tensor is read and written once, whatever is
// needed of the whole row (the mean square, the largest value, the backward's dot product) in between, and
// an output may be an input's own memory: a row's values are all in registers before any is written. Loads
// and stores are 16 bytes wide at any alignment of the element type; only the last values of a row whose H is
// not a multiple of 8 are stored one by one.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lce_aux.hpp"

namespace lce {

constexpr int kNormVec = 8;

// 8 values of a row as they are stored, in 32-bit registers that hold them until they are needed.
template <typename T>
struct RawRow {
  uint32_t w[kNormVec * sizeof(T) / 4];
  __device__ __forceinline__ float at(int e) const {
    if constexpr (sizeof(T) == 4) {
      return __builtin_bit_cast(float, w[e]);
    } else if constexpr (std::is_same_v<T, bf16>) {
      return __builtin_bit_cast(float, e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    } else {
      return (float)__builtin_bit_cast(f16, (uint16_t)(e & 1 ? w[e / 2] >> 16 : w[e / 2]));
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t& v : w) v = 0u;
  }
  // Drops the first `d` values (1 to 7) and fills up with zeros.
  __device__ __forceinline__ void drop(int d) {
    constexpr int kW = kNormVec * sizeof(T) / 4;
    auto words = [&](int by) {
#pragma unroll
      for (int k = 0; k < kW; ++k) w[k] = k + by < kW ? w[k + by] : 0u;
    };
    if (d & 4) words(kW / 2);
    if (d & 2) words(kW / 4);
    if (d & 1) {
      if constexpr (sizeof(T) == 4) {
        words(1);
      } else {
#pragma unroll
        for (int k = 0; k < kW; ++k) w[k] = w[k] >> 16 | (k + 1 < kW ? w[k + 1] << 16 : 0u);
      }
    }
  }
};
// How rows end. WHOLE: H is a multiple of 8, so a thread's 8 values all exist or none does. PART: a row's last
// values are loaded as the 8 that end the row, and align_end moves them into place, so that they, too, are one
// load that nothing waits for. (Loaded one by one behind a branch they keep the compiler from requesting several
// rows' values together: backward of 8192 x 4097 in bf16 218 us, 95 so, 69 where rows begin at
// 4 bytes.) TINY: H < 8, value by value.
enum RowEnd { WHOLE = 0, PART = 1, TINY = 2 };

// The values at p, of which the first n exist (n <= 0: the registers stay as they are).
template <RowEnd END, typename T>
__device__ __forceinline__ void load_raw(const T* p, int n, RawRow<T>& raw) {
  if constexpr (END == TINY) {
    T v[kNormVec];
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) v[e] = e < n ? p[e] : (T)0.f;
    __builtin_memcpy(raw.w, v, sizeof(v));
  } else if (n > 0) {
    __builtin_memcpy(raw.w, END == WHOLE ? p : p + min(0, n - kNormVec), sizeof(raw.w));
  }
}
template <RowEnd END, typename... Raw>
__device__ __forceinline__ void align_end(int n, Raw&... raw) {
  if constexpr (END == PART) {
    if (n > 0 && n < kNormVec) (raw.drop(kNormVec - n), ...);
  }
}

template <RowEnd END, typename T>
__device__ __forceinline__ void store_row(T* p, int n, const float (&v)[kNormVec]) {
  if (n >= kNormVec) {
    T raw[kNormVec];
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) raw[e] = from_f32<T>(v[e]);
    __builtin_memcpy(p, raw, sizeof(raw));
  } else if constexpr (END != WHOLE) {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e)
      if (e < n) p[e] = from_f32<T>(v[e]);
  }
}

// 8 values in e4m3, to nearest even. All are NaN or at most 448 (up to an fp32 rounding, which goes to
// 448): nothing has to be clamped.
template <RowEnd END>
__device__ __forceinline__ void store_row_fp8(uint8_t* p, int n, const float (&v)[kNormVec]) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    int q = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
    w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], q, true);
  }
  if (n >= kNormVec) {
    __builtin_memcpy(p, w, 8);
  } else if constexpr (END != WHOLE) {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e)
      if (e < n) p[e] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
  }
}

// The TPR threads' sum (or, of bit patterns, maximum) of a row, in a fixed order, for all of them. More
// than a wave's goes through `lds`, one entry per wave; two buffers in turn need one barrier a row. More than four
// waves' are joined in pairs: a chain of 16 would round more often than all that is before it, a thread's 32 terms
// apart. So no value goes through more than 10 joins.
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
    constexpr int kWaves = TPR / 64;
    if constexpr (kWaves > 4) {
      V of[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) of[w] = lds[w];
#pragma unroll
      for (int n = kWaves / 2; n > 0; n /= 2)
#pragma unroll
        for (int w = 0; w < n; ++w) of[w] = Op::of(of[w], of[w + n]);
      v = of[0];
    } else {
      v = lds[0];
#pragma unroll
      for (int w = 1; w < kWaves; ++w) v = Op::of(v, lds[w]);
    }
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
constexpr float kScaleMin = 1.17549435e-38f;  // 2^-126

// e4m3's rounding turns a difference of 2^-24 next to a border into one of 2^-4, so what is rounded is computed to
// better than fp32's rounding. r is in every value and in the scale, so normed / scale = u (448 / top) with
// u = s gamma and top = max |u|; u and 448 / top come with their rounding errors, which cost three instructions a
// value. What is left is the rounding of top and of the result: half as many values as in plain fp32 lie on the
// other side of a border than in 64 bits. (In 64-bit products none do, but 8192 x 4096 in bf16 take
// 48.5 us; 45.4 so, and 43.7 in plain fp32.)
//
// s comes here times r's power of two, and r without it, in [1, 2): u is then at most normed and more than half of
// it, so it leaves fp32 only where normed does. Without that, s gamma of a row of small values may be 2^8 times
// smaller than normed, and 448 / top infinite beside an ordinary scale. (One product a value: 0.7 us of 40.)
struct RowScale {
  float p, r;  // 1 / rms = p r; p a power of two
};
__device__ __forceinline__ RowScale row_scale(float r) {
  // (r = 0 where a value or the mean square is infinite: finite values become 0 at once. A NaN stays one.)
  return {r == 0.f ? 0.f : __builtin_amdgcn_ldexpf(1.f, __builtin_amdgcn_frexp_expf(r) - 1), 2.f * __builtin_amdgcn_frexp_mantf(r)};
}
struct QuantFactor {
  float inv, inv_lo, r;
  bool tiny;  // the scale is at its least: no value is above 448 x 2^-126
};
// From the largest |u| of a group, by its bits (among which a NaN's are above all others). Where the scale is not
// at its least, top is above 448 x 2^-127 and 448 / top at most 2^127.
__device__ __forceinline__ QuantFactor quant_factor(uint32_t top_bits, float r, float& scale) {
  const float top = __builtin_bit_cast(float, top_bits);
  const float sc = top * (r * (1.f / kFp8Max));
  QuantFactor f;
  f.tiny = sc < kScaleMin;  // (a NaN's is not)
  scale = f.tiny ? kScaleMin : sc;
  f.inv = kFp8Max / top;
  f.inv_lo = fmaf(-top, f.inv, kFp8Max) * (f.inv * (1.f / kFp8Max));
  if (r != r) f.inv = r;  // a NaN elsewhere in the row makes all its values NaN
  f.r = r;
  return f;
}
// s becomes what is rounded to e4m3.
template <typename T>
__device__ __forceinline__ void quantise(float (&s)[kNormVec], const RawRow<T>& g, const QuantFactor& f) {
  if (f.tiny) {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) s[e] = s[e] * g.at(e) * f.r * 0x1p126f;
  } else {
#pragma unroll
    for (int e = 0; e < kNormVec; ++e) {
      const float u = s[e] * g.at(e), u_lo = fmaf(s[e], g.at(e), -u);
      s[e] = fmaf(u, f.inv, fmaf(u, f.inv_lo, u_lo * f.inv));
    }
  }
}

// TPR threads a row, several rows a workgroup where TPR is below 256. Bound by HBM: 8192 x 4096 in bf16 with a
// residual 48 us (268 MB, 5.5 TB/s; a large copy moves 5.15), e4m3 in groups of 128 45 us (236 MB, 5.2 TB/s); one
// row 2.6 us, the latency of a load and two barriers.
template <typename T, int TPR, int CH, bool QUANT, RowEnd END>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void add_rmsnorm_kernel(const NormArgs a) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR, kWaves = TPR > 64 ? TPR / 64 : 1;
  __shared__ float sums[2][kWaves];
  __shared__ uint32_t tops[2][kWaves];
  const int t = threadIdx.x % TPR;
  const float inv_h = 1.f / (float)a.H;
  int turn = 0;
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.N; base += (int64_t)gridDim.x * kRows, turn ^= 1) {
    const int64_t i = base + threadIdx.x / TPR;
    const bool live = i < a.N;
    const T *px = (const T*)a.x + i * a.x_ld, *pres = (const T*)a.residual + i * a.residual_ld;
    RawRow<T> x[CH], res[CH], gamma[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
      x[k].clear();
      res[k].clear();
      gamma[k].clear();
      load_raw<END>(px + c, n, x[k]);
      if (a.residual != nullptr) load_raw<END>(pres + c, n, res[k]);
      load_raw<END>((const T*)a.gamma + c, n, gamma[k]);
    }
    float s[CH][kNormVec];
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      align_end<END>(live ? a.H - (k * TPR + t) * kNormVec : 0, x[k], res[k], gamma[k]);
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) {
        s[k][e] = x[k].at(e) + res[k].at(e);
        ss = fmaf(s[k][e], s[k][e], ss);
      }
    }
    ss = row_reduce<TPR, AddOp>(ss, sums[turn]);
    const float r = rsqrtf(fmaf(ss, inv_h, a.eps));
    if (live && t == 0 && a.rstd != nullptr) a.rstd[i] = r;
    uint32_t top = 0;
    const RowScale rs = QUANT ? row_scale(r) : RowScale{};
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
      if (a.added != nullptr) store_row<END>((T*)a.added + i * a.added_ld + c, n, s[k]);
      if constexpr (!QUANT) {
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) s[k][e] = s[k][e] * r * gamma[k].at(e);
        store_row<END>((T*)a.normed + i * a.normed_ld + c, n, s[k]);
      } else {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) s[k][e] *= rs.p;
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) m = MaxOp::of(m, __builtin_bit_cast(uint32_t, s[k][e] * gamma[k].at(e)) & 0x7fffffffu);
        if (a.group == 0) {
          top = MaxOp::of(top, m);
        } else {
          for (int o = 1; o < a.group / kNormVec; o <<= 1) m = MaxOp::of(m, (uint32_t)__shfl_xor((int)m, o));
          float scale;
          const QuantFactor f = quant_factor(m, rs.r, scale);
          if (n > 0 && c % a.group == 0) a.scales[i * ((a.H + a.group - 1) / a.group) + c / a.group] = scale;
          quantise(s[k], gamma[k], f);
          store_row_fp8<END>((uint8_t*)a.normed + i * a.normed_ld + c, n, s[k]);
        }
      }
    }
    if constexpr (QUANT) {
      if (a.group == 0) {
        top = row_reduce<TPR, MaxOp>(top, tops[turn]);
        float scale;
        const QuantFactor f = quant_factor(top, rs.r, scale);
        if (live && t == 0) a.scales[i] = scale;
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const int c = (k * TPR + t) * kNormVec, n = live ? a.H - c : 0;
          quantise(s[k], gamma[k], f);
          store_row_fp8<END>((uint8_t*)a.normed + i * a.normed_ld + c, n, s[k]);
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
//
// Bound by HBM, so the loads may not stop while a row is reduced: AHEAD requests the next row's values
// before the current one's dot product is joined. (A row's barrier and its joins take as long as its
// loads.) What waits in registers waits in the input type. 8192 x 4096 in bf16, all of its tensors: 65 us
// (336 MB, 5.1 TB/s; 106 in the first version, which held more in registers and requested less ahead).
template <typename T, int TPR, int CH, RowEnd END, bool AHEAD>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void add_rmsnorm_backward_kernel(const NormBackwardArgs a) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR, kWaves = TPR > 64 ? TPR / 64 : 1;
  constexpr int kCols = TPR * CH * kNormVec;
  __shared__ float sums[2][kWaves];
  const int t = threadIdx.x % TPR;
  const float inv_h = 1.f / (float)a.H;
  const bool has_res = a.residual != nullptr, has_ds = a.ds != nullptr;
  // Where they would not fit the registers (kWide), dgamma's sums are kept in LDS and gamma is read again for
  // each row (H = 12288 in bf16 fits: 100 us for 4096 rows, 106 so).
  constexpr bool kWide = TPR == 1024 || (TPR == 512 && (CH == 4 || sizeof(T) == 4));
  __shared__ f32x4 wide_acc[kWide ? CH * 2 * TPR : 1];
  float acc[kWide ? 1 : CH][kNormVec];
  RawRow<T> g[kWide ? 1 : CH], x[CH], res[CH], dy[CH], ds[CH];
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = (k * TPR + t) * kNormVec;
    // Columns past the row's end are 0 in registers from here on and add nothing to any sum.
    x[k].clear();
    res[k].clear();
    dy[k].clear();
    ds[k].clear();
    if constexpr (kWide) {
      wide_acc[2 * k * TPR + t] = wide_acc[(2 * k + 1) * TPR + t] = (f32x4){};
    } else {
      g[k].clear();
      load_raw<END>((const T*)a.gamma + c, a.H - c, g[k]);
      align_end<END>(a.H - c, g[k]);
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) acc[k][e] = 0.f;
    }
  }
  const int64_t stride = (int64_t)gridDim.x * kRows;
  float r = 0.f;
  // The last rows' workgroup may have threads without a row: they take the last one again, and leave its
  // gradients out.
  auto request = [&](int64_t i) {
    const int64_t row = min(i, a.N - 1);
    r = a.rstd[row];
    const T *pdy = (const T*)a.dy + row * a.dy_ld, *px = (const T*)a.x + row * a.x_ld;
    const T *pres = (const T*)a.residual + row * a.residual_ld, *pds = (const T*)a.ds + row * a.ds_ld;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = a.H - c;
      load_raw<END>(pdy + c, n, dy[k]);
      load_raw<END>(px + c, n, x[k]);
      if (has_res) load_raw<END>(pres + c, n, res[k]);
      if (has_ds) load_raw<END>(pds + c, n, ds[k]);
    }
  };
  int64_t i = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  int turn = 0;
  if (AHEAD) request(i);
  for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.N; base += stride, i += stride, turn ^= 1) {
    if (!AHEAD) request(i);
    const float ri = r;
    float s[CH][kNormVec];
    RawRow<T> dyi[CH], dsi[CH];
    float dot = 0.f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec;
      align_end<END>(a.H - c, dy[k], x[k], res[k], ds[k]);
      dyi[k] = dy[k];
      dsi[k] = ds[k];
      RawRow<T>& gk = g[kWide ? 0 : k];
      if (kWide) {
        gk.clear();
        load_raw<END>((const T*)a.gamma + c, a.H - c, gk);
        align_end<END>(a.H - c, gk);
      }
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) {
        s[k][e] = x[k].at(e) + res[k].at(e);
        dot = fmaf(dyi[k].at(e) * gk.at(e), s[k][e], dot);
      }
    }
    if (AHEAD && base + stride < a.N) request(i + stride);
    dot = row_reduce<TPR, AddOp>(dot, sums[turn]);
    const float c1 = ri * ri * (dot * inv_h);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec, n = i < a.N ? a.H - c : 0;
      float dx[kNormVec];
      RawRow<T>& gk = g[kWide ? 0 : k];
      if (kWide) {
        gk.clear();
        load_raw<END>((const T*)a.gamma + c, a.H - c, gk);
        align_end<END>(a.H - c, gk);
      }
      if (kRows == 1 || i < a.N) {
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) {
          const float dg = dyi[k].at(e) * (s[k][e] * ri);
          if constexpr (kWide) ((float*)&wide_acc[(2 * k + e / 4) * TPR + t])[e % 4] += dg;
          else acc[k][e] += dg;
        }
      }
#pragma unroll
      for (int e = 0; e < kNormVec; ++e) {
        const float d = dyi[k].at(e);
        dx[e] = fmaf(ri, d * gk.at(e) - s[k][e] * c1, dsi[k].at(e));
      }
      store_row<END>((T*)a.dx + i * a.dx_ld + c, n, dx);
    }
  }
  if (a.part == nullptr) return;
  float* out = a.part + (size_t)blockIdx.x * a.H;
  if constexpr (kRows == 1) {
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TPR + t) * kNormVec;
      if constexpr (kWide) {
#pragma unroll
        for (int e = 0; e < kNormVec; ++e) acc[0][e] = wide_acc[(2 * k + e / 4) * TPR + t][e % 4];
      }
      store_row<END>(out + c, a.H - c, acc[kWide ? 0 : k]);
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

// dgamma_j = sum_b part[b][j] in a fixed order: 16 columns per workgroup, every 64th row of part per thread
// (eight requested at once: 512 rows are one round of loads), then the threads' sums in order. A chain of
// loads, so what counts is how many threads share it.
template <typename T>
__global__ __launch_bounds__(1024) void gamma_sum_kernel(const float* __restrict__ part, int rows, int H,
                                                         T* __restrict__ dgamma) {
  constexpr int kAhead = 8, kCols = 16, kGroups = 64, kWaves = 16;
  __shared__ float sums[kWaves][kCols];
  const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols;
  const int j = blockIdx.x * kCols + col;
  float acc = 0.f;
  if (j < H) {
    for (int b0 = grp; b0 < rows; b0 += kGroups * kAhead) {
      float v[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) v[u] = b0 + kGroups * u < rows ? part[(size_t)(b0 + kGroups * u) * H + j] : 0.f;
#pragma unroll
      for (int u = 0; u < kAhead; ++u) acc += v[u];
    }
  }
#pragma unroll
  for (int o = kCols; o < 64; o <<= 1) acc += __shfl_xor(acc, o);
  if ((threadIdx.x & 63) < kCols) sums[threadIdx.x >> 6][col] = acc;
  __syncthreads();
  if (grp == 0 && j < H) {
    float v = sums[0][col];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) v += sums[w][col];
    dgamma[j] = from_f32<T>(v);
  }
}

}  // namespace lce
