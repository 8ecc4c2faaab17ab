// A row's values in registers, 8 a thread, loaded and stored 16 bytes wide at any alignment of the element type.
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

}  // namespace lce
