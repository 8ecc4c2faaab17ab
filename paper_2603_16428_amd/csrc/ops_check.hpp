// Argument checks that the operators' C entries share (host code; in a namespace of each source's own).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <utility>

#include "lce.h"
#include "lce_gemm.hpp"

namespace lce {
namespace {

int64_t cdiv(int64_t x, int64_t m) { return (x + m - 1) / m; }
bool dtype_ok(int dtype) { return dtype == LCE_DTYPE_FP32 || dtype == LCE_DTYPE_BF16 || dtype == LCE_DTYPE_FP16; }
int64_t size_of(int dtype) { return dtype == LCE_DTYPE_FP32 ? 4 : 2; }
// Calls f with a value of the element type.
template <typename F>
lce_status_t by_type(int dtype, F f) {
  if (dtype == LCE_DTYPE_BF16) return f(bf16{});
  if (dtype == LCE_DTYPE_FP16) return f(f16{});
  return f(float{});
}
lce_status_t launched() { return hipGetLastError() == hipSuccess ? LCE_OK : LCE_ERR_HIP; }

// ---- row tensors ----

// N rows of `row` bytes, `pitch` bytes apart.
struct Rows {
  const void* p;
  int64_t pitch, row, N;
};

// Whether two tensors share a byte. Rows with one pitch may lie side by side in one buffer (columns
// of a wider one); rows with different pitches count as one block each.
bool overlap(const Rows& a, const Rows& b) {
  if (a.p == nullptr || b.p == nullptr) return false;
  const intptr_t a0 = (intptr_t)a.p, b0 = (intptr_t)b.p;
  const intptr_t a1 = a0 + (a.N - 1) * a.pitch + a.row, b1 = b0 + (b.N - 1) * b.pitch + b.row;
  if (a1 <= b0 || b1 <= a0) return false;
  if (a.pitch != b.pitch || a.pitch == 0) return true;
  const int64_t d = ((b0 - a0) % a.pitch + a.pitch) % a.pitch;  // from one of a's rows to the next of b's
  return d < a.row || d + b.row > a.pitch;
}
bool same(const Rows& a, const Rows& b) { return a.p == b.p && (a.pitch == b.pitch || a.N == 1) && a.row == b.row; }

// Workgroups at most of kernels that walk on over rows.
constexpr int64_t kRowBlocks = int64_t(1) << 20;
constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1, kMaxPitch = int64_t(1) << 30;

// Pitch and alignment of rows (`size`: bytes of an element).
lce_status_t check_pitch(const void* p, int64_t ld, int64_t least, int64_t size) {
  if (p == nullptr) return LCE_OK;
  if (ld < least || (intptr_t)p % size != 0) return LCE_ERR_INVALID_ARGUMENT;
  return ld > kMaxPitch ? LCE_ERR_UNSUPPORTED : LCE_OK;
}

// Outputs against each other, against the inputs `ins`, which the outputs marked true may be in place, and
// against `apart`, which no output may touch.
lce_status_t check_overlaps(std::initializer_list<std::pair<Rows, bool>> outs, std::initializer_list<Rows> ins,
                            std::initializer_list<Rows> apart) {
  for (auto a = outs.begin(); a != outs.end(); ++a) {
    for (auto b = a + 1; b != outs.end(); ++b)
      if (overlap(a->first, b->first)) return LCE_ERR_INVALID_ARGUMENT;
    for (const Rows& in : ins)
      if (overlap(a->first, in) && !(a->second && same(a->first, in))) return LCE_ERR_INVALID_ARGUMENT;
    for (const Rows& in : apart)
      if (overlap(a->first, in)) return LCE_ERR_INVALID_ARGUMENT;
  }
  return LCE_OK;
}

}  // namespace
}  // namespace lce
