// C ABI of the operators around the output-layer step (lce_ops.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <vector>

#include "lce_ops.h"
#include "ops_clip.hpp"
#include "ops_rmsnorm.hpp"

namespace lce {
namespace {

int64_t cdiv(int64_t x, int64_t m) { return (x + m - 1) / m; }
bool dtype_ok(int dtype) { return dtype == LCE_DTYPE_FP32 || dtype == LCE_DTYPE_BF16 || dtype == LCE_DTYPE_FP16; }
int64_t size_of(int dtype) { return dtype == LCE_DTYPE_FP32 ? 4 : 2; }
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

constexpr int64_t kMaxRows = (int64_t(1) << 31) - 1, kMaxPitch = int64_t(1) << 30;

lce_status_t check_rows(int64_t N, int64_t H, int dtype) {
  if (N < 0 || H < 1 || !dtype_ok(dtype)) return LCE_ERR_INVALID_ARGUMENT;
  return N > kMaxRows || H > LCE_NORM_MAX_H ? LCE_ERR_UNSUPPORTED : LCE_OK;
}
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

// ---- which threads share a row ----

// The threads that share a row, and their steps of 8 values. A wave or less needs no barrier, so up to 1024 values
// are a wave's (32768 x 1024 in bf16, 128 threads against 64: forward 47.5 us against 47.3, backward 66.8 against
// 65.9) or the part of one that they fill (131072 x 256: a whole wave, half of it idle, 51.8 and 78.9 us; 32 threads
// 47.6 and 66.5); but no wave takes more steps instead of more threads, which few rows wait for (24 x 2048: 64
// threads in four steps 3.1 and 6.2 us, 256 in one 2.5 and 4.7). Above, workgroups of 256 threads as long as four
// steps do, then of 512 (4096 x 8192 in two steps of 512: 48.4 and 68.5 us against 49.0 and 69.2, e4m3 51.1 against
// 49.7), of 1024 only where those do not hold the row (2730 x 12288: 51.8 and 77.5 us against 49.1 and 73.3).
template <typename F>
void by_width(int64_t H, F f) {
  auto go = [&](auto tpr, auto ch) { f(tpr, ch); };
  using std::integral_constant;
#define LCE_WIDTH(TPR, CH) \
  if (H <= (TPR) * (CH) * kNormVec) return go(integral_constant<int, TPR>{}, integral_constant<int, CH>{})
  LCE_WIDTH(16, 1);
  LCE_WIDTH(32, 1);
  LCE_WIDTH(64, 1);
  LCE_WIDTH(64, 2);
  LCE_WIDTH(256, 1);
  LCE_WIDTH(256, 2);
  LCE_WIDTH(256, 3);
  LCE_WIDTH(256, 4);
  LCE_WIDTH(512, 3);
  LCE_WIDTH(512, 4);
  LCE_WIDTH(1024, 4);
#undef LCE_WIDTH
}
static_assert(1024 * 4 * kNormVec == LCE_NORM_MAX_H, "the widest variant");

constexpr int threads_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// Workgroups of the forward: one per group of rows (the kernel walks on where a grid that large is not
// allowed).
constexpr int64_t kForwardBlocks = int64_t(1) << 20;
// Workgroups of the backward, each of which leaves H fp32 sums for dgamma: no more than keep the loads going.
// One per CU where a thread holds 16 or more values of a row and those of the next one (8192 x 4096 in bf16:
// 65 us, 68 with two, 76 with four), two where it holds 8 (16384 x 2048: 64 us, 70 with one; 262144 x 128: 42
// and 58). Of fewer rows than that each takes one, or two where the sums of one each would be 2 MB or more
// (512 x 2048: 8.2 us against 10.2, 256 x 4096: 8.8 against 10.0; but 128 x 2048: 6.5 against 6.0).
constexpr int64_t kGammaSums = int64_t(1) << 19;
struct BackwardGrid {
  int64_t rows, most;  // rows a workgroup takes at a time; workgroups at most
};
BackwardGrid backward_grid(int64_t H) {
  BackwardGrid g{1, 256};
  by_width(H, [&](auto tpr, auto ch) {
    constexpr int kTpr = decltype(tpr)::value;
    g.rows = threads_of(kTpr) / kTpr;
    if (decltype(ch)::value == 1) g.most = 512;
  });
  return g;
}
int64_t backward_blocks(int64_t N, int64_t H) {
  const BackwardGrid g = backward_grid(H);
  int64_t blocks = cdiv(N, g.rows);
  if (blocks * H >= kGammaSums) blocks = cdiv(blocks, 2);
  return std::max<int64_t>(1, std::min(blocks, g.most));
}
// The most workgroups that N rows or fewer take: the last number of rows before two a workgroup may take more than N.
// (So a workspace for N rows serves any smaller batch.)
int64_t workspace_blocks(int64_t N, int64_t H) {
  const int64_t one_each = (kGammaSums - 1) / H * backward_grid(H).rows;
  return std::max(backward_blocks(N, H), backward_blocks(std::min(N, one_each), H));
}

template <typename T, bool QUANT>
lce_status_t run_forward(const NormArgs& a, hipStream_t s) {
  by_width(a.H, [&](auto tpr, auto ch) {
    constexpr int kTpr = decltype(tpr)::value, kCh = decltype(ch)::value, kThreads = threads_of(kTpr);
    const int64_t blocks = std::min(cdiv(a.N, kThreads / kTpr), kForwardBlocks);
    auto kernel = a.H % kNormVec == 0 ? add_rmsnorm_kernel<T, kTpr, kCh, QUANT, WHOLE> : add_rmsnorm_kernel<T, kTpr, kCh, QUANT, PART>;
    if constexpr (kTpr == 16)
      if (a.H < kNormVec) kernel = add_rmsnorm_kernel<T, kTpr, kCh, QUANT, TINY>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, a);
  });
  return launched();
}

template <typename T>
lce_status_t run_backward(const NormBackwardArgs& a, int64_t blocks, void* dgamma, hipStream_t s) {
  if (a.N > 0)
    by_width(a.H, [&](auto tpr, auto ch) {
      constexpr int kTpr = decltype(tpr)::value, kCh = decltype(ch)::value;
      constexpr bool kAhead = kTpr < 512 || (kTpr == 512 && (kCh < 4 || sizeof(T) == 2));  // as registers allow
      auto kernel = a.H % kNormVec == 0 ? add_rmsnorm_backward_kernel<T, kTpr, kCh, WHOLE, kAhead>
                                        : add_rmsnorm_backward_kernel<T, kTpr, kCh, PART, kAhead>;
      if constexpr (kTpr == 16)
        if (a.H < kNormVec) kernel = add_rmsnorm_backward_kernel<T, kTpr, kCh, TINY, kAhead>;
      hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(threads_of(kTpr)), 0, s, a);
    });
  if (dgamma != nullptr)
    hipLaunchKernelGGL(gamma_sum_kernel<T>, dim3((unsigned)cdiv(a.H, 16)), dim3(1024), 0, s, a.part,
                       a.N > 0 ? (int)blocks : 0, a.H, (T*)dgamma);
  return launched();
}

bool eps_ok(float eps) { return eps >= 0.f && std::isfinite(eps); }

// ---- lists of tensors ----

// The pieces of each entry; the total, or -1 where the kernels' 32-bit numbers would not hold it.
int64_t count_pieces(const lce_tensor_t* grads, int64_t count, std::vector<TensorEntry>& table, void* const* out) {
  int64_t pieces = 0;
  for (int64_t k = 0; k < count; ++k) {
    const lce_tensor_t& g = grads[k];
    table[k] = {g.data, out != nullptr ? out[k] : g.data, g.n, (int32_t)pieces, g.dtype};
    if (g.n > (int64_t(1) << 47)) return -1;
    pieces += cdiv(g.n * size_of(g.dtype), kPieceBytes);
    if (pieces > INT32_MAX) return -1;
  }
  return pieces;
}

// Whether the norm or the workspace, which every call writes, overlap each other or a gradient.
bool norm_overlaps(const std::vector<TensorEntry>& table, const float* norm, const void* workspace) {
  const int64_t space = (int64_t)lce_grad_norm_workspace_size((int64_t)table.size());
  const Rows n{norm, sizeof(float), sizeof(float), 1}, w{workspace, space, space, 1};
  if (overlap(n, w)) return true;
  for (const TensorEntry& e : table) {
    const int64_t bytes = e.n * size_of(e.dtype);
    const Rows g{bytes > 0 ? e.in : nullptr, bytes, bytes, 1};
    if (overlap(g, n) || overlap(g, w)) return true;
  }
  return false;
}

// Whether memory that a clip writes (the norm and the workspace too) overlaps any other of the call; out[k] may
// be grads[k].data.
bool clip_overlaps(const std::vector<TensorEntry>& table, const float* norm, const void* workspace) {
  struct Range {
    uintptr_t lo, hi;
    bool written;
  };
  std::vector<Range> r;
  r.reserve(2 * table.size() + 2);
  r.push_back({(uintptr_t)norm, (uintptr_t)norm + sizeof(float), true});
  r.push_back({(uintptr_t)workspace, (uintptr_t)workspace + lce_grad_norm_workspace_size((int64_t)table.size()), true});
  for (const TensorEntry& e : table) {
    const uintptr_t bytes = (uintptr_t)(e.n * size_of(e.dtype));
    if (bytes == 0) continue;
    r.push_back({(uintptr_t)e.out, (uintptr_t)e.out + bytes, true});
    if (e.in != e.out) r.push_back({(uintptr_t)e.in, (uintptr_t)e.in + bytes, false});
  }
  auto before = [](const Range& a, const Range& b) { return a.lo < b.lo; };
  if (!std::is_sorted(r.begin(), r.end(), before)) std::sort(r.begin(), r.end(), before);
  uintptr_t any = 0, written = 0;  // the furthest ends so far
  for (const Range& x : r) {
    if (x.lo < (x.written ? any : written)) return true;
    any = std::max(any, x.hi);
    if (x.written) written = std::max(written, x.hi);
  }
  return false;
}

size_t table_bytes(int64_t count) { return count > kInlineTensors ? (size_t)cdiv(count * (int64_t)sizeof(TensorEntry), 256) * 256 : 0; }

// Launches with the table among the arguments, or in the workspace after the shares of the norm.
template <typename Inline, typename Many>
void with_table(const std::vector<TensorEntry>& table, void* workspace, bool fill, hipStream_t s, Inline inl, Many many) {
  const int64_t count = (int64_t)table.size();
  TensorTable t;
  if (count <= kInlineTensors) {
    std::copy(table.begin(), table.end(), t.entry);
    inl(t);
    return;
  }
  TensorEntry* dst = (TensorEntry*)((char*)workspace + kGradBlocks * sizeof(double));
  for (int64_t k = 0; fill && k < count; k += kInlineTensors) {
    const int n = (int)std::min<int64_t>(kInlineTensors, count - k);
    std::copy(table.begin() + k, table.begin() + k + n, t.entry);
    hipLaunchKernelGGL(grad_table_kernel, dim3(1), dim3(128), 0, s, t, n, dst + k);
  }
  many(dst);
}

template <bool INF>
lce_status_t run_norm(const std::vector<TensorEntry>& table, int64_t pieces, bool clip, bool in_place, float max_norm,
                      float* norm, void* workspace, hipStream_t s) {
  double* part = (double*)workspace;
  const unsigned blocks = (unsigned)std::max<int64_t>(1, std::min<int64_t>(pieces, kGradBlocks));
  const GradRun run{(int)table.size(), pieces};
  with_table(table, workspace, true, s,
             [&](const TensorTable& t) {
               hipLaunchKernelGGL(grad_norm_kernel<INF>, dim3(blocks), dim3(kGradThreads), 0, s, t, run, part);
             },
             [&](const TensorEntry* e) {
               hipLaunchKernelGGL(grad_norm_many_kernel<INF>, dim3(blocks), dim3(kGradThreads), 0, s, e, run, part);
             });
  if (!clip) {
    hipLaunchKernelGGL(grad_norm_finish_kernel<INF>, dim3(1), dim3(kGradThreads), 0, s, part, (int)blocks, norm);
    return launched();
  }
  const ClipArgs a{part, (int)blocks, (double)max_norm, norm, in_place ? 1 : 0};
  with_table(table, workspace, false, s,
             [&](const TensorTable& t) {
               hipLaunchKernelGGL(clip_kernel<INF>, dim3(blocks), dim3(kGradThreads), 0, s, t, run, a);
             },
             [&](const TensorEntry* e) {
               hipLaunchKernelGGL(clip_many_kernel<INF>, dim3(blocks), dim3(kGradThreads), 0, s, e, run, a);
             });
  return launched();
}

lce_status_t grad_norm_call(const lce_tensor_t* grads, int64_t count, int norm_type, bool clip, float max_norm,
                            void* const* out, float* norm, void* workspace, size_t workspace_bytes, hipStream_t s) {
  if (!grads || count < 1 || !norm || (norm_type != LCE_NORM_L2 && norm_type != LCE_NORM_INF) || !(max_norm >= 0.f) ||
      (uintptr_t)norm % sizeof(float) != 0)
    return LCE_ERR_INVALID_ARGUMENT;
  if (count > INT32_MAX) return LCE_ERR_UNSUPPORTED;
  for (int64_t k = 0; k < count; ++k) {
    if (grads[k].n < 0 || !dtype_ok(grads[k].dtype)) return LCE_ERR_INVALID_ARGUMENT;
    if (grads[k].n > 0 && (!grads[k].data || (out != nullptr && !out[k]))) return LCE_ERR_INVALID_ARGUMENT;
    const uintptr_t bits = (uintptr_t)grads[k].data | (out != nullptr ? (uintptr_t)out[k] : 0);
    if (bits % size_of(grads[k].dtype) != 0) return LCE_ERR_INVALID_ARGUMENT;
  }
  try {  // the host's own memory: no exception leaves a C entry
    std::vector<TensorEntry> table((size_t)count);
    const int64_t pieces = count_pieces(grads, count, table, out);
    if (pieces < 0) return LCE_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < lce_grad_norm_workspace_size(count)) return LCE_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace % 256 != 0 || (clip ? clip_overlaps : norm_overlaps)(table, norm, workspace)) return LCE_ERR_INVALID_ARGUMENT;
    return norm_type == LCE_NORM_INF ? run_norm<true>(table, pieces, clip, out == nullptr, max_norm, norm, workspace, s)
                                     : run_norm<false>(table, pieces, clip, out == nullptr, max_norm, norm, workspace, s);
  } catch (...) {
    return LCE_ERR_HIP;
  }
}

// The forward's common checks and arguments; `normed_row`: bytes of an output row.
lce_status_t forward_args(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld, const void* gamma,
                          int64_t N, int64_t H, int dtype, float eps, void* normed, int64_t normed_ld,
                          int64_t normed_size, float* scales, int64_t groups, void* added, int64_t added_ld,
                          float* rstd, NormArgs& a) {
  lce_status_t st = check_rows(N, H, dtype);
  if (st != LCE_OK) return st;
  if (!eps_ok(eps)) return LCE_ERR_INVALID_ARGUMENT;
  if (N == 0) return LCE_OK;
  if (!x || !gamma || !normed) return LCE_ERR_INVALID_ARGUMENT;
  const int64_t z = size_of(dtype);
  for (const lce_status_t e : {check_pitch(x, x_ld, 0, z), check_pitch(residual, residual_ld, 0, z), check_pitch(gamma, H, H, z),
                               check_pitch(normed, normed_ld, H, normed_size), check_pitch(added, added_ld, H, z),
                               check_pitch(rstd, 1, 1, 4), check_pitch(scales, groups, groups, 4)})
    if (e != LCE_OK) return e;
  const bool quant = scales != nullptr;
  st = check_overlaps({{{normed, normed_ld * normed_size, H * normed_size, N}, !quant},
                       {{added, added_ld * z, H * z, N}, true},
                       {{rstd, 4, 4, N}, false},
                       {{scales, 4 * groups, 4 * groups, N}, false}},
                      {{x, x_ld * z, H * z, N}, {residual, residual_ld * z, H * z, N}},
                      {{gamma, H * z, H * z, 1}});
  if (st != LCE_OK) return st;
  a = {x, residual, gamma, normed, added, rstd, scales, x_ld, residual_ld, normed_ld, added_ld, N, (int)H, 0, eps};
  return LCE_OK;
}

}  // namespace
}  // namespace lce

extern "C" {

lce_status_t lce_add_rmsnorm_forward(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld,
                                     const void* gamma, int64_t N, int64_t H, int dtype, float eps, void* normed,
                                     int64_t normed_ld, void* added, int64_t added_ld, float* rstd, void* stream) {
  lce::NormArgs a;
  const lce_status_t st = lce::forward_args(x, x_ld, residual, residual_ld, gamma, N, H, dtype, eps, normed, normed_ld,
                                            lce::size_of(dtype), nullptr, 0, added, added_ld, rstd, a);
  if (st != LCE_OK || N == 0) return st;
  hipStream_t s = (hipStream_t)stream;
  if (dtype == LCE_DTYPE_BF16) return lce::run_forward<lce::bf16, false>(a, s);
  if (dtype == LCE_DTYPE_FP16) return lce::run_forward<lce::f16, false>(a, s);
  return lce::run_forward<float, false>(a, s);
}

lce_status_t lce_add_rmsnorm_quant(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld,
                                   const void* gamma, int64_t N, int64_t H, int dtype, float eps, int group,
                                   void* quantised, int64_t quantised_ld, float* scales, void* added,
                                   int64_t added_ld, float* rstd, void* stream) {
  if (group != 0 && group != 32 && group != 64 && group != 128) return LCE_ERR_INVALID_ARGUMENT;
  if (N > 0 && !scales) return LCE_ERR_INVALID_ARGUMENT;
  lce::NormArgs a;
  const lce_status_t st =
      lce::forward_args(x, x_ld, residual, residual_ld, gamma, N, H, dtype, eps, quantised, quantised_ld, 1, scales,
                        group == 0 ? 1 : lce::cdiv(H, group), added, added_ld, rstd, a);
  if (st != LCE_OK || N == 0) return st;
  a.group = group;
  hipStream_t s = (hipStream_t)stream;
  if (dtype == LCE_DTYPE_BF16) return lce::run_forward<lce::bf16, true>(a, s);
  if (dtype == LCE_DTYPE_FP16) return lce::run_forward<lce::f16, true>(a, s);
  return lce::run_forward<float, true>(a, s);
}

size_t lce_add_rmsnorm_workspace_size(int64_t N, int64_t H, int dtype) {
  if (lce::check_rows(N, H, dtype) != LCE_OK) return 0;
  return (size_t)lce::cdiv(lce::workspace_blocks(N, H) * H * 4, 256) * 256;
}

lce_status_t lce_add_rmsnorm_backward(const void* grad_normed, int64_t grad_normed_ld, const void* grad_added,
                                      int64_t grad_added_ld, const void* x, int64_t x_ld, const void* residual,
                                      int64_t residual_ld, const void* gamma, const float* rstd, int64_t N, int64_t H,
                                      int dtype, void* grad_hidden, int64_t grad_hidden_ld, void* grad_gamma,
                                      void* workspace, size_t workspace_bytes, void* stream) {
  lce_status_t st = lce::check_rows(N, H, dtype);
  if (st != LCE_OK) return st;
  const int64_t z = lce::size_of(dtype);
  if (N > 0) {
    if (!grad_normed || !x || !gamma || !rstd || !grad_hidden) return LCE_ERR_INVALID_ARGUMENT;
    for (const lce_status_t e :
         {lce::check_pitch(grad_normed, grad_normed_ld, 0, z), lce::check_pitch(grad_added, grad_added_ld, 0, z),
          lce::check_pitch(x, x_ld, 0, z), lce::check_pitch(residual, residual_ld, 0, z), lce::check_pitch(gamma, H, H, z),
          lce::check_pitch(rstd, 1, 1, 4), lce::check_pitch(grad_hidden, grad_hidden_ld, H, z), lce::check_pitch(grad_gamma, H, H, z)})
      if (e != LCE_OK) return e;
    const int64_t space = (int64_t)lce_add_rmsnorm_workspace_size(N, H, dtype);
    st = lce::check_overlaps({{{grad_hidden, grad_hidden_ld * z, H * z, N}, true},
                              {{grad_gamma, H * z, H * z, 1}, false},
                              {{grad_gamma != nullptr ? workspace : nullptr, space, space, 1}, false}},
                             {{grad_normed, grad_normed_ld * z, H * z, N},
                              {grad_added, grad_added_ld * z, H * z, N},
                              {x, x_ld * z, H * z, N},
                              {residual, residual_ld * z, H * z, N}},
                             {{gamma, H * z, H * z, 1}, {rstd, 4, 4, N}});
    if (st != LCE_OK) return st;
  }
  if (grad_gamma != nullptr) {
    if (!workspace || workspace_bytes < lce_add_rmsnorm_workspace_size(N, H, dtype)) return LCE_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace % 256 != 0) return LCE_ERR_INVALID_ARGUMENT;
  }
  if (N == 0 && grad_gamma == nullptr) return LCE_OK;
  const lce::NormBackwardArgs a{grad_normed, grad_added, x, residual, gamma, rstd, grad_hidden,
                                grad_gamma != nullptr ? (float*)workspace : nullptr, grad_normed_ld, grad_added_ld,
                                x_ld, residual_ld, grad_hidden_ld, N, (int)H};
  const int64_t blocks = lce::backward_blocks(N, H);
  hipStream_t s = (hipStream_t)stream;
  if (dtype == LCE_DTYPE_BF16) return lce::run_backward<lce::bf16>(a, blocks, grad_gamma, s);
  if (dtype == LCE_DTYPE_FP16) return lce::run_backward<lce::f16>(a, blocks, grad_gamma, s);
  return lce::run_backward<float>(a, blocks, grad_gamma, s);
}

size_t lce_grad_norm_workspace_size(int64_t count) {
  if (count < 1 || count > INT32_MAX) return 0;
  return lce::kGradBlocks * sizeof(double) + lce::table_bytes(count);
}

lce_status_t lce_grad_norm(const lce_tensor_t* grads, int64_t count, int norm_type, float* norm, void* workspace,
                           size_t workspace_bytes, void* stream) {
  return lce::grad_norm_call(grads, count, norm_type, false, 0.f, nullptr, norm, workspace, workspace_bytes,
                             (hipStream_t)stream);
}

lce_status_t lce_clip_grad_norm(const lce_tensor_t* grads, int64_t count, int norm_type, float max_norm,
                                void* const* out, float* norm, void* workspace, size_t workspace_bytes, void* stream) {
  return lce::grad_norm_call(grads, count, norm_type, true, max_norm, out, norm, workspace, workspace_bytes,
                             (hipStream_t)stream);
}

}  // extern "C"
