/*
 * lce_ops.h -- C ABI of the operators on either side of the output-layer step (lce.h) for MI355X
 * (gfx950): the residual's addition with the RMSNorm of the sum in front of it (rows in the input
 * type or in 8 bits with scales, and the backward), and the global norm of many gradients with its
 * clipping behind it.
 *
 * Conventions are those of lce.h (device pointers owned by the caller, work enqueued in order on
 * `stream`, which belongs to the current device, no allocation and no synchronisation, arguments
 * validated before anything is enqueued, status codes, deterministic results), except:
 *   - Tensors need only their element type's alignment (any other gives LCE_ERR_INVALID_ARGUMENT).
 *   - Row tensors [N, H] have a pitch of their own (`*_ld`, elements between rows): any for an input,
 *     0 included (one row for all), at least H for an output. The H values of a row are consecutive.
 *   - N >= 0 (N = 0 does nothing), H from 1 to LCE_NORM_MAX_H, any values: rows need not be whole
 *     16-byte pieces.
 */
#ifndef LCE_OPS_H_
#define LCE_OPS_H_

#include "lce.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * s = x + residual (x alone where residual is NULL), and the RMSNorm of s:
 *
 *     r_i = 1 / sqrt(mean_j s_ij^2 + eps),   normed_ij = s_ij r_i gamma_j
 *
 * in fp32, each output rounded once to its type. The norm takes s before its rounding to `dtype`.
 *   x, residual : device [N,H] of dtype; residual may be NULL.
 *   gamma       : device [H] of dtype.
 *   eps         : >= 0 and finite. The mean square has to stay within fp32: values below about 1e19, and
 *                 with eps = 0 above about 1e-18 (a row of zeros then gives NaN).
 *   normed      : device [N,H] of dtype.
 *   added       : device [N,H] of dtype, receives s; NULL where it is not wanted.
 *   rstd        : device fp32 [N], receives r (the backward needs it); NULL where it is not wanted.
 * An output may be an input's own memory (same pointer and pitch, as in a residual stream updated in
 * place); other overlaps of outputs with inputs or with each other give LCE_ERR_INVALID_ARGUMENT.
 */
#define LCE_NORM_MAX_H 32768
lce_status_t lce_add_rmsnorm_forward(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld,
                                     const void* gamma, int64_t N, int64_t H, int dtype, float eps,
                                     void* normed, int64_t normed_ld, void* added, int64_t added_ld,
                                     float* rstd, void* stream);

/*
 * The same with the normalised rows in 8 bits (OCP e4m3: 4 exponent bits, 3 mantissa bits, largest
 * 448, no infinities) and a scale for each group of consecutive values of a row:
 *
 *     scale_ig = max(max_{j in g} |normed_ij| / 448, 2^-126),   quantised_ij = e4m3(normed_ij / scale_ig)
 *
 * from the unrounded values of normed, to nearest even.
 *   group      : 32, 64 or 128 values (the row's last group may be shorter), or 0: the whole row.
 *   quantised  : device bytes [N,H] (pitch in bytes).
 *   scales     : device fp32 [N, ceil(H / group)] ([N, 1] for group 0), row-major. Not
 *                finite where its group holds a value that is not (its quantised values are NaN then).
 * quantised and scales overlap no other tensor of the call.
 */
lce_status_t lce_add_rmsnorm_quant(const void* x, int64_t x_ld, const void* residual, int64_t residual_ld,
                                   const void* gamma, int64_t N, int64_t H, int dtype, float eps, int group,
                                   void* quantised, int64_t quantised_ld, float* scales,
                                   void* added, int64_t added_ld, float* rstd, void* stream);

/*
 * The backward of lce_add_rmsnorm_forward (and, with the rounding taken as the identity, of
 * lce_add_rmsnorm_quant), given the upstream gradients of normed and of added:
 *
 *     c_i = (1/H) sum_k grad_normed_ik gamma_k s_ik
 *     grad_hidden_ij = r_i gamma_j grad_normed_ij - r_i^3 s_ij c_i + grad_added_ij
 *     grad_gamma_j   = sum_i grad_normed_ij s_ij r_i
 *
 * grad_hidden is the gradient of x and of the residual alike.
 *   grad_normed : device [N,H] of dtype.
 *   grad_added  : device [N,H] of dtype; NULL: nothing came back through added.
 *   x, residual : as the forward call had them, so that s is the same unrounded sum. A caller that
 *                 keeps one tensor instead of two passes added for x and NULL: s is then off by its
 *                 rounding to dtype.
 *   rstd        : r of the forward call.
 *   grad_hidden : device [N,H] of dtype; may be grad_normed's, grad_added's, x's or residual's own
 *                 memory.
 *   grad_gamma  : device [H] of dtype, summed over the rows in fp32 in a fixed order; NULL where it is
 *                 not wanted (no workspace then). N = 0 gives zeros.
 *   workspace   : device memory of lce_add_rmsnorm_workspace_size(N, H, dtype) bytes, 256-byte aligned.
 *                 The size does not fall as N grows: one for the largest batch serves the smaller ones.
 */
size_t lce_add_rmsnorm_workspace_size(int64_t N, int64_t H, int dtype);
lce_status_t lce_add_rmsnorm_backward(const void* grad_normed, int64_t grad_normed_ld, const void* grad_added,
                                      int64_t grad_added_ld, const void* x, int64_t x_ld, const void* residual,
                                      int64_t residual_ld, const void* gamma, const float* rstd, int64_t N,
                                      int64_t H, int dtype, void* grad_hidden, int64_t grad_hidden_ld,
                                      void* grad_gamma, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The norm over all values of many tensors (a model's gradients) as if they were one vector, and
 * gradients scaled so that it is at most max_norm:
 *
 *     norm = sqrt(sum_k g_k^2)   (LCE_NORM_L2)   or   max_k |g_k|   (LCE_NORM_INF)
 *     factor = min(1, max_norm / (norm + 1e-6));   out = g factor (in fp32, rounded once)
 *
 * Squares are summed in fp64: no value of the types under- or overflows the sum. A NaN among the
 * values makes the norm NaN, and every clipped gradient too; an infinite norm has factor 0 (finite
 * values become 0, infinite ones NaN).
 *   grads     : `count` (>= 1) entries in HOST memory, read during the call; `data` is device memory of
 *               n >= 0 consecutive values of `dtype` (NULL where n = 0). Types may differ.
 *   out       : NULL: the gradients themselves are scaled (and, within the limit, not written at all).
 *               Otherwise `count` device pointers in HOST memory, which receive the scaled values in
 *               the gradient's type. Memory that is written overlaps no other tensor of the call, but
 *               out[k] may be grads[k].data; else LCE_ERR_INVALID_ARGUMENT.
 *   max_norm  : >= 0; infinity makes the factor 1 whatever the norm is.
 *   norm      : device fp32 [1].
 *   workspace : device memory of lce_grad_norm_workspace_size(count) bytes, 256-byte aligned. Calls
 *               (and captured graphs) that may run at the same time need one each.
 * norm and workspace overlap no tensor of the call and not each other, else LCE_ERR_INVALID_ARGUMENT;
 * gradients that are only read (lce_grad_norm) may overlap.
 * All the values together are below 2^31 pieces of 16 KB.
 */
typedef struct {
  void* data;
  int64_t n;
  int32_t dtype;    /* an lce_dtype_t value */
  int32_t reserved; /* 0 */
} lce_tensor_t;
typedef enum { LCE_NORM_L2 = 0, LCE_NORM_INF = 1 } lce_norm_t;
size_t lce_grad_norm_workspace_size(int64_t count);
lce_status_t lce_grad_norm(const lce_tensor_t* grads, int64_t count, int norm_type, float* norm,
                           void* workspace, size_t workspace_bytes, void* stream);
lce_status_t lce_clip_grad_norm(const lce_tensor_t* grads, int64_t count, int norm_type, float max_norm,
                                void* const* out, float* norm, void* workspace, size_t workspace_bytes,
                                void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LCE_OPS_H_ */
