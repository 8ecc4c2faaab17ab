/*
 * lce_vocab.h -- C ABI of the operators on the vocabulary's matrix and logits beside the output-layer step (lce.h) for
 * MI355X (gfx950): the embedding lookup and its gradient, rows and weights in 4 bits and their product, and the choice
 * of a token from logits.
 *
 * Conventions are those of lce_ops.h: device pointers owned by the caller, work enqueued in order on `stream`, which
 * belongs to the current device, no allocation and no synchronisation, arguments validated before anything is enqueued,
 * deterministic results; tensors need only their element type's alignment unless noted; row tensors have a pitch of their
 * own (`*_ld`, elements between rows): any for an input, 0 included, at least the row's length for an output; no rows are
 * a call that does nothing. Outputs overlap neither inputs nor each other, else LCE_ERR_INVALID_ARGUMENT.
 */
#ifndef LCE_VOCAB_H_
#define LCE_VOCAB_H_

#include "lce.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * out_i = scale weight_{t_i}, in fp32, rounded once. A token outside [0, V) gives a row of NaN and reads nothing.
 *   tokens      : device [N], integers of token_bytes (4 or 8) bytes.
 *   weight      : device [V,H] of dtype, 1 <= V < 2^31, 1 <= H <= LCE_EMBEDDING_MAX_H.
 *   scale       : finite.
 *   out         : device [N,H] of dtype.
 */
#define LCE_EMBEDDING_MAX_H (1 << 20)
lce_status_t lce_embedding_forward(const void* tokens, int token_bytes, int64_t N, const void* weight, int64_t weight_ld,
                                   int64_t V, int64_t H, int dtype, float scale, void* out, int64_t out_ld, void* stream);

/*
 * The gradient of weight: for each v, scale times the sum of grad's rows whose token is v, in fp32 in an order that the tokens
 * alone fix, rounded once.
 *   grad        : device [N,H] of dtype, N <= LCE_EMBEDDING_MAX_N.
 *   padding_idx : a token whose rows count for nothing, or -1. Tokens outside [0, V) count for nothing either.
 *   grad_weight : device [V,H] of dtype. accumulate = 0: all of it is written, zeros where no token points. Otherwise the sum is
 *                 added to the value there (in fp32, rounded once), and only rows that a counting token names are touched.
 *   workspace   : device memory of lce_embedding_workspace_size(N, H) bytes, 256-byte aligned. The size does not
 *                 fall as N or H grows. Calls (and captured graphs) that may run at the same time need one each.
 */
#define LCE_EMBEDDING_MAX_N (1 << 28)
size_t lce_embedding_workspace_size(int64_t N, int64_t H);
lce_status_t lce_embedding_backward(const void* grad, int64_t grad_ld, const void* tokens, int token_bytes, int64_t N,
                                    int64_t V, int64_t H, int dtype, float scale, int64_t padding_idx, void* grad_weight,
                                    int64_t grad_weight_ld, int accumulate, void* workspace, size_t workspace_bytes,
                                    void* stream);

/*
 * Rows in 4 bits with a scale for each 32 consecutive values (OCP MXFP4): H a multiple of 32, 32 <= H <= LCE_MXFP4_MAX_H.
 *
 *     scale_ig = 2^e, e = max(floor(log2(max_{j in g} |x_ij|)) - 2, -127);   code_ij = e2m1(x_ij / scale_ig)
 *
 * to nearest even; magnitudes above 6 become 6. A group of zeros has e = -127, one that holds a NaN or an infinity the
 * scale byte 255 (NaN) and codes 0.
 *   x           : device [N,H] of dtype.
 *   codes       : device bytes [N, H/2], contiguous, 16-byte aligned: sign, two bits of exponent, one of mantissa (0, 0.5, 1,
 *                 1.5, 2, 3, 4, 6), the first value of two in a byte's low half.
 *   scales      : device bytes [N, H/32], contiguous: e + 127.
 */
#define LCE_MXFP4_MAX_H (1 << 20)
lce_status_t lce_mxfp4_quantize(const void* x, int64_t x_ld, int64_t N, int64_t H, int dtype, void* codes, void* scales,
                                void* stream);
/* The values that codes and scales stand for, in dtype, rounded once (NaN in groups of scale byte 255). */
lce_status_t lce_mxfp4_dequantize(const void* codes, const void* scales, int64_t N, int64_t H, int dtype, void* y,
                                  int64_t y_ld, void* stream);
/*
 * out = X W^T for X [M,H] and W [V,H] in 4 bits, summed in fp32 and rounded once to dtype.
 *   codes, scales : as lce_mxfp4_quantize leaves them. A group whose scale byte is 255 makes the sums that it enters NaN.
 *   out           : device [M,V] of dtype. M, V >= 0 (M, V < 2^31; for M > 128 at most LCE_MXFP4_MAX_TILES tiles of 256 x 256 values,
 *                   for M from 49 to 128 as many of M x 256, else LCE_ERR_UNSUPPORTED).
 */
#define LCE_MXFP4_MAX_TILES (1 << 22)
lce_status_t lce_mxfp4_matmul(const void* x_codes, const void* x_scales, int64_t M, const void* w_codes, const void* w_scales,
                              int64_t V, int64_t H, int dtype, void* out, int64_t out_ld, void* stream);

/*
 * A token for each row of logits z. With m the row's largest logit and w_v = exp((z_v - m) / temperature), in the order of falling
 * z, equal ones by rising v:
 *   top_k  keeps the first top_k (0 or at least V: all),
 *   top_p  of these, the ones whose predecessors weigh less than top_p of these together (1 or more: all; the first always),
 *   min_p  of these, the ones with w_v >= min_p (0 or less: all; 1 at most).
 * token = the first kept v for which the sum of kept w up to and with v, by rising v, is above u times the sum of all kept.
 * A temperature that is not above 0 takes the largest logit's first place (above 1e30: as 1e30). A row with a NaN, or nothing above -inf, or whose u is NaN, gives
 * -1; u below 0 counts as 0, from 1 on the last kept token comes. +inf are the largest and equal. Weights are computed in 64 bits and
 * added in integers, so that a result does not depend on the order of additions: a running sum is off by less than a 2^25th of the
 * kept weights together (half of the finest step of u below 1), and the sum that top_p's end is found by likewise.
 *   logits      : device [N,V] of dtype, 1 <= V <= LCE_SAMPLE_MAX_V, N <= LCE_SAMPLE_MAX_N; only read.
 *   uniforms    : device fp32 [N], the random numbers u.
 *   settings    : in HOST memory, read during the call: one value for all rows, or, where the pointer is not NULL, device [N] with
 *                 each row's.
 *   tokens      : device int64 [N].
 *   logprobs    : device fp32 [N], the log of token's share of the kept weights (0 for a temperature not above 0, NaN with token -1);
 *                 NULL where it is not wanted.
 *   workspace   : device memory of lce_sample_workspace_size(N, V) bytes, 256-byte aligned. The size does not fall as N grows. Calls
 *                 (and captured graphs) that may run at the same time need one each.
 */
#define LCE_SAMPLE_MAX_V (1 << 20)
#define LCE_SAMPLE_MAX_N (1 << 16)
typedef struct {
  float temperature, top_p, min_p;
  int32_t top_k;
  const float *temperatures, *top_ps, *min_ps;
  const int32_t* top_ks;
} lce_sample_t;
size_t lce_sample_workspace_size(int64_t N, int64_t V);
lce_status_t lce_sample(const void* logits, int64_t logits_ld, int64_t N, int64_t V, int dtype, const float* uniforms,
                        const lce_sample_t* settings, int64_t* tokens, float* logprobs, void* workspace,
                        size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LCE_VOCAB_H_ */
