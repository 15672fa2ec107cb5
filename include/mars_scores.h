/*
 * mars_scores.h -- the target model's output side of libmars: the output projection in 8-bit integers, log
 * probabilities of tokens with entropy and best alternatives, and their gradient.
 *
 * Verification (mars.h) decides on the target's logits rows; these calls give what a program reports and
 * trains with beside the decision: softmax probabilities P (Eq. 3 of the paper, at a temperature T) of the
 * emitted tokens, which a server returns with each answer, and the gradient by the logits, which a drafter
 * or a policy that learns from verified rows needs.
 *
 * The conventions of mars.h hold: device pointers owned by the caller, nothing allocated, nothing
 * synchronised, work enqueued on `cuda_stream`; host-detectable errors are returned and nothing is
 * launched then.  A call reads and writes nothing before its predecessor on the stream has completed.
 */
#ifndef MARS_SCORES_H_
#define MARS_SCORES_H_

#include "mars.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MARS_SCORES_MAX_TOKENS 1024 /* cap on J, tokens per row        */
#define MARS_SCORES_MAX_TOP 32      /* cap on k, alternatives per row  */
#define MARS_PROJECT_COUNTER_BYTES 16384 /* counters at the head of mars_project_int8's workspace */

/*
 * Rows as signed 8-bit codes with one scale each: with a = max |x| of a row,
 *   scale = a / 127,  code = rint(x * (127 * (1 / a))),
 * every operation one fp32 IEEE operation, rint to nearest even.  A row whose a is below 2^-119 gets scale 0
 * and zero codes; one that holds a NaN or an infinity gets scale NaN and zero codes, so that whatever is
 * computed from it is NaN.
 *   x        [rows, ldx] of `dt` (MARS_BF16, MARS_FP32, or MARS_FP16 of mars_kv.h), K columns of each row are
 *            read; rows that start on 16-byte boundaries are read in 16-byte steps.
 *   q        int8 [rows, ldq], 16-byte aligned, ldq a multiple of 16; columns 0 .. K-1 are written.
 *   scale    float [rows].      K <= 2^17.
 */
mars_status_t mars_quantize_rows(const void *x, int64_t ldx, int dt, int64_t rows, int K, void *q, int64_t ldq,
                                 float *scale, void *cuda_stream);

/*
 * Output projection (Eq. 2 of the paper: z = W_o h + b_o) in 8-bit integers:
 *   out[m, v] = (sum_k xq[m, k] wq[v, k]) * x_scale[m] * w_scale[v] + bias[v].
 * The sum is exact; the rest is fp32, in that order, the second product and the bias as one fused operation,
 * and the result is rounded to `dt`.  Products run on the tensor cores (tcgen05, kind::i8).
 *   xq       int8 [M, ldx], the tokens' codes (mars_quantize_rows); x_scale float [M].
 *   wq       int8 [V, ldw], the weights' codes, quantised once; w_scale float [V].  Codes are -127 .. 127.
 *   bias     float [V] or NULL.
 *            Both matrices start on 16-byte boundaries, ldx and ldw are multiples of 16; K <= 2^17 is any.
 *   out      `dt` (MARS_BF16 or MARS_FP32) [M, ldo], any alignment; columns 0 .. V-1 are written.
 *   flags    MARS_COUNTERS_ZERO: the caller vouches that the first MARS_PROJECT_COUNTER_BYTES bytes of `workspace`
 *            were zeroed once and it was used by completed calls of this function only since, whatever their
 *            outcome; otherwise the call clears them (one stream operation more).
 *   workspace  mars_project_int8_workspace_bytes() bytes (0 for unsupported sizes; never less for a larger M,
 *            whatever V and K), 256-byte aligned; two calls that may overlap on the GPU need separate ones.
 *   The first call on a device sets function attributes: make it outside any stream capture.
 *   If a bounded device-side wait gives up (a fault in the pipeline, not a property of the data), logits
 *   that were not computed are NaN and the first uint32 of the workspace is MARS_SEQ_TIMEOUT until the next
 *   call; it is 0 otherwise.  The workspace serves further calls all the same.
 */
size_t mars_project_int8_workspace_bytes(int64_t M, int V, int K);
mars_status_t mars_project_int8(const void *xq, int64_t ldx, const float *x_scale, const void *wq, int64_t ldw,
                                const float *w_scale, const float *bias, int64_t M, int V, int K, void *out,
                                int64_t ldo, mars_dtype_t dt, uint32_t flags, void *workspace,
                                size_t workspace_bytes, void *cuda_stream);

/*
 * Log probabilities of tokens.  For every row z of V logits, with p = softmax(z / T):
 *   logprob     float [rows, J]: ln p of tok[r, j]; 0 for an id outside [0, V) (no token there);
 *   entropy     float [rows]: -sum p ln p (terms of probability 0 count 0);
 *   stats       float [rows, 2]: the largest logit m and s = sum exp((z - m) / T), so that
 *               ln p_v = (z_v - m) / T - ln s; mars_token_logprobs_backward reads them;
 *   top_id, top_logprob   int32, float [rows, k]: the k best tokens and their ln p, best first in the order
 *               of mars.h (larger logit first, lower id first among equal ones, NaN counts as -inf); a row
 *               with fewer than k logits above -inf is completed with the lowest unused ids at ln p = -inf.
 * One pass over the row, one kernel; NaN logits count as -inf.  A row whose largest logit is -inf or +inf has no softmax: its
 * logprob (of ids in [0, V)), entropy, s and top_logprob are NaN (m is that logit, top_id is valid).
 *
 *   logits      [n, ld] of `dt`, first V columns of each row are read (16-byte aligned rows are not required).
 *   row_ids     int32 [rows]: output row r is logits row row_ids[r] (any order, repeats allowed; the rows of
 *               accepted paths, say), an id outside [0, n) is an absent row: logprob and entropy 0, stats
 *               (-inf, 0), top_id -1, top_logprob -inf.  NULL: row r itself, rows == n.
 *   temperature T > 0, finite.
 *   tok         int32 [rows, J], 0 <= J <= MARS_SCORES_MAX_TOKENS; NULL with J = 0.
 *   k           0 <= k <= MARS_SCORES_MAX_TOP, k <= V.
 *   entropy, stats may be NULL; logprob is required with J > 0, top_id and top_logprob with k > 0.
 * Sums and exponents are in fp32 relative to the largest logit seen.  Results do not vary from run to run.
 */
mars_status_t mars_token_logprobs(const void *logits, int64_t ld, mars_dtype_t dt, int64_t n,
                                  const int32_t *row_ids, int64_t rows, int V, float temperature,
                                  const int32_t *tok, int J, int k, float *logprob, float *entropy,
                                  float *stats, int32_t *top_id, float *top_logprob, void *cuda_stream);

/*
 * Gradient by the logits of  sum_r ( sum_j grad_logprob[r, j] * logprob[r, j] + grad_entropy[r] * entropy[r] ):
 *   dz_v = (1/T) ( sum_j g_j ([v == tok_j] - p_v) - h p_v (ln p_v + entropy) ).
 * Ids outside [0, V) take no part; a token named twice in a row counts twice.  Rows without a softmax get
 * zeros.  One kernel, each logit read once and each gradient written once, rounded once.
 *   logits, ld, dt, rows, V, temperature, tok, J: as in the forward call (without row_ids), J >= 1.
 *   stats, entropy   of the forward call on these logits (entropy may be NULL if grad_entropy is).
 *   grad_logprob     float [rows, J]; grad_entropy float [rows] or NULL.
 *   grad             [rows, ld_grad] of `dt`, columns 0 .. V-1 are written; may be the logits themselves
 *                    (then ld_grad == ld), may not overlap them otherwise.  Rows of it that lie on 16-byte
 *                    boundaries like the logits' rows are written in 16-byte steps, others an element at a time.
 */
mars_status_t mars_token_logprobs_backward(const void *logits, int64_t ld, mars_dtype_t dt, int64_t rows, int V,
                                           float temperature, const int32_t *tok, int J, const float *stats,
                                           const float *entropy, const float *grad_logprob,
                                           const float *grad_entropy, void *grad, int64_t ld_grad,
                                           void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* MARS_SCORES_H_ */
