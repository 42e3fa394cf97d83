/*
 * viscache_step.h -- the rest of a decode step around the 8-bit paged cache
 * (viscache.h): query and key heads normed and rotated in one pass, with the
 * gradient; the attention each token receives added up, and the cache held to
 * a budget by it; the next token drawn from the logits.
 *
 * The conventions are those of viscache.h: int status codes, caller-owned
 * buffers, work queued on the caller's stream, 16-byte aligned rows, no device
 * memory allocated, nothing printed, no C++ exception.
 */
#ifndef VISCACHE_STEP_H_
#define VISCACHE_STEP_H_

#include "viscache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * viscache_norm_mrope -- query and key heads normed (root mean square over the
 * head's d values, a weight a channel) and rotated as viscache_mrope does, in
 * the same pass:
 *     r = 1 / sqrt(sum_c x_c^2 / d + eps),   y = R(positions) (x r w).
 * Each head is normed by itself; w is q_weight for query heads, k_weight for
 * key heads.  Sums, products and the rotation in fp32, one rounding to the
 * type.  A head whose squares pass fp32's range is summed again scaled, so that
 * finite rows of any size give what the formula says; a head with a value that
 * is not finite gives NaN in that value's place at least.
 *   rope, positions, q, k, q_out, k_out, strides   as in viscache_mrope (an
 *             output may be its input, same pointer and stride)
 *   q_weight, k_weight   device [d] of `dtype`
 *   eps       1e-20 .. 1
 * Hq or Hkv may be 0 (its pointers may then be NULL).  n_rows = 0 does nothing.
 * Errors: VC_ERR_INVALID_ARG, VC_ERR_CUDA.
 */
int viscache_norm_mrope(const vc_rope* rope, const int32_t* positions, int dtype, int64_t n_rows, int32_t Hq,
                        int32_t Hkv, int32_t d, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        const void* q_weight, const void* k_weight, float eps, void* q_out, int64_t q_out_stride,
                        void* k_out, int64_t k_out_stride, void* stream);

/*
 * viscache_norm_mrope_grad -- its gradient.  With dy the gradient of a head's
 * output, x its input, n = x r, g = R(positions)^T dy and h = g w:
 *     dx = r (h - n sum_c(h n) / d),      dw = sum over rows and heads of g n.
 *   q, k                    the forward call's inputs
 *   q_out_grad, k_out_grad  gradients of its outputs, rows with their own strides
 *   q_grad, k_grad          gradients of its inputs; may be the forward's input or
 *             the output's gradient (same pointer and stride), and may not overlap
 *             them otherwise
 *   q_weight_grad, k_weight_grad  device fp32 [d], 16-byte aligned: written, not
 *             added to (n_rows = 0 writes zeros).  The order of the sums depends on
 *             the sizes alone: the same call gives the same bits.
 * Workspace: viscache_norm_mrope_grad_workspace_size(n_rows, Hq, Hkv, d) bytes
 * (0 for arguments that the call refuses), 256-byte aligned.
 * Errors: VC_ERR_INVALID_ARG, VC_ERR_WORKSPACE, VC_ERR_CUDA.
 */
size_t viscache_norm_mrope_grad_workspace_size(int64_t n_rows, int32_t Hq, int32_t Hkv, int32_t d);
int viscache_norm_mrope_grad(const vc_rope* rope, const int32_t* positions, int dtype, int64_t n_rows, int32_t Hq,
                             int32_t Hkv, int32_t d, const void* q, int64_t q_stride, const void* k,
                             int64_t k_stride, const void* q_out_grad, int64_t q_out_grad_stride,
                             const void* k_out_grad, int64_t k_out_grad_stride, const void* q_weight,
                             const void* k_weight, float eps, void* q_grad, int64_t q_grad_stride, void* k_grad,
                             int64_t k_grad_stride, float* q_weight_grad, float* k_weight_grad, void* ws,
                             size_t ws_bytes, void* stream);

/*
 * viscache_kv8_weigh -- what attention each cached token gets from the step's
 * query rows, added up for each KV head:
 *     A[t][g] = sum over the rows i that see t and the query heads j of group g
 *               of exp(scale * q[i][j] . K_hat[t][g] - lse[i][j]),
 *     weights[t][g] <- A[t][g] + (weights[t][g] if t < seq_lens - m else 0),
 * m the request's rows: the step's own tokens start from A.  Rows, `causal` and
 * `scale` mean what they mean in viscache_kv8_attention, whose `lse` this call
 * reads; it is called after the rows have been appended and attended.
 *   lse       device fp32 [n_rows][Hq].  A row whose lse is -inf (one that sees
 *             no token) adds nothing; a row that is no token (more rows than
 *             tokens) adds nothing whatever its queries and its lse hold
 *   weights   device fp32 [n_pages][Hkv][page], a number for every slot of the
 *             pool; 16-byte aligned.  Slots past seq_lens are left as they were.
 * The pages of a call's requests must be different ones (a page of two requests
 * would be written by both): requests that share a prefix's pages are weighed
 * in calls of their own.
 * Rows enter the products as in viscache_kv8_attention (fp32 rows as two fp16
 * numbers); bf16 rows of calls of many rows (more than 64 of a KV head per request on
 * average) as they are, so that their values' products with codes have to stay below
 * 2^127 there, and count as 0 below 2^-126.  Scores as there below 2^22.  Sums in fp32
 * in an order that the call's sizes, lengths and the device's SMs decide: the same
 * call gives the same bits.  A key that is not finite makes its token's weight NaN; the
 * attention's lse of a row that sees it is NaN, and a row with such an lse makes the
 * weights of all tokens that it sees NaN, which they then stay.
 * After VC_ERR_DEVICE_TIMEOUT (prunekv_get_status) clear the workspace before a
 * captured call is replayed with it.
 * Workspace: viscache_kv8_workspace_size(n_rows, Hq, Hkv, d), as for the
 * attention; device checks and prunekv_get_status too.
 * Errors: VC_ERR_INVALID_ARG, VC_ERR_WORKSPACE, VC_ERR_CUDA, and
 * VC_ERR_UNSUPPORTED where the rows times max_pages are past 2^37 tiles.
 */
int viscache_kv8_weigh(const vc_kv8* cache, const vc_kv8_step* step, int dtype, int32_t Hq, const void* q,
                       int64_t q_stride, const float* lse, float scale, int causal, float* weights, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * viscache_kv8_evict -- hold requests to a budget: of each request and KV head
 * the keep[r] tokens with the largest weights stay, in their order, and move
 * together; the others are gone.  A request of no more than keep[r] tokens is
 * left as it is.
 *   weights   as in viscache_kv8_weigh; moved with their tokens
 *   keep      device int32 [n_req], 0 .. max_keep
 *   sink, recent   the first `sink` and the last `recent` tokens of a request
 *             count as heavier than any weight but +inf; among equal weights the
 *             lower token stays; NaN counts as less than any number
 *   kept      device int32 [n_req][Hkv][max_keep]: the tokens that stayed, by
 *             their old places, ascending; entries past the new length are left as
 *             they were
 *   new_lens  device int32 [n_req]: min(seq_lens, keep).  May be step->seq_lens
 *             itself; else seq_lens is left as it was, and the caller goes on with
 *             new_lens
 * Each page from the one with the first gap on holds what viscache_kv8_append
 * would write into it from the values x_hat that stayed: scales are taken anew,
 * codes are re-encoded where the scale changed (exact but for values that fall
 * below e4m3's smallest normal number under a larger scale).  Slots past the new
 * length, and pages past it, hold what they held.  Of the step only n_req, the
 * block table and seq_lens count.  The pages of the call's requests must be
 * different ones.
 * Workspace: viscache_kv8_evict_workspace_size(n_req, Hkv) bytes (0 for arguments
 * that the call refuses), 256-byte aligned; prunekv_get_status(ws) reports device
 * checks: a length or a page out of range (VC_ERR_DEVICE_INDEX), keep outside
 * [0, max_keep].  They are clamped; a request with a page out of range is left
 * as it was, with new_lens its (clamped) length and no `kept`.
 * Errors: VC_ERR_INVALID_ARG, VC_ERR_WORKSPACE, VC_ERR_CUDA.
 */
size_t viscache_kv8_evict_workspace_size(int32_t n_req, int32_t Hkv);
int viscache_kv8_evict(const vc_kv8* cache, const vc_kv8_step* step, float* weights, const int32_t* keep,
                       int32_t max_keep, int32_t sink, int32_t recent, int32_t* kept, int32_t* new_lens, void* ws,
                       size_t ws_bytes, void* stream);

/*
 * viscache_sample -- the next token of each row of logits, from a given random
 * number.  With x the row, M its maximum, T its temperature:
 *     w_i = exp((x_i - M) / T);   order: by logit descending, ties by index;
 *     kept: the first min(top_k, n_p, n_m) tokens of the order, at least one,
 *       n_p  the least n whose first n weights reach top_p times the weights of
 *            the first top_k,
 *       n_m  the number of tokens with w_i >= min_p;
 *     token = the least i with  sum_{kept j <= i} w_j > u * sum_kept w,
 *     logprob = log(w_token / sum_kept w).
 * T <= 0 (or NaN) is greedy (a positive T below 2^-127 counts as 2^-127): the first of the largest logits, logprob 0.  top_k <= 0,
 * top_p >= 1 and min_p <= 0 (or NaN) keep everything, and so does a NULL array;
 * top_p <= 0 and min_p >= 1 keep the first, min_p >= 1 all that tie with it.
 * u below 0 (or NaN) counts as 0, of 1 and more as the last kept token with a weight.
 *   logits    device rows of `dtype`, row r at element r * stride; any stride of at
 *             least vocab and any alignment of the type
 *   u, temperature   device fp32 [n_rows]; top_k int32, top_p, min_p fp32 [n_rows]
 *   token     device int32 [n_rows];  logprob device fp32 [n_rows] (nullable)
 * A logit of -inf or NaN has weight 0; of +inf, weight 1 and all others 0.  A row with
 * nothing above -inf gives token -1 and logprob NaN.
 * Weights are whole numbers of 2^-44 (2^-45 at 131072 tokens and fewer, 2^-47 at 32768)
 * from an exponential of about 38 bits: sums are exact and do not depend on their order,
 * and a token differs from the formula's only where u, top_p or min_p lie within about
 * 2^-36 of a border.  vocab 1 .. 262144; n_rows 0 .. 65535.  No workspace.
 * Errors: VC_ERR_INVALID_ARG, VC_ERR_CUDA.
 */
int viscache_sample(int dtype, int64_t n_rows, int64_t vocab, const void* logits, int64_t stride, const float* u,
                    const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                    int32_t* token, float* logprob, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* VISCACHE_STEP_H_ */
