/*
 * sift_serve.h - C ABI of libsift around the sparse prefill (sift.h): dense
 * attention of a plan's prompts with transformed scores, and the paged cache
 * that a prefill leaves: attention of new tokens over it, the accumulated
 * attention weights of its keys, and the eviction of those with the least.
 *
 * The conventions of sift.h hold (tensors, layouts, streams, errors, threads).
 */
#ifndef SIFT_SERVE_H_
#define SIFT_SERVE_H_

#include "sift.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Transform of the attention scores, of the calls that take one.  With z =
 * softmax_scale * (q . k), a score is s = cap * tanh(z / cap) (z itself where
 * cap is 0), less slopes[h] * |position of the query - position of the key|
 * where slopes are given.
 *   softmax_scale  <= 0 selects 1/sqrt(D)
 *   cap            0 for none; negative or not finite: SIFT_E_UNSUPPORTED
 *   slopes         device float [Hq], or NULL; positions are exact up to 2^24
 * A NULL score is the default scale alone.
 */
typedef struct sift_score {
  float softmax_scale;
  float cap;
  const float* slopes;
} sift_score;

/* What a row of the dense attention sees of its prompt. */
typedef enum sift_mask {
  SIFT_MASK_CAUSAL = 0,   /* every token up to itself                          */
  SIFT_MASK_DOCUMENT = 1, /* a document's row: its own document up to itself;
                             a query's row: every token up to itself           */
  SIFT_MASK_PREFIX = 2    /* all of the prompt's documents, and every token up
                             to itself                                         */
} sift_mask;

/*
 * Dense attention of the plan's prompts with transformed scores, for the
 * layers of a model that are not sparse, or whose documents are prefilled
 * each by itself: softmax over the visible keys times V, no bit vectors.
 *   q, k, v, out   device tensors as everywhere else, all SIFT_BF16 or all
 *                  SIFT_F32, D 64 or 128 (any tile), 16-byte aligned
 *   mask           a sift_mask
 *   score          see sift_score; positions are the tokens' places in their
 *                  prompt
 *   lse            device float [tokens][Hq], or NULL: receives each row's
 *                  log sum exp of its scores (natural logarithm), as
 *                  sift_cache_accumulate takes it
 * Keys that a row does not see have no influence on it, whatever they hold.
 * The plan's lists are neither read nor changed.  bf16: the weights are
 * rounded to bf16 for their product with V, as in the sparse attention, the
 * sums are fp32.
 * Errors: SIFT_E_NULL, SIFT_E_SHAPE, SIFT_E_UNSUPPORTED (mask, cap, dtypes,
 *   alignment), SIFT_E_PLAN (another device is current), SIFT_E_CAPACITY (2^24
 *   workgroups of 128 rows of a head or more), SIFT_E_HIP.
 */
sift_status sift_plan_dense(sift_plan* plan, const sift_tensor* q, const sift_tensor* k,
                            const sift_tensor* v, int32_t mask, const sift_score* score,
                            sift_tensor* out, float* lse, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SIFT_SERVE_H_ */
