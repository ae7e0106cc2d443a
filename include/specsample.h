/*
 * specsample.h -- C ABI of sampling: a token of each row of logits by
 * temperature, top-k, top-p and min-p from a given uniform, and the distribution
 * that it was drawn from.
 *
 * A drafting step needs both: the tokens are spec_accept's draft_tokens and the
 * probability rows its draft_probs (specverify.h, the test of Eq. (1) of arXiv
 * 2505.17074 compares them with the target's).  With SPEC_SAMPLE_LOGITS a target's
 * rows become the logits of its own truncated distribution, spec_accept's
 * target_logits.  A row without drafts gets its token here.
 *
 * Conventions: those of specverify.h for streams, errors and argument checks.
 */
#ifndef SPECSAMPLE_H
#define SPECSAMPLE_H

#include "specverify.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum spec_sample_rows {
  SPEC_SAMPLE_NONE = 0,
  SPEC_SAMPLE_PROBS = 1,
  SPEC_SAMPLE_LOGITS = 2
} spec_sample_rows_t;

/*
 * One row's tokens in the order of their logits, the largest first and the
 * lower id first among equals, have the weights w = exp((l - l_max) / T).  What
 * stays is the shortest of
 *   top-k   the first top_k of the order;
 *   top-p   the shortest run from the front whose weight is at least top_p times
 *           that of the tokens that top-k leaves;
 *   min-p   the tokens with w >= min_p;
 * the first token in any case.  The sampled one is the smallest id whose
 * cumulative weight, over ids ascending among what stays, exceeds u times the
 * total (spec_accept's convention).
 *
 *   num_rows, vocab   >= 1; rows below 2^22, tokens up to 2^28
 *                     (SPEC_ERR_UNSUPPORTED otherwise).
 *   dtype             of the logits: SPEC_F32 or SPEC_BF16.
 *   logits            [num_rows, vocab] (device), row stride logits_stride
 *                     elements (>= vocab), aligned to their elements.  Minus
 *                     infinity is a token that is masked out, NaN the same; of
 *                     plus infinities each has weight 1 and all else none.
 *   temperature       fp32 [num_rows] (device) or NULL: 1.  Not above zero (or
 *                     NaN): the first token alone.
 *   top_k             int32 [num_rows] or NULL; below one: no limit.
 *   top_p             fp32 [num_rows] or NULL; one and above: no limit, not above
 *                     zero (or NaN): the first token alone.
 *   min_p             fp32 [num_rows] or NULL; zero and below: no limit, above
 *                     one (or NaN): the first token alone.
 *   uniforms          fp32 [num_rows] in [0, 1).  May be NULL without tokens.
 *   tokens            int32 [num_rows] out, or NULL.  -1 where a row has no token
 *                     that is not masked out.
 *   rows, rows_stride, rows_kind
 *                     [num_rows, vocab] out in the logits' dtype, row stride
 *                     rows_stride (>= vocab); the logits themselves (in place) or
 *                     no memory that the call reads.  SPEC_SAMPLE_PROBS: the
 *                     tokens' probabilities, zero for those that do not stay;
 *                     SPEC_SAMPLE_LOGITS: l / T (one token alone: 0), the type's
 *                     lowest value for those that do not stay; SPEC_SAMPLE_NONE:
 *                     not written (rows may be NULL).  A row without tokens has
 *                     zero probabilities, or all logits at the lowest value.
 * Weights are taken in 64 bits, off by 1e-11 of their value at most, and summed in
 * 64 bits, top-p's in fixed point: n weights to n^2 2^-61 of the largest (7e-9 for
 * 128256 of them) at the worst.  Tokens and the sets that stay are those of the
 * definition unless a sum is that near to its border.  Results are deterministic.
 * A row costs two reads of its logits and of some of them a third.  These rows are
 * searched by one work-group alone instead, 0.06-0.45 ms for 32000-128256 tokens
 * where others take 0.01-0.06:
 *   top-k from 1025 on with a top-p below one, whatever the logits, and from 513 on
 *     with one where no more than top_k tokens are not masked out;
 *   top-k whose last token has others within 1/32 of its logit (whatever T), equal
 *     ones among them, so that they, and for a top_k of up to 1024 all tokens before
 *     them, are more than 2048; or whose last token is more than 62 below the
 *     largest logit;
 *   a top_k of up to 512 where the large logits, or all that a mask leaves, have
 *     neighbouring ids: its last token is looked for among the largest of each of
 *     1024 threads, which read 16 bytes of a row in turn, and then more than 2048
 *     tokens may be above what they have (3000 neighbours in bf16 are 375 threads',
 *     for a top_k of 400);
 *   top-p alone with its cut among more than 2048 tokens within T / 64 of each
 *     other's logits (logits that are nearly all the same), or so near one that
 *     tokens below e^-31 of the largest weight make it up (rows of millions);
 *   a largest logit of 2^18 and above in magnitude with top-k, of 2^17 T with top-p
 *     alone (T very small, or infinite).
 */
typedef struct spec_sample_args {
  int32_t num_rows;
  int32_t vocab;
  spec_dtype_t dtype;
  int32_t rows_kind;
  const void* logits;
  int64_t logits_stride;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  const float* uniforms;
  int32_t* tokens;
  void* rows;
  int64_t rows_stride;
} spec_sample_args_t;

/* Device workspace of a call (256-byte aligned; it needs no initialisation and may hold
 * anything between calls). */
SPEC_API spec_status_t spec_sample_workspace_bytes(const spec_sample_args_t* args, size_t* device_bytes);

SPEC_API spec_status_t spec_sample(const spec_sample_args_t* args, void* workspace, size_t workspace_bytes,
                                   void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SPECSAMPLE_H */
