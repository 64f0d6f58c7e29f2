/*
 * rtams_logits.h - what rows of logits say: the log probabilities of given tokens, the entropy, and the most likely tokens.
 * What a program that answers over the cache of rtams_cache.h does with a model's output.  Part of librtams.so; the conventions
 * are those of rtams.h (d_* are device pointers, calls enqueue on the stream given and return, the library owns no device memory, every
 * function returns RTAMS_OK or a negative rtams_status, rtams_last_error() describes a failure).  No state is kept between calls.  Memory and
 * stream are those of the thread's current device.
 *
 * Of a row x of `vocab` logits, x' = scale * x:
 *   lse = log sum exp(x'),  log probability of token t = x'_t - lse,  entropy = lse - sum exp(x'_t - lse) x'_t  (natural logarithms)
 * in 32 bits, relative to the row's largest.  A logit of -inf is a token that is not allowed: its probability is 0, its log probability -inf.
 * Of a row in which nothing is above -inf, lse and log probabilities are -inf and the entropy is 0; of a row that holds a NaN or +inf all numbers are NaN.
 * The most likely tokens are in descending order of the logits, of equal ones (0 and -0 are) the lowest first; tokens of -inf are not
 * among them, places left over, and all places of a row of NaN, have token -1 (and -inf, or NaN).
 */
#ifndef RTAMS_LOGITS_H
#define RTAMS_LOGITS_H

#include "rtams_cache.h" /* rtams_type */

#ifdef __cplusplus
extern "C" {
#endif

typedef struct rtams_logits_query {
  int64_t rows;
  int64_t row_stride;      /* elements */
  int32_t vocab;           /* below 2^30 */
  int32_t type;            /* rtams_type */
  int32_t top;             /* most likely tokens asked for, 0..64 */
  int32_t tokens;          /* tokens given for each row */
  float scale;             /* positive, at most 1e30: the inverse of a temperature */
  const void *d_logits;    /* [rows][vocab], logits of a row next to each other */
  const int32_t *d_tokens; /* [rows][tokens]; one outside 0..vocab - 1 has log probability -inf */
  float *d_lse;            /* [rows], or NULL */
  float *d_entropy;        /* [rows], or NULL */
  float *d_logprobs;       /* [rows][tokens] */
  int32_t *d_top;          /* [rows][top] */
  float *d_top_logprobs;   /* [rows][top], or NULL */
  void *d_scratch;         /* device memory, 16-byte aligned, of this call alone until it is done */
  size_t scratch_bytes;
} rtams_logits_query;

/* Scratch that a call needs (it goes by the alignment of d_logits too): 0 where rows are many.  (size_t)-1 on bad arguments. */
size_t rtams_logits_scratch_bytes_for(const rtams_logits_query *q);

int rtams_logits_score(const rtams_logits_query *q, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* RTAMS_LOGITS_H */
