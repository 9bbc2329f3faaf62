/*
 * wisp_logprobs.h -- C ABI of the log probabilities that a server answers beside its tokens.
 *
 * A verification (arxiv 2601.11652, Eq. 1-3) commits L_r accepted drafts and one extra token per request.  Their
 * log probabilities under the target model, the entropy of each position and its most likely alternatives follow from
 * the same logit rows that wisp_verify_accept read.
 *
 * Conventions as in wisp_verify.h: device pointers owned by the caller, asynchronous calls on `stream`, host-visible
 * argument errors returned before anything is enqueued, data errors recorded in the workspace's status word
 * (wisp_verify_get_device_status; the request id is the row's index) with the row skipped.
 */
#ifndef WISP_LOGPROBS_H
#define WISP_LOGPROBS_H

#include "wisp_verify.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * With p = softmax of row i:
 *   logprob[i]        log p(tokens[i])
 *   entropy[i]        -sum p log p, in nats
 *   top_tokens[i]     the top_n most likely tokens, by falling logit, the lower id first among equal ones
 *   top_logprobs[i]   their log probabilities
 * A logit of -inf has probability 0, counts 0 in the entropy and is listed last (log probability -inf); where
 * top_n > V the entries past V are -1 and -inf.
 * A row whose token is negative is skipped: logprob, entropy and top_logprobs 0, top_tokens -1.  A row whose token is
 * V or more (WISP_DEV_BAD_TOKEN), or that has no softmax (a NaN or +inf, or -inf throughout; WISP_DEV_BAD_PROB), gets NaN
 * and -1.
 * Sums are in fp32.
 */
typedef struct {
  int32_t rows, V;
  int64_t row_stride;        /* elements between rows of logits, at least V; 0: V */
  wisp_dtype logits_dtype;   /* F32 or BF16 */
  const void *logits;        /* [rows, V] */
  const int32_t *tokens;     /* [rows] */
  int32_t top_n;             /* 0 to 32 */
  float *logprob;            /* [rows] out */
  float *entropy;            /* [rows] out; may be NULL */
  int32_t *top_tokens;       /* [rows, top_n] out; may be NULL if top_n is 0 */
  float *top_logprobs;       /* [rows, top_n] out; may be NULL if top_n is 0 */
} wisp_logprobs_args;

/* Bytes of workspace; 0 if the arguments are invalid. */
size_t wisp_verify_logprobs_workspace_size(const wisp_logprobs_args *a);

wisp_status wisp_verify_logprobs(const wisp_logprobs_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* The token that each logit row of a verified batch committed, as wisp_verify_logprobs takes them: row Q0_r + i
 * gets draft token i + 1 for i < L_r, next_token[r] for i = L_r, and -1 past that.  Rows of a request with L_r outside
 * [0, k_r] (one that the acceptance pass refused) and rows that belong to no request get -1.
 * row_tokens [total_q_rows] out.  Read of `acc`: B, total_q_rows, total_draft, draft_lens, draft_tokens, accepted_len,
 * next_token.  Enqueued after the acceptance pass on its stream; no workspace. */
wisp_status wisp_verify_committed_tokens(const wisp_accept_args *acc, int32_t *row_tokens, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* WISP_LOGPROBS_H */
