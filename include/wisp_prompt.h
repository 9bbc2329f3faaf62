/*
 * wisp_prompt.h -- C ABI of the attention of whole prompts, and of batches whose requests begin with the same pages.
 *
 * A session's cached prefix (arxiv 2601.11652, Sec. 4.4-4.5) is computed once, when its prompt is prefilled, and sessions
 * behind the same system prompt may hold the same pages of it in their block tables.  wisp_prompt_attention is the attention of
 * the prefill, behind wisp_kv_reserve_append (or its form with rotation); wisp_verify_attention_shared is the attention of a
 * verification over such sessions, which reads the shared pages once for a whole run of requests.
 *
 * Conventions and data layout as in wisp_verify.h: device pointers owned by the caller, asynchronous calls on `stream`,
 * host-visible argument errors returned before anything is enqueued, data errors recorded in the workspace's status word
 * (wisp_verify_get_device_status) with the request skipped.  Calls that share a workspace must not overlap in time.  A call is three
 * launches and may be captured into a graph (make a device's first call before).  Outputs repeat to the bit.
 */
#ifndef WISP_PROMPT_H
#define WISP_PROMPT_H

#include "wisp_kv8.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * wisp_attn_args without its limit on query rows: request r's k_r + 1 query rows (draft_lens[r] = k_r >= 0) are a prompt, or the
 * chunk of one behind c_r cached tokens; row j sees keys 0 .. c_r + j of its sequence, which must all be in the pool already.
 *   out[row, h] = sum_t softmax_t(<q[row, h], K[t, h / (Hq/Hkv)]> / sqrt(D)) V[t, h / (Hq/Hkv)]
 * The cache has the queries' type, or holds e4m3 codes with a scale per page and KV head (wisp_kv8.h).
 * Supported: D in {64, 128}, block_size == 16, Hq / Hkv <= 128, k_r < 2^24, and total_q_rows * Hq * (D + 2) < 2^29 with shared pages (partial
 * results have 32-bit offsets: larger calls may return WISP_ERR_UNSUPPORTED).
 * Scores, softmax statistics and outputs accumulate in fp32, and finite inputs whose scores fp32 holds give finite outputs (a weight below 2^-110 of
 * the sum of its row's counts as zero).  With bf16 queries a weight enters the second product in bf16
 * (relative error 2^-9), and so do code * scale of an e4m3 cache, K and V (exactly where the scale is a power of two of magnitude 2^-100
 * to 2^100; values past the bf16 range count as its largest).  With fp32 queries every factor enters its product with
 * 22 significant bits or more: queries, and K and V of an fp32 cache, down to steps of 2^-38 of the largest value of their row; a weight times its
 * key's largest |V| (its V scale) down to steps of 2^-36 of the row's largest weight times the largest such value that the row sees among 64
 * consecutive keys.
 * A key that a row does not see adds nothing to it, whatever its K and V hold (NaN and infinities too; slots past a request's
 * tokens may hold anything).  A NaN that a row does see, or a row whose scores are all -inf, makes that row NaN (of V: in its element).
 */
typedef struct {
  wisp_attn_args attn;
  wisp_dtype cache_dtype;          /* attn.qkv_dtype, or WISP_E4M3 */
  const float *k_scale, *v_scale;  /* [num_blocks, Hkv] with WISP_E4M3: finite, not negative; else not used */
} wisp_prompt_args;

/* Bytes of workspace (on the current device); 0 if the arguments are invalid. */
size_t wisp_prompt_workspace_size(const wisp_prompt_args *a);

wisp_status wisp_prompt_attention(const wisp_prompt_args *a, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The same for a batch whose requests share the first pages of their sequences.  Consecutive requests with the same
 * shared_ids[r] >= 0 and the same shared_pages[r] > 0 are a run; the first shared_pages[r] pages of all its requests are those that
 * the block table of the run's first request that is not refused names (the others' entries for them are not read).  The run's rows
 * attend to them together, each request's rows to its own keys behind them, and the two are joined by their log-sum-exp.  Requests with a negative id or no
 * shared pages, and runs of one request, are computed alone.
 * shared_pages[r] * block_size must be at most c_r: such a request is flagged WISP_DEV_BAD_LENGTH.
 */
typedef struct {
  wisp_prompt_args rows;
  const int32_t *shared_ids;    /* [B] */
  const int32_t *shared_pages;  /* [B] */
} wisp_shared_args;

size_t wisp_verify_shared_workspace_size(const wisp_shared_args *a);

wisp_status wisp_verify_attention_shared(const wisp_shared_args *a, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* WISP_PROMPT_H */
