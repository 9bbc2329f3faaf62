/*
 * wisp_kv8.h -- C ABI of the projection-side append (position rotation applied on the way) and of KV caches in 8 bits.
 *
 * The verification forward (arxiv 2601.11652, Sec. 4.5) attends a block of new tokens over the cached prefix.  Its
 * queries and keys carry a rotation by their absolute position; wisp_kv_reserve_append_rope applies it while it
 * writes the new rows of the QKV projection into the paged cache (wisp_kv.h), so that neither is stored in between.
 *
 * 8-bit caches.  k_cache and v_cache [num_blocks, Hkv, 16, D] hold e4m3 codes (no infinities, largest magnitude 448,
 * NaN 0x7f and 0xff), k_scale and v_scale [num_blocks, Hkv] one fp32 scale per page and KV head; an element is worth
 * code * scale.  The append writes scales 2^e: the least e (from -96 to 120) such that the page's largest finite live
 * magnitude is at most 448 * 2^e (1 where all are zero).  Live are the page's tokens before the new ones and the new
 * ones themselves: a page filled over several calls is decoded and, where its scale changes, encoded again.  Values
 * are rounded to the nearest code (ties to even), infinities become the largest code, NaN stays NaN.
 *
 * Conventions as in wisp_verify.h and wisp_kv.h: device pointers owned by the caller, asynchronous calls on `stream`,
 * host-visible argument errors returned before anything is enqueued, data errors recorded in the workspace's status
 * word (wisp_verify_get_device_status) with the request skipped.
 */
#ifndef WISP_KV8_H
#define WISP_KV8_H

#include "wisp_kv.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The rotation.  Row j of request r is at position t = c_r + j.  With half = rot_dim / 2 and the table's row t
 * (half cosines, then half sines), pair i (elements i and half + i, or 2i and 2i + 1 if interleaved) of a query or key
 * head becomes (a cos_i - b sin_i, b cos_i + a sin_i), products and sums rounded to fp32 one by one; elements from
 * rot_dim on and values pass unchanged.  Results are rounded once to their type.
 */
typedef struct {
  wisp_kv_args kv;           /* as for wisp_kv_reserve_append; kv_dtype is the type of q, k_new, v_new and q_out.  Caches
                                hold cache_dtype */
  wisp_dtype cache_dtype;    /* kv.kv_dtype, or WISP_E4M3 */
  float *k_scale, *v_scale;  /* [num_blocks, Hkv]; read and written with WISP_E4M3, else not used */
  const float *rope;         /* [rope_positions, rot_dim] cosines and sines; may be NULL if rot_dim is 0 */
  int32_t rope_positions;    /* a request with c_r + k_r + 1 > rope_positions is flagged WISP_DEV_BAD_LENGTH */
  int32_t rot_dim;           /* rotated elements of a head: a multiple of 16, 0 (none) to D */
  int32_t interleaved;       /* 0: pairs (i, half + i); else pairs (2i, 2i + 1) */
  int32_t Hq;                /* query heads; 0: no queries */
  const void *q;             /* [total_q_rows, Hq, D] */
  void *q_out;               /* [total_q_rows, Hq, D] packed; q itself where q is packed, or apart from it */
  int64_t q_stride, k_stride, v_stride;  /* elements between rows of q, k_new and v_new (they may be parts of one
                                            projection output); 0: packed.  A multiple of 16 bytes each */
} wisp_kv_rope_args;

/* Bytes of workspace; 0 if the arguments are invalid. */
size_t wisp_kv_rope_workspace_size(const wisp_kv_rope_args *a);

/* wisp_kv_reserve_append (pages for tokens 0 .. c_r + k_r, new K/V rows at c_r + j) with the rotation applied to K on
 * the way, and the rotated queries in q_out.  A request that is refused (for its length, its table or for want of pages) is
 * left alone altogether: its rows of q_out stay as they are, so that queries rotated in place may be sent again.
 * wisp_kv_commit_rope follows a step. */
wisp_status wisp_kv_reserve_append_rope(const wisp_kv_rope_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* wisp_kv_commit with the append's limit on lengths: a request with c_r + k_r + 1 > rope_positions, whose rows the append refused,
 * is flagged WISP_DEV_BAD_LENGTH and left unchanged.  (wisp_kv_commit knows the block table's length only, and would move such a
 * request's prefix over tokens that were never stored, where its pages exist already.)  Reads what wisp_kv_commit reads of `kv`,
 * rot_dim and rope_positions; the workspace is wisp_kv_rope_workspace_size's. */
wisp_status wisp_kv_commit_rope(const wisp_kv_rope_args *a, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Attention over an 8-bit cache: wisp_attn_args with k_cache and v_cache e4m3 codes; qkv_dtype is the type of q and out.
 * Workspace: wisp_verify_workspace_size(&a->attn, acc).
 *   out[row, h] = sum_t softmax_t(<q[row, h], K[t]> / sqrt(D)) V[t], K[t] = k_code * k_scale, V[t] = v_code * v_scale
 * Scales are finite and not negative (those that the append writes are; others may be any such fp32 value).  Codes past a
 * request's tokens are not judged: pages may hold anything there.  Accumulation is fp32.  With bf16 queries, V scales from 2^-60
 * to 2^40, and 0, take the tensor cores; a work item that meets others is computed in fp32 on the CUDA cores, many times as slowly.
 * Otherwise an element of a query, and a weight times its page's V scale, enter the products with 8 significant bits (a bf16
 * value's own) where they are large, and smaller ones in steps: an element is off by at most 2^-17 of the largest one among the queries
 * that share a work item, a key's weight * V scale by 2^-15 of the largest such product among 128 consecutive keys.  A product below
 * 2^-30 of the row's largest one may count as nothing.  (So a page whose V scale is far above another's also sets the steps of
 * the elements in which it holds zeros.)  A query that is not finite makes its own row of its head NaN, a value that is NaN the
 * rows that see it in its element.
 */
typedef struct {
  wisp_attn_args attn;
  const float *k_scale, *v_scale;  /* [num_blocks, Hkv] */
} wisp_attn_kv8_args;

wisp_status wisp_verify_attention_kv8(const wisp_attn_kv8_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* wisp_verify_step over an 8-bit cache: attention and acceptance in one call. */
wisp_status wisp_verify_step_kv8(const wisp_attn_kv8_args *a, const wisp_accept_args *acc, void *workspace,
                                 size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* WISP_KV8_H */
