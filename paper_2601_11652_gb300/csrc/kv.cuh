// kv.cuh -- parameters, workspace and host helpers shared by the paged KV calls.
#pragma once

#include "common.cuh"
#include "wisp_kv.h"

namespace wisp {

constexpr int kKvPage = 16;

struct KvParams {
  int B, Hkv, D, max_blocks, num_blocks, total_rows, esize;
  int64_t max_tokens;  // longest sequence a request may reach: its table's, or that of the rotation's table
  const int64_t *request_ids;
  const int32_t *draft_lens;
  int32_t *context_lens, *block_tables, *free_blocks, *free_count;
  char *k_cache, *v_cache;
  const char *k_new, *v_new;
  const int32_t *accepted_len;
  DeviceStatus *status;
  int32_t *row_req, *row_pos;  // [total_rows]: request of a new row (-1: skipped) and its position
  int32_t *need, *first;       // [B]: a request's missing pages (-code: refused), its first missing table entry
};

struct KvLayout {
  size_t status = 0, row_req = 0, row_pos = 0, need = 0, first = 0, total = 0;
};

KvLayout kv_layout(const wisp_kv_args *a);
// need_new: k_cache, v_cache, k_new and v_new are given and aligned; need_accepted: accepted_len is given
wisp_status kv_check(const wisp_kv_args *a, bool need_new, bool need_accepted);
KvParams kv_params(const wisp_kv_args *a, void *ws, const KvLayout &L);
wisp_status kv_ws_ok(void *ws, size_t bytes, const KvLayout &L);
// The reservation: pages for tokens 0 .. c + k of every request, the new rows' requests and positions in
// row_req and row_pos.  Lets its programmatic dependent start at once.
cudaError_t kv_reserve_launch(const KvParams &p, cudaStream_t s);
// The commit of a checked batch, up to p.max_tokens.
wisp_status kv_commit_launch(const KvParams &p, cudaStream_t s);

inline bool al16(const void *p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace wisp
