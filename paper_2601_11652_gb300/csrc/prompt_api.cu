// prompt_api.cu -- host side of include/wisp_prompt.h: argument checks, workspace and launches.  No allocation, no
// synchronisation.
#include <algorithm>
#include <cstring>
#include <mutex>

#include "prompt.cuh"
#include "wisp_prompt.h"

using namespace wisp;

namespace {

constexpr int kMaxDevices = 64;
int g_sms[kMaxDevices];  // SMs of a device that has been set up
std::mutex g_mu;

wisp_status setup(int *sms) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return WISP_ERR_CUDA;
  std::lock_guard<std::mutex> lk(g_mu);
  if (!g_sms[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return WISP_ERR_CUDA;
    if (prompt_f32_setup() != cudaSuccess || prompt_tc_setup() != cudaSuccess || prompt_plan_setup() != cudaSuccess) return WISP_ERR_CUDA;
    g_sms[dev] = n;
  }
  *sms = g_sms[dev];
  return WISP_OK;
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

wisp_status check(const wisp_prompt_args *x) {
  if (!x) return WISP_ERR_INVALID_ARG;
  const wisp_attn_args *a = &x->attn;
  if (a->B < 0 || a->Hq <= 0 || a->Hkv <= 0 || a->Hq % a->Hkv != 0) return WISP_ERR_INVALID_ARG;
  if (a->qkv_dtype != WISP_F32 && a->qkv_dtype != WISP_BF16) return WISP_ERR_INVALID_ARG;
  if (x->cache_dtype != a->qkv_dtype && x->cache_dtype != WISP_E4M3) return WISP_ERR_INVALID_ARG;
  if (a->D != 64 && a->D != 128) return WISP_ERR_UNSUPPORTED;
  if (a->block_size != 16 || a->Hq / a->Hkv > 128) return WISP_ERR_UNSUPPORTED;
  if (a->B == 0) return WISP_OK;
  if (a->max_blocks_per_seq <= 0 || a->num_blocks <= 0 || a->total_q_rows < a->B) return WISP_ERR_INVALID_ARG;
  if (!a->draft_lens || !a->context_lens || !a->block_tables || !a->q || !a->k_cache || !a->v_cache || !a->out)
    return WISP_ERR_INVALID_ARG;
  if (!aligned16(a->q) || !aligned16(a->k_cache) || !aligned16(a->v_cache) || !aligned16(a->out)) return WISP_ERR_INVALID_ARG;
  if (x->cache_dtype == WISP_E4M3 && (!x->k_scale || !x->v_scale)) return WISP_ERR_INVALID_ARG;
  if ((int64_t)a->max_blocks_per_seq * a->block_size > INT32_MAX / 2) return WISP_ERR_UNSUPPORTED;
  if ((int64_t)a->total_q_rows * (a->Hq / a->Hkv) > INT32_MAX / 2) return WISP_ERR_UNSUPPORTED;
  return WISP_OK;
}

wisp_status check(const wisp_shared_args *x) {
  const wisp_status st = check(x ? &x->rows : nullptr);
  if (st != WISP_OK || x->rows.attn.B == 0) return st;
  return x->shared_ids && x->shared_pages ? WISP_OK : WISP_ERR_INVALID_ARG;
}

struct Space {
  size_t status, header, q_row_start, req_flag, req_run, run_info, segs, items, handed_on, partials, total;
  int64_t max_rows, partial_cap;
  int unit_rows;
  bool fits;
};

// Rows of a unit, and bounds on list entries and partials.  Without cuts a request has ceil(rows / unit_rows) units, a run as many for its
// rows again, and both leave one partial per row and head.  Cuts add entries and partials of whole units: by the planner's rule a few
// items per SM, and no unit has more chunks than its keys (at most a table's) are cut into with the shortest ones; where they would not fit (a causal
// prompt's last units are twice as long as the average), it makes none.
Space space(const wisp_attn_args *a, bool shared, int sms) {
  Space s;
  const int g = a->Hq / a->Hkv;
  const int64_t T = a->B > 0 ? a->total_q_rows : 0;
  s.unit_rows = (a->qkv_dtype == WISP_BF16 ? 2 : 1) * g * prompt_tile_positions(g);
  const int64_t units = (T * g / s.unit_rows + a->B) * (shared ? 2 : 1);
  const int64_t tokens = (int64_t)a->max_blocks_per_seq * a->block_size;
  // chunks of a unit, at most: its first one may end anywhere
  auto chunks = [&](int shortest) -> int64_t { return tokens <= kChunkTile ? 1 : 2 + (tokens - kChunkTile - 1) / shortest; };
  auto slot = [&](int rows) { return std::min<int64_t>(rows, T * g) * (a->D + 2) + 4; };
  auto partials = [&](int shortest, int rows) { return chunks(shortest) > 1 ? chunks(shortest) * slot(rows) : 0; };
  const int64_t cuts = (std::min<int64_t>(2 * units * a->Hkv, (int64_t)12 * sms) + 4 * sms) / a->Hkv + 8;
  // (units of two tiles, with bf16 queries: a segment of one tile of rows is one unit, and there are as many segments as requests and runs)
  const int64_t small = partials(kLeastChunk, std::min(s.unit_rows, kChunkTile)), full = partials(kLeastFullChunk, s.unit_rows);
  const int64_t possible = s.unit_rows <= kChunkTile ? units * small : std::min(units * std::max(small, full), units * full + a->B * (shared ? 2 : 1) * small);
  s.max_rows = units + std::min(cuts, units * (chunks(kLeastChunk) - 1));
  s.partial_cap = std::min(cuts * slot(s.unit_rows), possible) * a->Hkv + (shared ? 2 * T * a->Hq * (a->D + 2) + 4 * units * a->Hkv : 0);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off = (off + bytes + 255) & ~(size_t)255;
    return at;
  };
  const size_t B = (size_t)a->B;
  s.status = take(sizeof(DeviceStatus));
  s.header = take(sizeof(PromptHeader));
  s.q_row_start = take(4 * (B + 1));
  s.req_flag = take(4 * B);
  s.req_run = take(4 * B);
  s.run_info = take(16 * B);
  s.segs = take(sizeof(Segment) * 2 * B);
  s.items = take(sizeof(WorkItem) * (size_t)s.max_rows);
  s.handed_on = take(sizeof(int2) * (size_t)(T * a->Hq + s.partial_cap / (a->D + 2)));  // (every row of every item: it writes an output or a partial)
  s.partials = take(4 * (size_t)s.partial_cap);
  s.total = off;
  s.fits = s.max_rows * a->Hkv < INT32_MAX / 2 && s.partial_cap < INT32_MAX;
  return s;
}

template <typename T>
T *at(void *ws, size_t off) {
  return reinterpret_cast<T *>(static_cast<char *>(ws) + off);
}

size_t workspace_size(const wisp_prompt_args *x, bool shared) {
  int sms = 0;
  if (setup(&sms) != WISP_OK) return 0;
  const Space sp = space(&x->attn, shared, sms);
  return sp.fits ? sp.total : 0;
}

wisp_status call(const wisp_prompt_args *x, const int32_t *ids, const int32_t *pages, void *ws, size_t ws_bytes, void *stream) {
  const wisp_attn_args *a = &x->attn;
  int sms = 0;
  const wisp_status st = setup(&sms);
  if (st != WISP_OK) return st;
  const Space sp = space(a, ids != nullptr, sms);
  if (!sp.fits) return WISP_ERR_UNSUPPORTED;
  if (!ws || ((uintptr_t)ws & 255) != 0 || ws_bytes < sp.total) return WISP_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const bool bf = a->qkv_dtype == WISP_BF16;
  PromptPlan p;
  std::memset(&p, 0, sizeof p);
  p.B = a->B;
  p.Hq = a->Hq;
  p.Hkv = a->Hkv;
  p.D = a->D;
  p.max_blocks_per_seq = a->max_blocks_per_seq;
  p.total_q_rows = a->total_q_rows;
  p.unit_rows = sp.unit_rows;
  p.sms = sms;
  p.merge_heads = (int64_t)a->total_q_rows * a->Hkv >= 4 * sms ? a->Hq / a->Hkv : 1;
  p.max_rows = sp.max_rows;
  p.partial_cap = sp.partial_cap;
  p.draft_lens = a->draft_lens;
  p.context_lens = a->context_lens;
  p.shared_ids = ids;
  p.shared_pages = pages;
  p.request_ids = a->request_ids;
  p.status = at<DeviceStatus>(ws, sp.status);
  p.header = at<PromptHeader>(ws, sp.header);
  p.q_row_start = at<int32_t>(ws, sp.q_row_start);
  p.req_flag = at<int32_t>(ws, sp.req_flag);
  p.req_run = at<int32_t>(ws, sp.req_run);
  p.run_info = at<int32_t>(ws, sp.run_info);
  p.segs = at<Segment>(ws, sp.segs);
  p.items = at<WorkItem>(ws, sp.items);
  p.partials = at<float>(ws, sp.partials);
  p.out = a->out;
  const int grid = (int)(sp.max_rows * a->Hkv < sms ? sp.max_rows * a->Hkv : sms);
  p.grid = grid;
  if (prompt_plan_launch(p, s) != cudaSuccess) return WISP_ERR_CUDA;
  if (a->B == 0) return WISP_OK;
  AttnParams ap;
  std::memset(&ap, 0, sizeof ap);
  ap.B = a->B;
  ap.Hq = a->Hq;
  ap.Hkv = a->Hkv;
  ap.D = a->D;
  ap.max_blocks_per_seq = a->max_blocks_per_seq;
  ap.num_blocks = a->num_blocks;
  ap.request_ids = a->request_ids;
  ap.block_tables = a->block_tables;
  ap.q = a->q;
  ap.k_cache = a->k_cache;
  ap.v_cache = a->v_cache;
  if (x->cache_dtype == WISP_E4M3) {
    ap.k_scale = x->k_scale;
    ap.v_scale = x->v_scale;
  }
  ap.out = a->out;
  ap.status = p.status;
  ap.header = &p.header->h;
  ap.header_mut = &p.header->h;
  ap.items = p.items;
  ap.partials = p.partials;
  ap.handed_on = at<int2>(ws, sp.handed_on);
  cudaError_t e = bf ? prompt_tc_launch(ap, a->total_q_rows, grid, s) : prompt_f32_launch(ap, grid, s);
  if (e == cudaSuccess) e = prompt_merge_launch(p, ap, !bf, s);
  return e == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t wisp_prompt_workspace_size(const wisp_prompt_args *a) { return check(a) == WISP_OK ? workspace_size(a, false) : 0; }

wisp_status wisp_prompt_attention(const wisp_prompt_args *a, void *ws, size_t ws_bytes, void *stream) {
  const wisp_status st = check(a);
  return st != WISP_OK ? st : call(a, nullptr, nullptr, ws, ws_bytes, stream);
}

size_t wisp_verify_shared_workspace_size(const wisp_shared_args *a) {
  return check(a) == WISP_OK ? workspace_size(&a->rows, true) : 0;
}

wisp_status wisp_verify_attention_shared(const wisp_shared_args *a, void *ws, size_t ws_bytes, void *stream) {
  const wisp_status st = check(a);
  return st != WISP_OK ? st : call(&a->rows, a->shared_ids, a->shared_pages, ws, ws_bytes, stream);
}

}  // extern "C"
