// prompt.cuh -- plan and parameters of the attention of whole prompts and of batches with shared prefixes
// (include/wisp_prompt.h).
//
// The work is cut into segments: rows of one KV head that see the same keys but for the causal end.  Request r is segment r, its
// query rows over its own keys [P_r, c_r + k_r + 1), where P_r is its run's shared prefix or 0; run i of requests that share
// pages is segment B + i, all its rows over keys [0, P).  A segment's rows are cut into units of `unit_rows`, its keys into chunks
// of its chunk length; an item (plan.cuh) is a chunk of a unit of one KV head.  The list holds them without the head: entry i / Hkv and head
// i mod Hkv make item i (item_at).  Where a row has its keys in more than one item
// the items leave partials (O, m, l), and prompt_merge_kernel joins them.
#pragma once

#include <cstddef>

#include "attn.cuh"

namespace wisp {

struct Segment {  // 64 bytes
  int32_t r;        // whose block table
  int32_t q0;       // first query row
  int32_t npos;     // query positions (0: no work)
  int32_t t0, t1;   // keys
  int32_t ctx;      // position j sees keys up to ctx + j
  int32_t units, chunks;
  int32_t pbase;    // first partial (floats), -1: the segment has none, its items write outputs
  int32_t part_h;   // floats of one KV head's partials
  int32_t first;    // first list entry (empty ones included)
  int32_t chunk;    // keys per chunk
  int32_t span;     // > 0: unit u's chunks end at multiples of `chunk` from base + u * span on, not from its first key
  int32_t base;
  int32_t shared;   // 1: its rows have keys in another segment, too
  int32_t pad;
};
static_assert(sizeof(Segment) == 64, "segment layout");

// Of the planner's chunks: whole key tiles, and not shorter than this, of units of more than one tile of rows (whose partials cost more) than that.
constexpr int kChunkTile = 128, kLeastChunk = 256, kLeastFullChunk = 1024;

struct PromptHeader {
  PlanHeader h;        // what the attention kernels read
  int32_t partials;    // 1: the merge has work
  int32_t pad[7];
};
static_assert(offsetof(PromptHeader, h) == 0, "the kernels that read a PlanHeader find it there");

struct PromptPlan {
  int B, Hq, Hkv, D, max_blocks_per_seq, total_q_rows;
  int unit_rows;       // rows of a unit: whole positions of an item's two tiles (bf16 queries) or of its one (fp32)
  int sms;
  int grid;            // CTAs of the attention kernel: each takes its first item by its index
  int64_t max_rows, partial_cap;  // list entries, floats
  const int32_t *draft_lens, *context_lens, *shared_ids, *shared_pages;  // shared_*: null without runs
  const int64_t *request_ids;
  DeviceStatus *status;
  PromptHeader *header;
  int32_t *q_row_start;  // [B + 1]
  int32_t *req_flag;     // [B]
  int32_t *req_run;      // [B] run of request r, -1: none
  int32_t *run_info;     // [4, B] per run: first request, end, first valid request, valid requests
  Segment *segs;         // [2 B]
  WorkItem *items;
  // of the merge
  int merge_heads;     // heads of a KV head's group that a warp takes one after the other: all, or one where rows are few
  float *partials;
  void *out;
};

// Item `it` of the list.  An entry's nrg is the distance of its heads' partials.
__device__ __forceinline__ WorkItem item_at(const AttnParams &p, int it) {
  const int row = it / p.Hkv;
  WorkItem w = p.items[row];
  w.h = it - row * p.Hkv;
  if (w.poff >= 0) w.poff += w.h * w.nrg;
  return w;
}

// Rows of a segment that share a partial's slot, and floats of a slot.
__device__ __forceinline__ int slot_floats(int rows, int D) { return (rows * (D + 2) + 3) / 4 * 4; }

// Rows that the attention kernels hand on to prompt_row.cuh, as they cannot hold them.
//
// A score becomes a weight in one fused multiply-add, 2^(x scale - m) from the sum x of products.  It is rounded once; but m is a rounded number, so
// where it is far from zero the largest weight is off by up to 2^(half a step of m), and a row that has had one beyond kFar is computed once more.
//
// The kernel for fp32 queries hands on rows whose queries are past 2^44, and (rows of a tile that not all see) rows whose largest V is 2^78 times
// that of the first one that it sees in the tile.
//
// They go into a list, once for every item that they are handed on from; the merge does not write those whose partials say so by the sign of their l
// (which is never negative).
constexpr float kFar = 0x1p23f;
__device__ __forceinline__ bool is_far(float m) { return fabsf(m) > kFar && fabsf(m) < INFINITY; }
__device__ __forceinline__ float marked(float l) { return __uint_as_float(__float_as_uint(l) | 0x80000000u); }
__device__ __forceinline__ bool is_marked(float l) { return __float_as_uint(l) >> 31; }
__device__ __forceinline__ void hand_on(const AttnParams &p, int row, int head) {
  p.handed_on[atomicAdd(&p.header_mut->handed_on, 1)] = make_int2(row, head);
}

cudaError_t prompt_plan_setup();  // once per device: shared-memory attributes
cudaError_t prompt_plan_launch(const PromptPlan &p, cudaStream_t s);
cudaError_t prompt_merge_launch(const PromptPlan &p, const AttnParams &a, bool f32, cudaStream_t s);

// query positions of a tile of 128 rows
inline int prompt_tile_positions(int g) { return 128 / g; }
cudaError_t prompt_tc_setup();
cudaError_t prompt_tc_launch(const AttnParams &p, int total_q_rows, int grid, cudaStream_t s);
// tcgen05 kernel for fp32 queries: an item is one tile
cudaError_t prompt_f32_setup();
cudaError_t prompt_f32_launch(const AttnParams &p, int grid, cudaStream_t s);

}  // namespace wisp
