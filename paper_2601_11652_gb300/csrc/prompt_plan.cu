// prompt_plan.cu -- planner and merge of the attention of whole prompts and of batches with shared prefixes.
//
// Lengths, and which requests share pages, live on the device, so the planner runs there: one CTA finds the rows' offsets, the
// runs, the segments (prompt.cuh), the chunk length and the items, longest first.
#include "attn_merge.cuh"
#include "prompt.cuh"
#include "prompt_row.cuh"

#include <algorithm>
#include <cstring>

namespace wisp {

namespace {

constexpr int kMaxThreads = 1024;  // of the planner: see prompt_plan_launch
constexpr int kPage = 16;
constexpr int kBuckets = 1024;     // of the dispatch order, by key tiles of 64
constexpr int kMinKeys = kLeastChunk, kMinFull = kLeastFullChunk, kTile = kChunkTile;
constexpr int kAllKeys = 1 << 30;  // the context of a run's segment: every row sees all its keys (a table has fewer)
constexpr int kMaxChunk = 1 << 28; // a segment's keys and two chunks stay below 2^31
constexpr int kMaxRows = 1 << 24;  // k_r limit
constexpr int kMergeThreads = 128, kMergePerSM = 3;  // of the merge; CTAs that fit an SM
constexpr int kFew = 4, kHeads = 4; // chunks of a row, and rows, that a warp of the merge has in registers at once

// Inclusive block scan; *total the block's sum.  One barrier: s_w (32 values) may be written again only after another one.
template <int kThreads, typename T>
__device__ T scan_incl(T v, T *s_w, T *total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, warps = kThreads >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  if constexpr (kThreads == 32) {
    *total = __shfl_sync(0xffffffffu, v, 31);
    return v;
  }
  if (lane == 31) s_w[w] = v;
  __syncthreads();
  T t = lane < warps ? s_w[lane] : (T)0;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T o = __shfl_up_sync(0xffffffffu, t, d);
    if (lane >= d) t += o;
  }
  const T before = __shfl_sync(0xffffffffu, t, (w + 31) & 31);
  *total = __shfl_sync(0xffffffffu, t, 31);
  return v + (w > 0 ? before : (T)0);
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// Every thread's v added to *sum in shared memory (one atomic per warp: they are a loop each).
__device__ __forceinline__ void add_warp(unsigned long long *sum, int64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0 && v) atomicAdd(sum, (unsigned long long)v);
}

// Keys of a unit: those that its last row sees.
__device__ __forceinline__ int unit_end(const Segment &s, int u, int unit_rows, int g) {
  const int last = min((u + 1) * unit_rows, s.npos * g) - 1;
  return min(s.t1, s.ctx + last / g + 1);
}

// Where unit u's chunks are cut: keys of the chunk that its first key falls in, in front of it.
__device__ __forceinline__ int cut_off(const Segment &s, int u) { return s.span ? (int)((s.base + (int64_t)u * s.span) % s.chunk) : 0; }
// Chunks of a unit with keys [s.t0, end), and the c-th of them.
__device__ __forceinline__ int unit_chunks(const Segment &s, int u, int end) { return (end - s.t0 + cut_off(s, u) + s.chunk - 1) / s.chunk; }

}  // namespace

// What the planner keeps in shared memory where all segments fit: run_info and the segments.
template <int kThreads>
struct PlanShared {
  int32_t run[4 * kThreads];
  struct {
    Segment s;
    int32_t pad;  // (threads read and write theirs together: an odd number of words apart)
  } segs[kThreads];
};

// One CTA.  Its warps all go through all of the code, so what bounds it is their number times the code's length, fetched for the first time (one
// request: 15400 cycles with 32 warps, 10600 with 4, 9200 with one): it gets about as many threads as there are segments and list entries, and
// below kMaxThreads no code for more.  With at most kThreads requests and segments nothing else goes
// through global memory, and a list entry stands for all KV heads (an item is an entry and a head), so that most batches have at
// most one per thread.  48 prompts of up to 1500 tokens, 590 entries: 17300 cycles, 9 us.
template <int kThreads>
__global__ void __launch_bounds__(kThreads, 1) prompt_plan_kernel(const PromptPlan p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ __align__(16) uint8_t plan_smem[];
  PlanShared<kThreads> &sh = *reinterpret_cast<PlanShared<kThreads> *>(plan_smem);
  constexpr int kNb = kThreads == 32 ? 128 : kBuckets, kOwn = kNb / kThreads;  // buckets, and of a thread
  __shared__ int64_t s_scan[2][32];
  __shared__ int s_iscan[4][32];
  __shared__ unsigned long long s_keys, s_units, s_rows, s_floats;
  __shared__ int s_hist[kNb];
  __shared__ int s_first[kThreads + 1];
  __shared__ int s_any;
  const int tid = threadIdx.x;
  const int g = p.Hq / p.Hkv, R = p.unit_rows;
  if (tid == 0) {
    p.status->code = 0;
    p.status->pad = 0;
    p.status->request_id = 0;
    s_keys = s_units = 0;
    s_any = 0;
  }
#pragma unroll
  for (int i = 0; i < kOwn; ++i) s_hist[kOwn * tid + i] = 0;
  const int64_t cap_tokens = (int64_t)p.max_blocks_per_seq * kPage;
  constexpr bool kAll = kThreads < kMaxThreads;  // by the launch's choice: every segment has a thread
  const bool one = kAll || p.B <= kThreads;      // every request has one
  const int RS = one ? kThreads : p.B;
  int32_t *run_start = one ? sh.run : p.run_info;
  int32_t *run_end = run_start + RS, *run_first = run_start + 2 * RS, *run_valid = run_start + 3 * RS;

  // pass 1: offsets, validation, runs
  int64_t carry_k = 0;
  int n_runs = 0;
  int my_k = 0, my_ctx = 0, my_pages = 0, my_q0 = 0, my_run = -1;  // (of the last chunk: the only one where `one`)
  bool my_ok = false;
  for (int base = 0; base < (kAll ? 1 : p.B); base += kThreads) {
    const int r = base + tid;
    int64_t k = 0;
    int bad = 0, pages = 0, id = -1;
    bool start = false, last = false;
    if (r < p.B) {
      k = p.draft_lens[r];
      my_k = (int)k;
      const int64_t c = p.context_lens[r];
      my_ctx = (int)c;
      if (p.shared_ids) {
        id = p.shared_ids[r];
        pages = p.shared_pages[r];
      }
      const bool in = id >= 0 && pages > 0;
      if (in) {
        start = r == 0 || p.shared_ids[r - 1] != id || p.shared_pages[r - 1] != pages;
        last = r == p.B - 1 || p.shared_ids[r + 1] != id || p.shared_pages[r + 1] != pages;
      }
      if (k < 0) { bad = WISP_DEV_BAD_LENGTH; k = 0; }
      if (!bad && k >= kMaxRows) bad = WISP_DEV_UNSUPPORTED;
      if (!bad && (c < 0 || c + k + 1 > cap_tokens || (in && (int64_t)pages * kPage > c))) bad = WISP_DEV_BAD_LENGTH;
    }
    int64_t block_k;
    const int64_t q0 = carry_k + scan_incl<kThreads, int64_t>(k, s_scan[base / kThreads % 2], &block_k) - k + r;
    int starts = 0;
    const int run = n_runs + (p.shared_ids ? scan_incl<kThreads, int>(start, s_iscan[base / kThreads % 2], &starts) : 0) - 1;
    if (r < p.B) {
      if (!bad && q0 + k + 1 > p.total_q_rows) bad = WISP_DEV_BAD_LENGTH;  // rows outside the caller's buffers
      my_q0 = (int32_t)min(q0, (int64_t)INT32_MAX);
      my_ok = !bad;
      my_pages = pages;
      my_run = id >= 0 && pages > 0 ? run : -1;
      p.q_row_start[r] = my_q0;
      if (!kAll) p.req_flag[r] = bad ? REQ_BAD : REQ_OK;
      p.req_run[r] = my_run;
      if (bad) report(p.status, bad, p.request_ids, r);
      if (start) {
        run_start[run] = r;
        run_first[run] = INT32_MAX;
        run_valid[run] = 0;
      }
      if (last) run_end[run] = r + 1;
    }
    if (p.shared_ids) {
      __syncthreads();
      // a warp's members of a run together
      const int key = r < p.B && !bad ? my_run : -1;
      const unsigned same = __match_any_sync(0xffffffffu, key);
      if (key >= 0 && (tid & 31) == __ffs(same) - 1) {
        atomicMin(&run_first[run], r);
        atomicAdd(&run_valid[run], __popc(same));
      }
    }
    carry_k += block_k;
    n_runs += starts;
  }
  __syncthreads();
  if (tid == 0) {
    p.q_row_start[p.B] = (int32_t)min(carry_k + p.B, (int64_t)INT32_MAX);
    if (carry_k + p.B != p.total_q_rows) atomicCAS(&p.status->code, 0, (int32_t)WISP_DEV_BAD_LENGTH);
  }

  // pass 2: segments, their units, and how many keys all units have
  const int n_segs = p.B + n_runs;
  const bool few = kAll || n_segs <= kThreads;
  auto seg = [&](int i) -> Segment & { return few ? sh.segs[i].s : p.segs[i]; };
  int64_t sum_keys = 0, sum_units = 0;  // of this thread
  for (int i = tid; i < n_segs; i += kAll ? kAllKeys : kThreads) {
    Segment s;
    memset(&s, 0, sizeof s);
    s.pbase = -1;
    if (i < p.B) {
      const int run = one ? my_run : p.req_run[i];
      const bool shared = run >= 0 && run_valid[run] > 1;
      if (run >= 0 && !shared) p.req_run[i] = -1;
      s.r = i;
      if (one ? my_ok : p.req_flag[i] == REQ_OK) {
        s.q0 = one ? my_q0 : p.q_row_start[i];
        s.npos = (one ? my_k : p.draft_lens[i]) + 1;
        s.ctx = one ? my_ctx : p.context_lens[i];
        s.t0 = shared ? (one ? my_pages : p.shared_pages[i]) * kPage : 0;
        s.t1 = s.ctx + s.npos;
        s.shared = shared;
      }
    } else if (run_valid[i - p.B] > 1) {
      const int run = i - p.B, a = run_first[run], b = run_end[run];
      s.r = a;
      s.q0 = p.q_row_start[a];
      s.npos = min(b < p.B ? p.q_row_start[b] : p.total_q_rows, p.total_q_rows) - s.q0;
      s.ctx = kAllKeys;
      s.t1 = p.shared_pages[a] * kPage;
      s.shared = 1;
    }
    if (s.npos > 0) {
      s.units = ceil_div(s.npos * g, R);  // (rows times g: below 2^30)
      const int64_t len = ((int64_t)(unit_end(s, 0, R, g) - s.t0) + (s.t1 - s.t0) + 1) / 2;
      sum_keys += len * s.units;
      sum_units += s.units;
    }
    seg(i) = s;
  }
  add_warp(&s_keys, sum_keys);
  add_warp(&s_units, sum_units);
  __syncthreads();

  // Where sequences are cut.  A cut costs a merge, and its chunks begin and end like items of their own.  With at least as many units
  // as SMs the longest-first order balances units of many lengths: only a segment whose longest unit is above 5/4 of an SM's
  // average work is cut.  Many units of one length it balances badly (168 equal ones on 152 SMs: two rounds), so where they are
  // three quarters of all work (the rest fills gaps), they are cut from a fifth of an SM's work on: they lie one behind the other, and every
  // multiple of an SM's average is a cut, whatever unit it falls in.  (1344 rows behind 16384 tokens: 250 us, 354 without.)  With fewer
  // units than SMs, about two items per SM.
  const int64_t keys = (int64_t)s_keys * p.Hkv, avg = keys < kAllKeys ? ceil_div((int)keys, p.sms) : (keys + p.sms - 1) / p.sms;  // (a division in 64 bits is 100 instructions)
  const bool many = (int64_t)s_units * p.Hkv >= p.sms;
  const int64_t want = many ? avg : (avg + 1) / 2;
  const int average = (int)min((want + kTile - 1) / kTile * kTile, (int64_t)kMaxChunk);
  bool cuts = true;
  // how a segment is cut: its chunk length, and whether its units are cut as they lie one behind the other
  auto rule = [&](Segment &s) {
    const int len = s.t1 - s.t0, shortest = unit_end(s, 0, R, g) - s.t0;
    const int chunk = max(average, min(R, s.npos * g) > kTile ? kMinFull : kMinKeys);
    const bool even = s.units > 1 && 2 * (int64_t)shortest > len && 4 * (int64_t)s.units * p.Hkv * len >= 3 * keys;
    const bool cut = cuts && (many ? (even ? 5 * (int64_t)len > avg : 4 * (int64_t)len > 5 * avg) : len > chunk);
    s.chunk = cut ? chunk : kAllKeys;
    s.span = cut && many ? (len + kTile - 1) / kTile * kTile : 0;
    s.chunks = cut ? (len + (s.span ? chunk - kTile : 0) + chunk - 1) / chunk : 1;  // at most
  };
  for (;;) {  // (twice at most: without cuts everything fits, by the host's bounds)
    if (tid == 0) s_rows = s_floats = 0;
    __syncthreads();
    int64_t sum_rows = 0, sum_floats = 0;
    for (int i = tid; i < n_segs; i += kAll ? kAllKeys : kThreads) {
      Segment s = seg(i);
      if (s.npos <= 0) continue;
      rule(s);
      sum_rows += (int64_t)s.units * s.chunks;
      s.part_h = 0;
      if (s.chunks > 1 || s.shared) {
        const int rows_last = s.npos * g - (s.units - 1) * R;
        const int64_t floats = s.chunks * ((int64_t)(s.units - 1) * slot_floats(R, p.D) + slot_floats(rows_last, p.D));
        sum_floats += p.Hkv * floats;
        s.part_h = (int)min(floats, (int64_t)INT32_MAX);
      }
      seg(i) = s;
    }
    add_warp(&s_rows, sum_rows);
    add_warp(&s_floats, sum_floats);
    __syncthreads();
    if (((int64_t)s_rows <= p.max_rows && (int64_t)s_floats <= p.partial_cap) || !cuts) break;
    cuts = false;
    __syncthreads();
  }

  // pass 3: entries and partials of each segment
  int64_t row_carry = 0, float_carry = 0, span_carry = 0;
  for (int base = 0; base < (kAll ? 1 : n_segs); base += kThreads) {
    const int i = base + tid;
    int rows = 0;
    int64_t floats = 0, spans = 0;
    Segment s;
    s.npos = 0;
    if (i < n_segs) s = seg(i);
    if (s.npos > 0) {
      rows = s.units * s.chunks;
      spans = (int64_t)s.units * s.span;
      floats = (int64_t)s.part_h * p.Hkv;
    }
    int ti;
    int64_t tf, ts;
    const int ii = scan_incl<kThreads, int>(rows, s_iscan[2], &ti);
    const int64_t fi = scan_incl<kThreads, int64_t>(floats, s_scan[0], &tf);
    const int64_t si = scan_incl<kThreads, int64_t>(spans, s_scan[1], &ts);
    s.base = s.span ? (int)((span_carry + si - spans) % s.chunk) : 0;
    if (i < n_segs) {
      if (s.npos > 0 && (row_carry + ii > p.max_rows || float_carry + fi > p.partial_cap)) {
        // cannot happen with the host's bounds; refuse rather than overflow
        report(p.status, WISP_DEV_UNSUPPORTED, p.request_ids, s.r);
        s.npos = s.units = s.chunks = 0;
      }
      s.pbase = floats > 0 ? (int32_t)(float_carry + fi - floats) : -1;
      if (s.npos > 0 && floats > 0) s_any = 1;
      s.first = (int32_t)(row_carry + ii - rows);
      if (few) s_first[tid] = s.first;
      seg(i) = s;
      if (few) p.segs[i] = s;  // (for the merge)
    }
    row_carry += ti;
    float_carry += tf;
    span_carry += ts;
    __syncthreads();
  }
  const int n_all = (int)min(row_carry, p.max_rows);
  const bool single = few && n_all <= kThreads;  // an entry per thread, kept from pass 4 to pass 5

  // pass 4: the histogram of the entries' lengths; pass 5: each entry at its place in the dispatch order, longest first
  auto bucket_of = [&](int tokens) { return kNb - 1 - min(ceil_div(tokens, 64), kNb - 1); };
  WorkItem w;
  int bucket = -1;
  for (int pass = 0; pass < 2; ++pass) {
    for (int base = 0; base < (kAll ? 1 : n_segs); base += kThreads) {
      const int in = min(kThreads, n_segs - base);
      int lo = 0, hi = n_all;
      if (!few) {
        if (tid < in) s_first[tid] = seg(base + tid).first;
        if (tid == 0) s_first[kThreads] = base + kThreads < n_segs ? seg(base + kThreads).first : n_all;
        __syncthreads();
        lo = s_first[0];
        hi = min(s_first[kThreads], n_all);
      }
      for (int x = lo + tid; x < hi; x += kThreads) {
        if (pass == 0 || !single) {
          bucket = -1;
          int a = 0, b = in - 1;  // the last segment whose first entry is <= x
          while (a < b) {
            const int mid = (a + b + 1) >> 1;
            if (s_first[mid] <= x) a = mid;
            else b = mid - 1;
          }
          const Segment s = seg(base + a);
          if (s.units <= 0) continue;
          const int rel = x - s.first, u = rel / s.chunks, c = rel - u * s.chunks;
          if (u >= s.units) continue;
          const int end = unit_end(s, u, R, g), off = cut_off(s, u);
          w.t0 = s.t0 + max(0, c * s.chunk - off);
          w.t1 = (int)min((int64_t)end, (int64_t)s.t0 - off + (int64_t)(c + 1) * s.chunk);
          if (w.t1 <= w.t0) continue;  // (the unit ends before this chunk)
          bucket = bucket_of(w.t1 - w.t0);
          w.r = s.r;
          w.h = 0;
          w.rows = min(R, s.npos * g - u * R);
          w.q0 = s.q0;
          w.ctx = s.ctx;
          w.row0 = u * R;
          w.rg = u;
          w.nrg = s.part_h;
          w.pbase = 0;
          const bool whole = w.t0 == s.t0 && w.t1 == end && !s.shared;  // its items write the outputs
          w.poff = s.pbase < 0 || whole ? -1 : s.pbase + u * s.chunks * slot_floats(R, p.D) + c * slot_floats(w.rows, p.D);
        }
        if (bucket < 0) continue;
        const int at = atomicAdd(&s_hist[bucket], 1);
        if (pass == 1) p.items[at] = w;
      }
      __syncthreads();
    }
    if (pass == 0) {
      int n[kOwn], sum = 0, total;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) sum += n[i] = s_hist[kOwn * tid + i];
      int at = scan_incl<kThreads, int>(sum, s_iscan[3], &total) - sum;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {  // (a thread's own)
        s_hist[kOwn * tid + i] = at;
        at += n[i];
      }
      if (tid == 0) {
        PromptHeader hd;
        memset(&hd, 0, sizeof hd);
        hd.h.n_items = total * p.Hkv;
        hd.h.next_item = p.grid;
        hd.partials = s_any;
        *p.header = hd;
      }
      __syncthreads();
    }
  }
}

// The partials of a row joined: O = sum_i O_i 2^(m_i - m) / sum_i l_i 2^(m_i - m), m = max m_i.  A warp takes a query position and a KV
// head, kHeads rows at a time (units are whole positions, so they lie in one; single rows where rows are few); grid columns are requests, so that no row has to
// look for its own.  Up to kFew chunks, as almost always, every lane computes their weights itself.  Bound by instructions, then by the
// partials' bytes (mostly in L2): 1300 rows of 32 heads of 128, three to five chunks each, 24 us.
template <int D, typename T, bool KV8>
__global__ void __launch_bounds__(kMergeThreads, kMergePerSM) prompt_merge_kernel(const __grid_constant__ PromptPlan p, const __grid_constant__ AttnParams a) {
  // Rows that are computed once more (prompt.cuh), behind the others, by one CTA per SM (where
  // every warp of all CTAs looked for their number, a prompt of 64 tokens took 1.3 us more, in a row for that line; every CTA that fits, 1 us).
  const int cta = blockIdx.y * gridDim.x + blockIdx.x;
  int n_on = 0;
  // (the attention's CTAs let this kernel start once the planner is done: what it has written may be read before they are)
  const bool partials = p.header->partials;
  if (!partials) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (cta >= p.sms || !__syncthreads_or(threadIdx.x == 0 ? __ldcg(&p.header->h.handed_on) : 0)) return;
    n_on = __ldcg(&p.header->h.handed_on);
  }
  const int takers = min((int)(gridDim.x * gridDim.y), p.sms), lane = threadIdx.x & 31;
  const int g = p.Hq / p.Hkv, R = p.unit_rows, subs = g / p.merge_heads;
  constexpr int CPL = D / 32;
  const int x0 = blockIdx.y * (kMergeThreads / 32) + (threadIdx.x >> 5), x_step = gridDim.y * (kMergeThreads / 32);

  for (int r = blockIdx.x; r < p.B && partials; r += gridDim.x) {
    const Segment own = p.segs[r];
    const int run = p.req_run[r];
    const Segment pre = p.segs[run >= 0 ? p.B + run : r];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (r == blockIdx.x && cta < takers) n_on = __ldcg(&p.header->h.handed_on);
    if (own.npos <= 0 || own.pbase < 0) continue;  // (refused, or its items have written the outputs)
    const int work = own.npos * p.Hkv * subs;
    for (int x = x0; x < work; x += x_step) {
      const int y = x / subs, j = y / p.Hkv, hk = y - j * p.Hkv, h0 = (x - y * subs) * p.merge_heads;
      // per segment (0: the run's, 1: the request's own): a row's first O and m, the distance of chunks and how many
      struct Where {
        const float *po[2], *pm[2];
        int step[2], n[2], nl[2];
      };
      auto where = [&](int hh) {
        Where w;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const Segment &s = i == 0 ? pre : own;
          const int rho = (own.q0 + j - s.q0) * g + hh, u = rho / R, rr = rho - u * R;
          const int rows = min(R, s.npos * g - u * R);
          w.step[i] = slot_floats(rows, D);
          w.nl[i] = rows;
          w.n[i] = i == 0 && run < 0 ? 0 : min(s.chunks, unit_chunks(s, u, unit_end(s, u, R, g)));
          const float *base = p.partials + (s.pbase + hk * s.part_h + u * s.chunks * slot_floats(R, D));
          w.po[i] = base + rr * D + lane * CPL;
          w.pm[i] = base + rows * D + rr;
        }
        return w;
      };
      Where w = where(h0);
      T *dst = static_cast<T *>(p.out) + ((int64_t)(own.q0 + j) * p.Hq + hk * g + h0) * D + lane * CPL;
      // a chunk none of whose keys a row sees adds nothing; its m is -inf and its l 0, or a NaN where its scores are no numbers
      if (w.n[0] + w.n[1] <= kFew) {
        const int total = w.n[0] + w.n[1];
        if (total == 1 && !own.shared) continue;  // (a unit that no cut fell in)
        for (int hh = 0; hh < p.merge_heads; hh += kHeads) {
          // all loads of kHeads rows first
          float v[kHeads][kFew][CPL], mc[kHeads][kFew], lc[kHeads][kFew];
#pragma unroll
          for (int x = 0; x < kHeads; ++x)
#pragma unroll
            for (int c = 0; c < kFew; ++c) {
              mc[x][c] = -INFINITY;
              lc[x][c] = 0.0f;
              if (c < total && hh + x < p.merge_heads) {
                const bool z = c < w.n[0];
                const int at = z ? c * w.step[0] : (c - w.n[0]) * w.step[1];
                const float *q = (z ? w.pm[0] : w.pm[1]) + at + hh + x;
                mc[x][c] = __ldcg(q);
                lc[x][c] = __ldcg(q + (z ? w.nl[0] : w.nl[1]));
                ld_cols<CPL>((z ? w.po[0] : w.po[1]) + at + (hh + x) * D, v[x][c]);
              }
            }
#pragma unroll
          for (int x = 0; x < kHeads; ++x) {
            if (hh + x >= p.merge_heads) break;
            uint32_t marks = 0;
#pragma unroll
            for (int c = 0; c < kFew; ++c) marks |= __float_as_uint(lc[x][c]);
            float m = -INFINITY, den = 0.0f, acc[CPL];
#pragma unroll
            for (int q = 0; q < CPL; ++q) acc[q] = 0.0f;
#pragma unroll
            for (int c = 0; c < kFew; ++c) m = fmaxf(m, mc[x][c]);
            m += 2.0f;  // (kFew sums that are each within the values' range)
#pragma unroll
            for (int c = 0; c < kFew; ++c) {
              if (mc[x][c] == -INFINITY) {
                den += lc[x][c];
              } else {
                const float f = ptx::ex2(mc[x][c] - m);
                den = fmaf(lc[x][c], f, den);
#pragma unroll
                for (int q = 0; q < CPL; ++q) acc[q] = fmaf(v[x][c][q], f, acc[q]);
              }
            }
            if (!(marks >> 31)) st_cols<CPL>(dst + (hh + x) * D, acc, 1.0f / den);
          }
        }
      } else {
        for (int hh = 0; hh < p.merge_heads; ++hh, dst += D) {
          const int total = w.n[0] + w.n[1];
          const float room = (float)(32 - __clz(total));  // (their sum stays within the values' range)
          auto at = [&](const float *const (&base)[2], int c) {
            return c < w.n[0] ? base[0] + c * w.step[0] : base[1] + (c - w.n[0]) * w.step[1];
          };
          float m = -INFINITY, den = 0.0f, acc[CPL];
          bool mark = false;
#pragma unroll
          for (int q = 0; q < CPL; ++q) acc[q] = 0.0f;
          for (int c0 = 0; c0 < total; c0 += 32) {  // 32 chunks at a time, a lane each
            const int c = c0 + lane;
            float mc = -INFINITY, lc = 0.0f;
            if (c < total) {
              const float *q = at(w.pm, c) + hh;
              mc = __ldcg(q);
              lc = __ldcg(q + (c < w.n[0] ? w.nl[0] : w.nl[1]));
              mark = mark || is_marked(lc);
            }
            const float mn = fmaxf(m, ptx::warp_max(mc));
            if (mn != m) {
              const float a = m == -INFINITY ? 0.0f : ptx::ex2(m - mn);
              den = m == -INFINITY ? den : den * a;
#pragma unroll
              for (int q = 0; q < CPL; ++q) acc[q] *= a;
              m = mn;
            }
            const float f = mc == -INFINITY ? -1.0f : ptx::ex2(mc - m - room);
            den = mc == -INFINITY ? den + lc : fmaf(lc, f, den);
            const int nc = min(32, total - c0);
#pragma unroll 4
            for (int i = 0; i < nc; ++i) {
              const float fi = __shfl_sync(0xffffffffu, f, i);
              float v[CPL];
              ld_cols<CPL>(at(w.po, c0 + i) + hh * D, v);
#pragma unroll
              for (int q = 0; q < CPL; ++q)
                if (!(fi < 0.0f)) acc[q] = fmaf(v[q], fi, acc[q]);
            }
          }
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
          if (!__any_sync(0xffffffffu, mark)) st_cols<CPL>(dst, acc, 1.0f / den);
        }
      }
    }
  }

  for (int i = kRowsAtOnce * (cta * (kMergeThreads / 32) + (threadIdx.x >> 5)); i < n_on; i += kRowsAtOnce * takers * (kMergeThreads / 32)) {
    int row[kRowsAtOnce], head[kRowsAtOnce];
    uint32_t todo = 0;
#pragma unroll
    for (int k = 0; k < kRowsAtOnce; ++k) {
      const int2 e = i + k < n_on ? __ldcg(a.handed_on + i + k) : make_int2(0, 0);
      row[k] = e.x;
      head[k] = e.y;
      todo |= i + k < n_on ? 1u << k : 0u;
    }
#pragma unroll 1
    while (todo) {  // those of the first one's request and KV head
      int row0 = 0, hk = 0;
#pragma unroll
      for (int k = kRowsAtOnce - 1; k >= 0; --k)
        if (todo >> k & 1) {
          row0 = row[k];
          hk = head[k] / g;
        }
      const int r = request_of(p, row0);
      uint32_t use = 0;
#pragma unroll
      for (int k = 0; k < kRowsAtOnce; ++k)
        if ((todo >> k & 1) && head[k] / g == hk && row[k] >= p.q_row_start[r] && row[k] < p.q_row_start[r + 1]) use |= 1u << k;
      todo &= ~use;
      if (p.segs[r].npos > 0) prompt_rows<D, T, KV8>(p, a, r, row, head, hk, use);  // (a run's rows are those of its refused requests, too)
    }
  }
}

namespace {

template <int kThreads>
cudaError_t plan_setup() {
  return cudaFuncSetAttribute(prompt_plan_kernel<kThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(PlanShared<kThreads>));
}
template <int kThreads>
void plan_launch(const PromptPlan &p, cudaStream_t s) {
  prompt_plan_kernel<kThreads><<<1, kThreads, sizeof(PlanShared<kThreads>), s>>>(p);
}

}  // namespace

cudaError_t prompt_plan_setup() {
  cudaError_t e = plan_setup<32>();
  if (e == cudaSuccess) e = plan_setup<128>();
  if (e == cudaSuccess) e = plan_setup<256>();
  if (e == cudaSuccess) e = plan_setup<512>();
  return e == cudaSuccess ? plan_setup<kMaxThreads>() : e;
}

cudaError_t prompt_plan_launch(const PromptPlan &p, cudaStream_t s) {
  // threads: requests and runs have one each, list entries about one (their number is bounded by the rows)
  const int64_t most = std::max<int64_t>((p.shared_ids ? 2 : 1) * (int64_t)p.B, (int64_t)p.total_q_rows * (p.Hq / p.Hkv) / p.unit_rows + p.B);
  if (most <= 32) plan_launch<32>(p, s);
  else if (most <= 128) plan_launch<128>(p, s);
  else if (most <= 256) plan_launch<256>(p, s);
  else if (most <= 512) plan_launch<512>(p, s);
  else plan_launch<kMaxThreads>(p, s);
  return cudaGetLastError();
}

cudaError_t prompt_merge_launch(const PromptPlan &p, const AttnParams &a, bool f32, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  // about 12 CTAs per SM (kMergePerSM fit), or one per four warps that have work
  const int most = p.sms * 12;
  const int64_t ctas = std::min<int64_t>(most, ((int64_t)p.total_q_rows * p.Hq / p.merge_heads + kMergeThreads / 32 - 1) / (kMergeThreads / 32));
  const int cols = std::min(p.B, most);
  cfg.gridDim = dim3((unsigned)cols, (unsigned)((ctas + cols - 1) / cols));
  cfg.blockDim = dim3(kMergeThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (a.k_scale) {
    if (f32) return cudaLaunchKernelEx(&cfg, p.D == 128 ? prompt_merge_kernel<128, float, true> : prompt_merge_kernel<64, float, true>, p, a);
    return cudaLaunchKernelEx(&cfg, p.D == 128 ? prompt_merge_kernel<128, uint16_t, true> : prompt_merge_kernel<64, uint16_t, true>, p, a);
  }
  if (f32) return cudaLaunchKernelEx(&cfg, p.D == 128 ? prompt_merge_kernel<128, float, false> : prompt_merge_kernel<64, float, false>, p, a);
  return cudaLaunchKernelEx(&cfg, p.D == 128 ? prompt_merge_kernel<128, uint16_t, false> : prompt_merge_kernel<64, uint16_t, false>, p, a);
}

}  // namespace wisp
