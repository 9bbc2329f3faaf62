// prompt_plan.cu -- planner and merge of the attention of whole prompts and of batches with shared prefixes.
//
// Lengths, and which requests share pages, live on the device, so the planner runs there: one CTA finds the rows' offsets, the
// runs, the segments (prompt.cuh), the chunk length and the items, longest first.
#include "attn_merge.cuh"
#include "prompt.cuh"

#include <cstring>

namespace wisp {

namespace {

constexpr int kThreads = 1024;
constexpr int kPage = 16;
constexpr int kBuckets = 1024;     // of the dispatch order, by key tiles of 64
constexpr int kMinKeys = 256;      // chunks are not shorter
constexpr int kTile = 128;         // and are whole key tiles
constexpr int kAllKeys = 1 << 30;  // the context of a run's segment: every row sees all its keys
constexpr int kMaxRows = 1 << 24;  // k_r limit
constexpr int kMergeThreads = 128;

// Inclusive block scan; *total the block's sum.  One barrier: s_w (32 values) may be written again only after another one.
template <typename T>
__device__ T scan_incl(T v, T *s_w, T *total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const T o = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += o;
  }
  if (lane == 31) s_w[w] = v;
  __syncthreads();
  T t = s_w[lane];
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

// Keys of a unit: those that its last row sees.
__device__ __forceinline__ int unit_end(const Segment &s, int u, int unit_rows, int g) {
  const int last = min((u + 1) * unit_rows, s.npos * g) - 1;
  return min(s.t1, s.ctx + last / g + 1);
}

}  // namespace

__global__ void __launch_bounds__(kThreads, 1) prompt_plan_kernel(const PromptPlan p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  __shared__ int64_t s_scan[2][32];
  __shared__ int s_iscan[4][32];
  __shared__ unsigned long long s_keys, s_units, s_items, s_floats;
  __shared__ int s_hist[kBuckets];
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
  s_hist[tid] = 0;
  static_assert(kBuckets == kThreads, "one bucket per thread");
  const int64_t cap_tokens = (int64_t)p.max_blocks_per_seq * kPage;
  int32_t *run_start = p.run_info, *run_end = p.run_info + p.B, *run_first = p.run_info + 2 * p.B, *run_valid = p.run_info + 3 * p.B;

  // pass 1: offsets, validation, runs
  int64_t carry_k = 0;
  int n_runs = 0;
  for (int base = 0; base < p.B; base += kThreads) {
    const int r = base + tid;
    int64_t k = 0;
    int bad = 0, pages = 0, id = -1;
    bool start = false, last = false;
    if (r < p.B) {
      k = p.draft_lens[r];
      const int64_t c = p.context_lens[r];
      if (p.shared_ids) {
        id = p.shared_ids[r];
        pages = p.shared_pages[r];
      }
      const bool in = id >= 0 && pages > 0;
      start = in && (r == 0 || p.shared_ids[r - 1] != id || p.shared_pages[r - 1] != pages);
      last = in && (r == p.B - 1 || p.shared_ids[r + 1] != id || p.shared_pages[r + 1] != pages);
      if (k < 0) { bad = WISP_DEV_BAD_LENGTH; k = 0; }
      if (!bad && k >= kMaxRows) bad = WISP_DEV_UNSUPPORTED;
      if (!bad && (c < 0 || c + k + 1 > cap_tokens || (in && (int64_t)pages * kPage > c))) bad = WISP_DEV_BAD_LENGTH;
    }
    int64_t block_k;
    const int64_t q0 = carry_k + scan_incl<int64_t>(k, s_scan[base / kThreads % 2], &block_k) - k + r;
    int starts = 0;
    const int run = n_runs + (p.shared_ids ? scan_incl<int>(start, s_iscan[base / kThreads % 2], &starts) : 0) - 1;
    if (r < p.B) {
      if (!bad && q0 + k + 1 > p.total_q_rows) bad = WISP_DEV_BAD_LENGTH;  // rows outside the caller's buffers
      p.q_row_start[r] = (int32_t)min(q0, (int64_t)INT32_MAX);
      p.req_flag[r] = bad ? REQ_BAD : REQ_OK;
      p.req_run[r] = id >= 0 && pages > 0 ? run : -1;
      if (bad) report(p.status, bad, p.request_ids, r);
      if (start) {
        run_start[run] = r;
        run_first[run] = INT32_MAX;
        run_valid[run] = 0;
      }
      if (last) run_end[run] = r + 1;
    }
    __syncthreads();
    if (r < p.B && !bad && id >= 0 && pages > 0) {
      atomicMin(&run_first[run], r);
      atomicAdd(&run_valid[run], 1);
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
  for (int i = tid; i < n_segs; i += kThreads) {
    Segment s;
    memset(&s, 0, sizeof s);
    s.pbase = -1;
    if (i < p.B) {
      const int run = p.req_run[i];
      const bool shared = run >= 0 && run_valid[run] > 1;
      if (run >= 0 && !shared) p.req_run[i] = -1;
      s.r = i;
      if (p.req_flag[i] == REQ_OK) {
        s.q0 = p.q_row_start[i];
        s.npos = p.draft_lens[i] + 1;
        s.ctx = p.context_lens[i];
        s.t0 = shared ? p.shared_pages[i] * kPage : 0;
        s.t1 = s.ctx + s.npos;
        if (shared) s.pbase = 0;
      }
    } else if (run_valid[i - p.B] > 1) {
      const int run = i - p.B, a = run_first[run], b = run_end[run];
      s.r = a;
      s.q0 = p.q_row_start[a];
      s.npos = min(b < p.B ? p.q_row_start[b] : p.total_q_rows, p.total_q_rows) - s.q0;
      s.ctx = kAllKeys;
      s.t1 = p.shared_pages[a] * kPage;
      s.pbase = 0;
    }
    if (s.npos > 0) {
      s.units = (int)(((int64_t)s.npos * g + R - 1) / R);
      const int64_t len = ((int64_t)(unit_end(s, 0, R, g) - s.t0) + (s.t1 - s.t0) + 1) / 2;
      atomicAdd(&s_keys, (unsigned long long)(len * s.units));
      atomicAdd(&s_units, (unsigned long long)s.units);
      if (s.pbase == 0) s_any = 1;
    }
    p.segs[i] = s;
  }
  __syncthreads();

  // the chunk length: with at least as many units as SMs, only sequences longer than 5/4 of the average work per SM are cut (a
  // longest-first order balances the rest, and a cut costs a merge); with fewer, about two items per SM
  const int64_t keys = (int64_t)s_keys * p.Hkv;
  const bool many = (int64_t)s_units * p.Hkv >= p.sms;
  int64_t want = many ? (keys + p.sms - 1) / p.sms * 5 / 4 : (keys + 2 * p.sms - 1) / (2 * p.sms);
  want = (want < kMinKeys ? kMinKeys : want + kTile - 1) / kTile * kTile;
  int chunk = (int)min(want, (int64_t)kAllKeys);
  for (;;) {  // (twice at most: without cuts everything fits, by the host's bounds)
    if (tid == 0) s_items = s_floats = 0;
    __syncthreads();
    for (int i = tid; i < n_segs; i += kThreads) {
      const Segment s = p.segs[i];
      if (s.npos <= 0) continue;
      const int chunks = (s.t1 - s.t0 + chunk - 1) / chunk;
      atomicAdd(&s_items, (unsigned long long)s.units * chunks * p.Hkv);
      if (chunks > 1 || s.pbase == 0) {
        const int rows_last = s.npos * g - (s.units - 1) * R;
        atomicAdd(&s_floats, (unsigned long long)p.Hkv * chunks *
                                 ((unsigned long long)(s.units - 1) * slot_floats(R, p.D) + slot_floats(rows_last, p.D)));
      }
    }
    __syncthreads();
    if (((int64_t)s_items <= p.max_items && (int64_t)s_floats <= p.partial_cap) || chunk == kAllKeys) break;
    chunk = kAllKeys;
    __syncthreads();
  }

  // pass 3: items and partials of each segment; lengths of the items
  int64_t item_carry = 0, float_carry = 0;
  for (int base = 0; base < n_segs; base += kThreads) {
    const int i = base + tid;
    int items = 0;
    int64_t floats = 0;
    Segment s;
    s.npos = 0;
    if (i < n_segs) s = p.segs[i];
    if (s.npos > 0) {
      s.chunks = (s.t1 - s.t0 + chunk - 1) / chunk;
      items = s.units * s.chunks * p.Hkv;
      if (s.chunks > 1 || s.pbase == 0) {
        s.part_h = s.chunks * ((s.units - 1) * slot_floats(R, p.D) + slot_floats(s.npos * g - (s.units - 1) * R, p.D));
        floats = (int64_t)s.part_h * p.Hkv;
      }
    }
    int ti;
    int64_t tf;
    const int ii = scan_incl<int>(items, s_iscan[2], &ti);
    const int64_t fi = scan_incl<int64_t>(floats, s_scan[0], &tf);
    if (i < n_segs) {
      if (s.npos > 0 && (item_carry + ii > p.max_items || float_carry + fi > p.partial_cap)) {
        // cannot happen with the host's bounds; refuse rather than overflow
        report(p.status, WISP_DEV_UNSUPPORTED, p.request_ids, s.r);
        s.npos = s.units = s.chunks = 0;
      }
      s.pbase = floats > 0 ? (int32_t)(float_carry + fi - floats) : -1;
      if (s.npos > 0 && floats > 0) s_any = 1;
      s.first = (int32_t)(item_carry + ii - items);
      if (s.npos > 0 || i >= p.B) p.segs[i] = s;
    }
    item_carry += ti;
    float_carry += tf;
    __syncthreads();
  }
  const int n_all = (int)min(item_carry, p.max_items);

  // passes 4 and 5: the histogram of the items' lengths, then each item at its place in the dispatch order
  auto bucket_of = [&](int tokens) { return kBuckets - 1 - min(ceil_div(tokens, 64), kBuckets - 1); };
  for (int pass = 0; pass < 2; ++pass) {
    for (int base = 0; base < n_segs; base += kThreads) {
      const int i = base + tid;
      s_first[tid] = i < n_segs ? p.segs[i].first : n_all;
      if (tid == 0) s_first[kThreads] = base + kThreads < n_segs ? p.segs[base + kThreads].first : n_all;
      __syncthreads();
      const int lo = s_first[0], hi = min(s_first[kThreads], n_all);
      for (int x = lo + tid; x < hi; x += kThreads) {
        int a = 0, b = min(kThreads, n_segs - base) - 1;  // the last segment whose first item is <= x
        while (a < b) {
          const int mid = (a + b + 1) >> 1;
          if (s_first[mid] <= x) a = mid;
          else b = mid - 1;
        }
        const Segment s = p.segs[base + a];
        if (s.units <= 0) continue;
        const int rel = x - s.first, per_h = s.units * s.chunks;
        const int h = rel / per_h, u = rel % per_h / s.chunks, c = rel % s.chunks;
        if (h >= p.Hkv) continue;
        const int t0 = s.t0 + c * chunk, t1 = (int)min((int64_t)unit_end(s, u, R, g), (int64_t)t0 + chunk);
        if (t1 <= t0) continue;  // (the unit ends before this chunk)
        const int bucket = bucket_of(t1 - t0);
        if (pass == 0) {
          atomicAdd(&s_hist[bucket], 1);
          continue;
        }
        const int rows = min(R, s.npos * g - u * R);
        WorkItem w;
        w.r = s.r;
        w.h = h;
        w.t0 = t0;
        w.t1 = t1;
        w.rows = rows;
        w.q0 = s.q0;
        w.ctx = s.ctx;
        w.row0 = u * R;
        w.rg = u;
        w.nrg = s.units;
        w.poff = -1;
        w.pbase = 0;
        if (s.pbase >= 0) {
          w.pbase = s.pbase + h * s.part_h + u * s.chunks * slot_floats(R, p.D);
          w.poff = w.pbase + c * slot_floats(rows, p.D);
        }
        p.items[atomicAdd(&s_hist[bucket], 1)] = w;
      }
      __syncthreads();
    }
    if (pass == 0) {
      const int n = s_hist[tid];
      int total;
      const int at = scan_incl<int>(n, s_iscan[3], &total) - n;
      __syncthreads();
      s_hist[tid] = at;
      if (tid == 0) {
        PromptHeader hd;
        memset(&hd, 0, sizeof hd);
        hd.h.n_items = total;
        hd.h.chunk_len = chunk;
        hd.h.attn_ctas = p.sms;
        hd.partials = s_any;
        hd.n_runs = n_runs;
        hd.chunk = chunk;
        *p.header = hd;
      }
      __syncthreads();
    }
  }
}

// The partials of a row joined: O = sum_i O_i 2^(m_i - m) / sum_i l_i 2^(m_i - m), m = max m_i.  A CTA takes a query row, its
// warps take the heads in turn.  Bound by the partials' bytes.
template <int D, typename T>
__global__ void __launch_bounds__(kMergeThreads) prompt_merge_kernel(const PromptPlan p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (!p.header->partials) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int g = p.Hq / p.Hkv, R = p.unit_rows, chunk = p.header->chunk;
  constexpr int CPL = D / 32;
  for (int t = blockIdx.x; t < p.total_q_rows; t += gridDim.x) {
    int a = 0, b = p.B - 1;  // the row's request
    while (a < b) {
      const int mid = (a + b + 1) >> 1;
      if (p.q_row_start[mid] <= t) a = mid;
      else b = mid - 1;
    }
    if (p.req_flag[a] != REQ_OK || t >= p.q_row_start[a + 1]) continue;
    const int run = p.req_run[a];
    Segment s[2];
    s[0] = p.segs[a];
    if (run >= 0) s[1] = p.segs[p.B + run];
    const int n_seg = run >= 0 ? 2 : 1;
    if (s[0].pbase < 0) continue;  // (its items have written the output)
    for (int h = warp; h < p.Hq; h += kMergeThreads / 32) {
      const int hk = h / g, hh = h % g;
      // per segment: the row's first slot (O, and its m), the distance of slots and how many
      const float *po[2], *pm[2];
      int step[2], n[2], nl[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        n[i] = 0;
        if (i >= n_seg) continue;
        const int rho = (t - s[i].q0) * g + hh, u = rho / R, rr = rho - u * R;
        const int rows = min(R, s[i].npos * g - u * R);
        step[i] = slot_floats(rows, D);
        nl[i] = rows;
        n[i] = min(s[i].chunks, (unit_end(s[i], u, R, g) - s[i].t0 + chunk - 1) / chunk);
        const float *base = p.partials + (s[i].pbase + hk * s[i].part_h + u * s[i].chunks * slot_floats(R, D));
        po[i] = base + rr * D;
        pm[i] = base + rows * D + rr;
      }
      const int total = n[0] + n[1];
      float m = -INFINITY;
      for (int c = lane; c < total; c += 32) {
        const bool z = c < n[0];
        m = fmaxf(m, __ldcg(z ? pm[0] + c * step[0] : pm[1] + (c - n[0]) * step[1]));
      }
      m = ptx::warp_max(m);
      float den = 0.0f, acc[CPL];
#pragma unroll
      for (int q = 0; q < CPL; ++q) acc[q] = 0.0f;
      for (int c0 = 0; c0 < total; c0 += 32) {
        float w = -1.0f;
        if (c0 + lane < total) {
          const int c = c0 + lane;
          const bool z = c < n[0];
          const float *q = z ? pm[0] + c * step[0] : pm[1] + (c - n[0]) * step[1];
          const float mc = __ldcg(q), lc = __ldcg(q + (z ? nl[0] : nl[1]));
          if (mc != -INFINITY) {
            w = ptx::ex2(mc - m);
            den = fmaf(lc, w, den);
          } else if (lc != 0.0f) {
            den = lc;  // (a NaN: a score that is no number)
          }
        }
        const int nc = min(32, total - c0);
#pragma unroll 4
        for (int c = 0; c < nc; ++c) {
          const float x = __shfl_sync(0xffffffffu, w, c);
          const bool z = c0 + c < n[0];
          float v[CPL];
          ld_cols<CPL>((z ? po[0] + (c0 + c) * step[0] : po[1] + (c0 + c - n[0]) * step[1]) + lane * CPL, v);
          // (a chunk none of whose keys the row sees adds nothing)
#pragma unroll
          for (int q = 0; q < CPL; ++q)
            if (!(x < 0.0f)) acc[q] = fmaf(v[q], x, acc[q]);
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
      st_cols<CPL>(static_cast<T *>(p.out) + ((int64_t)t * p.Hq + h) * D + lane * CPL, acc, 1.0f / den);
    }
  }
}

cudaError_t prompt_plan_launch(const PromptPlan &p, cudaStream_t s) {
  prompt_plan_kernel<<<1, kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t prompt_merge_launch(const PromptPlan &p, bool f32, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  const int most = p.sms * 16;
  cfg.gridDim = dim3((unsigned)(p.total_q_rows < most ? p.total_q_rows : most));
  cfg.blockDim = dim3(kMergeThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (f32) return cudaLaunchKernelEx(&cfg, p.D == 128 ? prompt_merge_kernel<128, float> : prompt_merge_kernel<64, float>, p);
  return cudaLaunchKernelEx(&cfg, p.D == 128 ? prompt_merge_kernel<128, uint16_t> : prompt_merge_kernel<64, uint16_t>, p);
}

}  // namespace wisp
