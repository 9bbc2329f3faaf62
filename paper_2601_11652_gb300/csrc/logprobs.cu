// logprobs.cu -- log probabilities of given tokens with the rows' entropies and top alternatives
// (include/wisp_logprobs.h), and the tokens that a verified batch committed.
//
// One pass over a row, which a cluster of one to eight CTAs shares (rows are few when a server answers a step, and one
// CTA alone would take a row's length at its own rate).  A thread keeps a reference r near the largest logit it has seen and
// sums s = sum exp(z - r) and w = sum exp(z - r) (z - r) in fp32; the reference moves only when a logit is kLazy above it,
// and pairs (r, s, w) join over threads, warps and CTAs:
//   to a reference m >= r:  s' = s f,  w' = (w + s (r - m)) f,  f = exp(r - m);   log p(y) = z_y - m - log s,
//   entropy = log s - w / s.
// Alternatives: the pass only leaves the maximum of each stretch of a thread's loads (32 bf16 or 16 fp32 logits of a vocabulary of
// 128K) in a table.  A logit that n stretches are known to reach follows from the warps' largest maxima, and only stretches
// that reach it, a few dozen, are read again (from L2) for their tokens: a test of every logit in the pass took 13 times the
// time of the pass itself.  Tokens are 64-bit keys, the logit's bits in an order-preserving form above the inverted id, so that a
// larger key is a better token and ties need no care; lists of keys are cut to the best n whenever they fill.
#include "common.cuh"
#include "sm100_ptx.cuh"
#include "wisp_logprobs.h"

#include <cmath>
#include <cstring>

namespace wisp {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kVecs = 4;             // 16-byte loads in flight per thread
constexpr int kMaxTop = 32;
constexpr int kList = 32 + 8 * 32;   // a warp's keys: the best so far and one load of every lane
constexpr int kTable = 16;           // stretches per thread at most
constexpr int kCutAt = 96;           // lists longer than this are cut at the next opportunity
constexpr int kFew = kThreads;       // so many keys are put in order by counting; more (many equal logits) go through the warps' lists
constexpr int kMaxCluster = 8;
constexpr float kLazy = 20.0f;       // a logit this far above the reference moves it
constexpr float kLeast = -200.0f;    // exp of it and of anything below is 0
constexpr int kTokThreads = 1024;

struct LogprobParams {
  int rows, V, top_n, cluster;
  int64_t stride;
  const void *logits;
  const int32_t *tokens;
  float *logprob, *entropy, *top_logprobs;
  int32_t *top_tokens;
  DeviceStatus *status;
};

__device__ __forceinline__ float element(const uint16_t *row, int i) { return bf16_bits_to_float(__ldg(row + i)); }
__device__ __forceinline__ float element(const float *row, int i) { return __ldg(row + i); }

// Keys that order tokens by falling logit, the lower id first: larger is better.  No key is 0 (ids are below 2^24).
__device__ __forceinline__ uint64_t key_of(float z, int id) {
  const uint32_t b = __float_as_uint(z + 0.0f);  // (-0 counts as 0)
  const uint32_t o = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)o << 32 | (0xffffffffu - (uint32_t)id);
}
// A logit as an integer of the same order.
__device__ __forceinline__ int order_of(float z) {
  const int b = __float_as_int(z + 0.0f);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ int id_of(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

__global__ void status_clear_kernel(DeviceStatus *st) {
  // the row kernel may start: it reports errors only after this grid is done
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  st->code = 0;
  st->pad = 0;
  st->request_id = 0;
}
__device__ __forceinline__ void report_row(DeviceStatus *st, int code, int row) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  report(st, code, nullptr, row);
}

__device__ __forceinline__ float max_nan(float a, float b) {  // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint32_t max_nan2(uint32_t a, uint32_t b) {  // of bf16 pairs
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// A thread's share of a row, then a warp's, a CTA's.
struct Stat {
  float r, s, w;
};
// `a` and `b` against the larger of their references.  (A reference of -inf: nothing so far.)
__device__ __forceinline__ Stat join(Stat a, Stat b) {
  const float m = max_nan(a.r, b.r);
  const float da = a.r - m, db = b.r - m;
  const float fa = a.r == -INFINITY ? 0.0f : ex2_approx(da * kLog2e), fb = b.r == -INFINITY ? 0.0f : ex2_approx(db * kLog2e);
  Stat c;
  c.r = m;
  c.s = a.s * fa + b.s * fb;
  c.w = (fa == 0.0f ? 0.0f : (a.w + a.s * da) * fa) + (fb == 0.0f ? 0.0f : (b.w + b.s * db) * fb);
  return c;
}

// Elements of a 16-byte load: 8 bf16 or 4 fp32.
template <typename T>
struct Vec {
  static constexpr int E = sizeof(T) == 2 ? 8 : 4;
  uint4 v;
  __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
  __device__ __forceinline__ float at(int i) const {
    if (E == 4) return __uint_as_float(word(i));
    return __uint_as_float(i & 1 ? word(i >> 1) & 0xffff0000u : word(i >> 1) << 16);
  }
  __device__ __forceinline__ void clear() {  // -inf throughout
    const uint32_t x = E == 4 ? 0xff800000u : 0xff80ff80u;
    v = make_uint4(x, x, x, x);
  }
};
template <typename T>
__device__ __forceinline__ float max_of(const Vec<T> (&x)[kVecs]) {
  if (Vec<T>::E == 8) {
    uint32_t m = x[0].v.x;
#pragma unroll
    for (int u = 0; u < kVecs; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) m = max_nan2(m, x[u].word(i));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  float m = x[0].at(0);
#pragma unroll
  for (int u = 0; u < kVecs; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) m = max_nan(m, x[u].at(i));
  return m;
}

__device__ __forceinline__ uint64_t shfl_xor64(uint64_t v, int m) { return __shfl_xor_sync(0xffffffffu, v, m); }
// The 32 lanes' keys in falling order (lane 0 gets the largest): bitonic sort.
__device__ __forceinline__ uint64_t warp_sort(uint64_t k, int lane) {
#pragma unroll 1
  for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll 1
    for (int d = size >> 1; d > 0; d >>= 1) {
      const uint64_t o = shfl_xor64(k, d);
      const bool keep_max = ((lane & d) == 0) == ((lane & size) == 0);
      k = keep_max ? max(k, o) : min(k, o);
    }
  }
  return k;
}
// The 32 largest of two sorted sets of 32, sorted.
__device__ __forceinline__ uint64_t warp_merge(uint64_t a, uint64_t b, int lane) {
  uint64_t k = max(a, __shfl_sync(0xffffffffu, b, 31 - lane));
#pragma unroll 1
  for (int d = 16; d > 0; d >>= 1) {
    const uint64_t o = shfl_xor64(k, d);
    k = (lane & d) == 0 ? max(k, o) : min(k, o);
  }
  return k;
}

// A warp's list of candidate keys.
struct List {
  uint64_t *keys;  // [kList]
  int count;
  int top_n;
  // the best min(count, 32) keys, sorted, one per lane (0: none)
  __device__ uint64_t best(int lane) const {
    uint64_t k = 0;
    for (int at = 0; at < count; at += 32) k = warp_merge(k, warp_sort(at + lane < count ? keys[at + lane] : 0, lane), lane);
    return k;
  }
  // cut to the best top_n; *threshold rises to the last of them
  __device__ void cut(int lane, unsigned long long *threshold) {
    __syncwarp();
    const uint64_t k = best(lane);
    __syncwarp();
    if (lane < top_n) keys[lane] = k;
    count = min(count, top_n);
    const uint64_t last = __shfl_sync(0xffffffffu, k, top_n - 1);
    if (lane == 0 && last > *threshold) atomicMax(threshold, (unsigned long long)last);
    __syncwarp();
  }
};

// The keys of a thread's loads above the threshold, into the warp's list.  id0(u): id of load u's first element.
template <typename T, typename Id>
__device__ void collect(const Vec<T> (&x)[kVecs], Id id0, List &list, unsigned long long *threshold, int lane) {
  constexpr int E = Vec<T>::E;
  uint64_t thr = *(volatile unsigned long long *)threshold;
  auto key = [&](int u, int i) -> uint64_t {
    const float z = x[u].at(i);
    return z > -INFINITY ? key_of(z, id0(u) + i) : 0;
  };
  // many at once (the first loads, or logits that rise along the row): the threshold rises to the top_n-th of the
  // lanes' largest first
  uint64_t mine = 0;
  int n = 0;
#pragma unroll
  for (int u = 0; u < kVecs; ++u)
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const uint64_t k = key(u, i);
      mine = max(mine, k);
      n += k > thr;
    }
  if (__reduce_add_sync(0xffffffffu, n) > 64) {
    const uint64_t t = __shfl_sync(0xffffffffu, warp_sort(mine, lane), list.top_n - 1);
    if (t > thr) {
      thr = t - 1;  // (that key itself is to be kept)
      if (lane == 0) atomicMax(threshold, (unsigned long long)thr);
    }
  }
#pragma unroll
  for (int u = 0; u < kVecs; ++u) {
    for (;;) {
      int c = 0;
#pragma unroll
      for (int i = 0; i < E; ++i) c += key(u, i) > thr;
      int before = c;
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += o;
      }
      const int total = __shfl_sync(0xffffffffu, before, 31);
      if (total == 0) break;
      if (list.count + total > kList) {
        list.cut(lane, threshold);
        thr = max(thr, (uint64_t)*(volatile unsigned long long *)threshold);
        continue;
      }
      int at = list.count + before - c;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const uint64_t k = key(u, i);
        if (k > thr) list.keys[at++] = k;
      }
      list.count += total;
      break;
    }
  }
  if (list.count > kCutAt) list.cut(lane, threshold);
}

struct Shared {
  Stat stat[kWarps];
  int found, pushed;                    // stretches to read again, keys found in them
  int floor;                            // the logit that they reach, in the form of order_of
  uint64_t best[kMaxCluster][kMaxTop];  // the first CTA's: the CTAs' alternatives
  Stat part[kMaxCluster];               // the first CTA's: the CTAs' sums
  unsigned long long threshold;
};

// The address of the same shared-memory object in the cluster's CTA `rank`.
template <typename P>
__device__ __forceinline__ uint32_t remote(P *p, uint32_t rank) {
  uint32_t r;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(ptx::smem_u32(p)), "r"(rank));
  return r;
}

// A cluster per row.  What bounds it: with many rows the logits' bytes (2432 rows of 128K bf16: 92 us at the copy rate) and, close
// behind, the instructions, about five an element and half as many around it; with few the way through a CTA's loads and
// barriers, of which the alternatives have eight more.  Measured, bf16 rows of 128K, without alternatives / with the top 5: 2432 rows
// 104 / 120 us (6.0, 5.2 TB/s), 176 rows 13.0 / 18.3, one row 9.3 / 10.4; 1200 fp32 rows 93 / 106 us (6.6, 5.8 TB/s).  (2432 rows
// with the top 5: 134 us at 80 registers a thread, three CTAs on an SM and not four; 130 with the next round's loads copied into the
// present ones and not taken in turn.  A reference in log2 units, one multiply-add for a difference and a product, gained 1%.)
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads, TOP ? 4 : 5) logprobs_kernel(const LogprobParams p) {
  constexpr int E = Vec<T>::E;
  __shared__ Shared sh;
  __shared__ uint64_t s_list[TOP ? kWarps * kList : 1];
  __shared__ float s_max[TOP ? kTable * kThreads : 1];       // the stretches' maxima
  __shared__ uint16_t s_again[TOP ? kTable * kThreads : 1];  // those to be read again
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int csize = p.cluster, row = blockIdx.x / csize, rank = blockIdx.x % csize;
  const int tok = p.tokens[row];
  const T *z = static_cast<const T *>(p.logits) + (int64_t)row * p.stride;
  auto write_all = [&](float v, int id) {
    if (rank != 0) return;
    if (tid == 0) {
      p.logprob[row] = v;
      if (p.entropy) p.entropy[row] = v;
    }
    if (tid < p.top_n) {
      p.top_tokens[(int64_t)row * p.top_n + tid] = id;
      p.top_logprobs[(int64_t)row * p.top_n + tid] = v;
    }
  };
  if (tok < 0) return write_all(0.0f, -1);  // (the same for the whole cluster)
  if (tok >= p.V) {
    if (tid == 0 && rank == 0) report_row(p.status, WISP_DEV_BAD_TOKEN, row);
    return write_all(NAN, -1);
  }
  // a CTA's shared memory is written by others only once it runs
  if (csize > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  const float zt = rank == 0 && tid == 0 ? element(z, tok) : 0.0f;

  // the row's aligned loads [0, nvec), `head` elements before them and `tail` after
  const int head = min(p.V, (int)((16 - ((uintptr_t)z & 15)) & 15) / (int)sizeof(T));
  const int nvec = (p.V - head) / E, tail = p.V - head - nvec * E;
  const uint4 *zv = reinterpret_cast<const uint4 *>(z + head);
  const int per = (nvec + csize - 1) / csize;
  const int v0 = min(nvec, rank * per), v1 = min(nvec, v0 + per);

  Stat st = {-INFINITY, 0.0f, 0.0f};
  float2 s2 = make_float2(0.0f, 0.0f), w2 = s2;
  // a thread's round of loads is a stretch, or several rounds are where the table has not room for all
  constexpr int kRound = kThreads * kVecs;
  const int rounds = (v1 - v0 + kRound - 1) / kRound, span = (rounds + kTable - 1) / kTable;

  auto take = [&](const Vec<T> (&x)[kVecs]) -> float {
    const float cm = max_of<T>(x);
    if (cm != -INFINITY) {
      if (!(cm <= st.r + kLazy)) {  // (a NaN too: it stays)
        if (st.r == -INFINITY) {
          st.r = cm;
        } else {
          const float d = st.r - cm, f = ex2_approx(d * kLog2e);
          // (f = 0: d may be past what a product holds)
          w2 = f == 0.0f ? make_float2(0.0f, 0.0f) : make_float2((w2.x + s2.x * d) * f, (w2.y + s2.y * d) * f);
          s2 = make_float2(s2.x * f, s2.y * f);
          st.r = cm;
        }
      }
      const float2 mr = make_float2(-st.r, -st.r), l2e = make_float2(kLog2e, kLog2e);
#pragma unroll
      for (int u = 0; u < kVecs; ++u) {
#pragma unroll
        for (int i = 0; i < E; i += 2) {
          float2 d = __fadd2_rn(make_float2(x[u].at(i), x[u].at(i + 1)), mr);
          d = make_float2(fmaxf(d.x, kLeast), fmaxf(d.y, kLeast));
          const float2 t = __fmul2_rn(d, l2e);
          const float2 e = make_float2(ex2_approx(t.x), ex2_approx(t.y));
          s2 = __fadd2_rn(s2, e);
          w2 = __ffma2_rn(e, d, w2);
        }
      }
    }
    if (cm != cm) s2.x = NAN;
    return cm;
  };

  Vec<T> cur[kVecs], nxt[kVecs];
  auto load = [&](int base, Vec<T> (&x)[kVecs]) {
#pragma unroll
    for (int u = 0; u < kVecs; ++u) {
      const int i = base + u * kThreads + tid;
      if (i < v1)
        x[u].v = __ldg(zv + i);
      else
        x[u].clear();
    }
  };
  if (v0 < v1) load(v0, cur);
  float most = -INFINITY;
  int slot = 0, left = span;
  float stretch = -INFINITY;
  auto round = [&](int base, Vec<T> (&now)[kVecs], Vec<T> (&then)[kVecs]) {
    if (base + kRound < v1) load(base + kRound, then);
    const float cm = take(now);
    if (TOP) {
      stretch = fmaxf(stretch, cm);
      most = fmaxf(most, cm);
      if (--left == 0 || base + kRound >= v1) {
        s_max[slot++ * kThreads + tid] = stretch;
        stretch = -INFINITY;
        left = span;
      }
    }
  };
  for (int base = v0; base < v1; base += 2 * kRound) {
    round(base, cur, nxt);
    if (base + kRound < v1) round(base + kRound, nxt, cur);
  }
  const bool edges = rank == 0 && warp == 0 && head + tail > 0;
  const int edge_id = lane < head ? lane : head + nvec * E + lane - head;
  if (edges) {  // the elements around the aligned loads, one per lane
#pragma unroll
    for (int u = 0; u < kVecs; ++u) cur[u].clear();
    if (lane < head + tail) {
      const float v = element(z, edge_id);
      if (E == 4)
        cur[0].v.x = __float_as_uint(v);
      else
        cur[0].v.x = (cur[0].v.x & 0xffff0000u) | __float_as_uint(v) >> 16;
    }
    take(cur);
  }

  st.s = s2.x + s2.y;
  st.w = w2.x + w2.y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    Stat b;
    b.r = __shfl_xor_sync(0xffffffffu, st.r, o);
    b.s = __shfl_xor_sync(0xffffffffu, st.s, o);
    b.w = __shfl_xor_sync(0xffffffffu, st.w, o);
    st = join(st, b);
  }
  if (lane == 0) sh.stat[warp] = st;
  uint64_t best = 0;
  if (TOP) {
    // at least top_n threads' maxima reach the least of the warps' q-th largest, q = top_n / 8 rounded up
    int o = order_of(most), least = 0;
    for (int i = 0; i < (p.top_n + kWarps - 1) / kWarps; ++i) {
      least = __reduce_max_sync(0xffffffffu, o);
      if (lane == __ffs(__ballot_sync(0xffffffffu, o == least)) - 1) o = INT32_MIN;
    }
    if (tid == 0) {
      sh.found = sh.pushed = 0;
      sh.floor = INT32_MAX;
    }
    if (warp == 0) sh.best[0][lane] = 0;
    auto push = [&](uint64_t k) {
      const int i = atomicAdd(&sh.pushed, 1);
      if (i < kFew) s_list[i] = k;
    };
    __syncthreads();
    if (lane == 0) atomicMin(&sh.floor, least);
    __syncthreads();
    const int floor = max(sh.floor, order_of(-3.402823466e38f));  // (stretches of -inf: nothing to find)
    for (int i = 0; i < slot; ++i)
      if (order_of(s_max[i * kThreads + tid]) >= floor) s_again[atomicAdd(&sh.found, 1)] = (uint16_t)(i * kThreads + tid);
    if (tid == 0) sh.threshold = ((unsigned long long)((uint32_t)floor ^ 0x80000000u) << 32) - 1;
    __syncthreads();
    // their tokens: a load of a stretch per thread, and the keys that reach the floor into one list
    const int found = sh.found;
    for (int i = tid; i < found * kVecs * span; i += kThreads) {
      const int e = s_again[i / (kVecs * span)], u = i % kVecs, r = i / kVecs % span;
      const int at = v0 + (e / kThreads * span + r) * kRound + u * kThreads + e % kThreads;
      if (at < v1) {
        Vec<T> x;
        x.v = __ldg(zv + at);
#pragma unroll
        for (int q = 0; q < E; ++q)
          if (order_of(x.at(q)) >= floor) push(key_of(x.at(q), head + at * E + q));
      }
    }
    if (edges && lane < head + tail) {
      const float v = element(z, edge_id);
      if (order_of(v) >= floor) push(key_of(v, edge_id));
    }
    __syncthreads();
    const int pushed = sh.pushed;
    if (pushed <= kFew) {
      // a key's place is the number of larger ones
      if (tid < pushed) {
        const uint64_t k = s_list[tid];
        int place = 0;
        for (int i = 0; i < pushed; ++i) place += s_list[i] > k;
        if (place < kMaxTop) sh.best[0][place] = k;
      }
      __syncthreads();
      best = warp == 0 ? sh.best[0][lane] : 0;
    } else {
      List list;
      list.keys = s_list + warp * kList;
      list.count = 0;
      list.top_n = p.top_n;
      for (int at = warp * 32; at < found; at += kThreads) {
        const int e = at + lane < found ? s_again[at + lane] : -1;
        for (int r = 0; r < span; ++r) {
          const int first = e < 0 ? v1 : v0 + (e / kThreads * span + r) * kRound + e % kThreads;
#pragma unroll
          for (int u = 0; u < kVecs; ++u) {
            if (first + u * kThreads < v1)
              cur[u].v = __ldg(zv + first + u * kThreads);
            else
              cur[u].clear();
          }
          collect<T>(cur, [&](int u) { return head + (first + u * kThreads) * E; }, list, &sh.threshold, lane);
        }
      }
      if (edges) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) cur[u].clear();
        if (lane < head + tail) {
          const float v = element(z, edge_id);
          if (E == 4)
            cur[0].v.x = __float_as_uint(v);
          else
            cur[0].v.x = (cur[0].v.x & 0xffff0000u) | __float_as_uint(v) >> 16;
        }
        collect<T>(cur, [&](int u) { return edge_id + u; }, list, &sh.threshold, lane);
      }
      best = list.best(lane);
      __syncwarp();
      list.keys[lane] = best;
      __syncthreads();
      if (warp == 0)
        for (int w = 1; w < kWarps; ++w) best = warp_merge(best, s_list[w * kList + lane], lane);
    }
  }
  __syncthreads();
  if (csize > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (warp == 0) {
    st = sh.stat[lane & (kWarps - 1)];
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) {
      Stat b;
      b.r = __shfl_xor_sync(0xffffffffu, st.r, o);
      b.s = __shfl_xor_sync(0xffffffffu, st.s, o);
      b.w = __shfl_xor_sync(0xffffffffu, st.w, o);
      st = join(st, b);
    }
    if (csize > 1) {  // to the first CTA
      if (TOP) {
        const uint32_t at = remote(&sh.best[rank][lane], 0);
        asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(at), "l"(best) : "memory");
      }
      if (lane == 0) {
        const uint32_t at = remote(&sh.part[rank], 0);
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(st.r) : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(st.s) : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(st.w) : "memory");
      }
    }
  }
  if (csize > 1) {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (rank != 0 || warp != 0) return;
  for (int c = 1; c < csize; ++c) {
    st = join(st, sh.part[c]);
    if (TOP) best = warp_merge(best, sh.best[c][lane], lane);
  }
  const bool bad = !(st.r > -INFINITY && st.r < INFINITY && st.s > 0.0f && st.s < INFINITY);
  if (bad) {
    if (lane == 0) report_row(p.status, WISP_DEV_BAD_PROB, row);
    return write_all(NAN, -1);
  }
  const float ls = logf(st.s);
  if (lane == 0) {
    p.logprob[row] = zt - st.r - ls;
    if (p.entropy) p.entropy[row] = ls - st.w / st.s;
  }
  if (TOP) {
    // fewer than top_n logits above -inf: tokens at -inf follow, by their ids; among the first 64 there are enough
    const unsigned have = __ballot_sync(0xffffffffu, best != 0);
    int id = best ? id_of(best) : -1;
    float lp = best ? logit_of(best) - st.r - ls : -INFINITY;
    const int n = __popc(have);
    if (n < p.top_n) {
      int found = n;
      for (int i = 0; i < min(p.V, 2 * kMaxTop) && found < p.top_n; ++i) {
        if (element(z, i) == -INFINITY) {
          if (lane == found) id = i;
          ++found;
        }
      }
    }
    if (lane < p.top_n) {
      p.top_tokens[(int64_t)row * p.top_n + lane] = id;
      p.top_logprobs[(int64_t)row * p.top_n + lane] = lp;
    }
  }
}

// One CTA: a request's rows start at the sum of the lengths before it, found by a scan; then a warp per request.
__global__ void __launch_bounds__(kTokThreads) committed_kernel(int B, int total_rows, int total_draft, const int32_t *draft_lens,
                                                                const int32_t *draft_tokens, const int32_t *accepted_len,
                                                                const int32_t *next_token, int32_t *row_tokens) {
  __shared__ int64_t s_w[32], s_d0[kTokThreads];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int64_t carry = 0;
  for (int base = 0; base < B; base += kTokThreads) {
    const int64_t k = base + tid < B ? max(0, draft_lens[base + tid]) : 0;
    int64_t x = k;
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, x, d);
      if (lane >= d) x += o;
    }
    if (lane == 31) s_w[warp] = x;
    __syncthreads();
    int64_t t = s_w[lane];
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xffffffffu, t, d);
      if (lane >= d) t += o;
    }
    const int64_t before = __shfl_sync(0xffffffffu, t, (warp + 31) & 31), total = __shfl_sync(0xffffffffu, t, 31);
    s_d0[tid] = carry + x - k + (warp > 0 ? before : 0);
    __syncthreads();
    for (int i = warp; i < min(kTokThreads, B - base); i += kTokThreads / 32) {
      const int r = base + i, kr = max(0, draft_lens[r]), L = accepted_len[r], nt = next_token[r];
      const int64_t d0 = s_d0[i], q0 = d0 + r;
      const bool ok = draft_lens[r] >= 0 && L >= 0 && L <= kr;
      for (int j = lane; j <= kr && q0 + j < total_rows; j += 32)
        row_tokens[q0 + j] = !ok || j > L ? -1 : j == L ? nt : d0 + j < total_draft ? draft_tokens[d0 + j] : -1;
    }
    carry += total;
    __syncthreads();
  }
  for (int64_t j = carry + B + tid; j < total_rows; j += kTokThreads) row_tokens[j] = -1;
}

wisp_status check(const wisp_logprobs_args *a) {
  if (!a) return WISP_ERR_INVALID_ARG;
  if (a->rows < 0 || a->V <= 0 || a->top_n < 0) return WISP_ERR_INVALID_ARG;
  if (a->logits_dtype != WISP_F32 && a->logits_dtype != WISP_BF16) return WISP_ERR_INVALID_ARG;
  if (a->row_stride != 0 && a->row_stride < a->V) return WISP_ERR_INVALID_ARG;
  if (a->row_stride > INT64_MAX / 4 / (a->rows > 0 ? a->rows : 1)) return WISP_ERR_INVALID_ARG;  // (byte offsets in 64 bits)
  if (a->V > (1 << 24) || a->top_n > kMaxTop) return WISP_ERR_UNSUPPORTED;
  if (a->rows == 0) return WISP_OK;
  if (!a->logits || !a->tokens || !a->logprob) return WISP_ERR_INVALID_ARG;
  if ((uintptr_t)a->logits % (a->logits_dtype == WISP_BF16 ? 2 : 4) != 0) return WISP_ERR_INVALID_ARG;
  if (a->top_n > 0 && (!a->top_tokens || !a->top_logprobs)) return WISP_ERR_INVALID_ARG;
  return WISP_OK;
}

}  // namespace

}  // namespace wisp

using namespace wisp;

extern "C" {

size_t wisp_verify_logprobs_workspace_size(const wisp_logprobs_args *a) { return check(a) == WISP_OK ? 256 : 0; }

wisp_status wisp_verify_logprobs(const wisp_logprobs_args *a, void *ws, size_t ws_bytes, void *stream) {
  const wisp_status st = check(a);
  if (st != WISP_OK) return st;
  if (!ws || ((uintptr_t)ws & 255) != 0 || ws_bytes < 256) return WISP_ERR_WORKSPACE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  LogprobParams p;
  std::memset(&p, 0, sizeof p);
  p.rows = a->rows;
  p.V = a->V;
  p.top_n = a->top_n;
  p.stride = a->row_stride ? a->row_stride : a->V;
  p.logits = a->logits;
  p.tokens = a->tokens;
  p.logprob = a->logprob;
  p.entropy = a->entropy;
  p.top_tokens = a->top_tokens;
  p.top_logprobs = a->top_logprobs;
  p.status = static_cast<DeviceStatus *>(ws);
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return WISP_ERR_CUDA;
  status_clear_kernel<<<1, 1, 0, s>>>(p.status);
  if (cudaGetLastError() != cudaSuccess) return WISP_ERR_CUDA;
  if (a->rows == 0) return WISP_OK;
  const bool bf = a->logits_dtype == WISP_BF16, top = a->top_n > 0;
  // CTAs per row: as many as keep all CTAs within three per SM with alternatives (four fit; a CTA's later part, with few loads,
  // then has others beside it) and five without (as many fit), as long as each has a whole round of its threads' loads.  Rows of
  // 128K bf16 logits with top 5, for at least four per SM and for at most three: 110 rows 20.4, 14.9 us; 150 25.0, 16.6; 176
  // 21.0, 18.8; 400 33.3, 30.8.  Without alternatives, at most three and at most five: 176 rows 14.5, 12.8 us.
  const int64_t rounds = ((int64_t)a->V * (bf ? 2 : 4) / 16 + kThreads * kVecs - 1) / (kThreads * kVecs);
  p.cluster = 1;
  while (p.cluster < kMaxCluster && 2 * p.cluster <= rounds && (int64_t)a->rows * 2 * p.cluster <= (int64_t)(top ? 3 : 5) * sms) p.cluster *= 2;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)p.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3((unsigned)(a->rows * p.cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = bf ? (top ? cudaLaunchKernelEx(&cfg, logprobs_kernel<uint16_t, true>, p) : cudaLaunchKernelEx(&cfg, logprobs_kernel<uint16_t, false>, p))
                           : (top ? cudaLaunchKernelEx(&cfg, logprobs_kernel<float, true>, p) : cudaLaunchKernelEx(&cfg, logprobs_kernel<float, false>, p));
  return e == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
}

wisp_status wisp_verify_committed_tokens(const wisp_accept_args *c, int32_t *row_tokens, void *stream) {
  if (!c || c->B < 0 || c->total_draft < 0 || c->total_q_rows < c->B) return WISP_ERR_INVALID_ARG;
  if (c->total_q_rows == 0) return WISP_OK;
  if (!row_tokens) return WISP_ERR_INVALID_ARG;
  if (c->B > 0 && (!c->draft_lens || !c->accepted_len || !c->next_token || (c->total_draft > 0 && !c->draft_tokens)))
    return WISP_ERR_INVALID_ARG;
  committed_kernel<<<1, kTokThreads, 0, static_cast<cudaStream_t>(stream)>>>(
      c->B, c->total_q_rows, c->total_draft, c->draft_lens, c->draft_tokens, c->accepted_len, c->next_token, row_tokens);
  return cudaGetLastError() == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
}

}  // extern "C"
