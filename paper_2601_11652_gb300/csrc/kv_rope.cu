// kv_rope.cu -- new K/V rows into the paged cache with the position rotation applied on the way, and the
// rotated queries beside them (wisp_kv_reserve_append_rope).
//
// Pair (a, b) of a row at position t becomes (a cos - b sin, b cos + a sin) with the table's values for t; each
// product and each sum is rounded to fp32 by itself (no contraction), so that a cache written elsewhere from the same
// definition agrees to the bit.  Into a cache of the rows' type the result is rounded once.  Into an e4m3
// cache a page of one head gets the scale 2^e with the least e such that its largest live magnitude is at most
// 448 * 2^e: a page that is filled over several calls is decoded, and where the scale changes (it grows with a new
// row, or shrinks after a larger rejected row went) its earlier codes are written again.
// A power of two costs an e4m3 code at most its lowest subnormal bits and makes that rewriting exact but for them.
#include "fp8.cuh"
#include "kv.cuh"
#include "sm100_ptx.cuh"
#include "wisp_kv8.h"

#include <cstring>

namespace wisp {

namespace {

constexpr int kThreads = 128;
constexpr int kCtasPerSM = 8;

struct RopeParams {
  int Hq, rot8;          // queries' heads; rotated elements / 8
  int interleaved;
  int q_ctas;            // CTAs that rotate queries, the first ones
  int group;             // consecutive new rows per K/V unit of an e4m3 cache, at most 16
  const float *table;    // [positions, 8 * rot8]: cosines, then sines
  const char *q;
  char *q_out;
  int64_t q_stride, k_stride, v_stride;  // bytes between rows
  float *k_scale, *v_scale;
};

// 8 elements of one head's row per lane, as two groups of 4: those that rotate into each other (lanes
// below rot8), or two groups that pass.  (With 16 elements a lane, a page's rows took twice the registers and an SM half the warps.)
struct Groups {
  int a, b;  // first elements
  bool turn;
};
__device__ __forceinline__ Groups groups_of(int l, const RopeParams &o) {
  Groups g;
  g.turn = l < o.rot8;
  const bool split = g.turn && !o.interleaved;
  g.a = split ? 4 * l : 8 * l;
  g.b = split ? 4 * (l + o.rot8) : 8 * l + 4;
  return g;
}

// Four elements, as they are in memory.
template <typename T>
struct Four {
  uint32_t w[sizeof(T)];
  __device__ __forceinline__ void read(const T *src) {
    if (sizeof(T) == 2) {
      const uint2 v = *reinterpret_cast<const uint2 *>(src);
      w[0] = v.x;
      w[1] = v.y;
    } else {
      const uint4 v = *reinterpret_cast<const uint4 *>(src);
      w[0] = v.x;
      w[1] = v.y;
      w[sizeof(T) - 2] = v.z;
      w[sizeof(T) - 1] = v.w;
    }
  }
  __device__ __forceinline__ void get(float *x) const {
    if (sizeof(T) == 2) {
      x[0] = __uint_as_float(w[0] << 16);
      x[1] = __uint_as_float(w[0] & 0xffff0000u);
      x[2] = __uint_as_float(w[1] << 16);
      x[3] = __uint_as_float(w[1] & 0xffff0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i < (int)sizeof(T) ? i : 0]);
    }
  }
};
__device__ __forceinline__ void store4(uint16_t *dst, const float *x) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
  *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store4(float *dst, const float *x) { *reinterpret_cast<float4 *>(dst) = make_float4(x[0], x[1], x[2], x[3]); }

// A lane's 8 elements as they were read; floats only where they are used.
template <typename T>
struct Raw {
  Four<T> a, b;
  // (plain loads: queries may be rotated in place, and what a kernel writes is not read-only memory to it)
  __device__ __forceinline__ void read(const T *row, const Groups &g) {
    a.read(row + g.a);
    b.read(row + g.b);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    a.get(x);
    b.get(x + 4);
  }
};

// The lane's 4 cosines and 4 sines of a position.
struct Angles {
  float4 c, s;
};
__device__ __forceinline__ Angles load_angles(const RopeParams &o, int pos, int l, bool turn) {
  Angles t = {};
  if (turn) {
    const float4 *p = reinterpret_cast<const float4 *>(o.table + (int64_t)pos * 8 * o.rot8) + l;
    t.c = __ldg(p);
    t.s = __ldg(p + o.rot8);
  }
  return t;
}
__device__ __forceinline__ void turn_pair(float &a, float &b, float c, float s) {
  const float u = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = u;
}
// x rotated where `turn` says so.  (Selected, not branched around: the compiler would hold every row's floats over the branches.)
template <bool INTER>
__device__ __forceinline__ void rotate(float (&x)[8], const Angles &t, bool turn) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = x[i];
  if (INTER) {
    turn_pair(y[0], y[1], t.c.x, t.s.x);
    turn_pair(y[2], y[3], t.c.y, t.s.y);
    turn_pair(y[4], y[5], t.c.z, t.s.z);
    turn_pair(y[6], y[7], t.c.w, t.s.w);
  } else {
    turn_pair(y[0], y[4], t.c.x, t.s.x);
    turn_pair(y[1], y[5], t.c.y, t.s.y);
    turn_pair(y[2], y[6], t.c.z, t.s.z);
    turn_pair(y[3], y[7], t.c.w, t.s.w);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = turn ? y[i] : x[i];
}

// Heads per unit of whole rows: so many loads in flight.
template <typename T, int D>
constexpr int heads_per_unit() { return (sizeof(T) == 2 ? 8 : 4) * (32 / (D / 8)); }

// Heads [h0, h0 + heads_per_unit) of one row: src -> dst, rotated if `turn`.  dst heads are DST_HEAD elements apart.
// The loads come first, then `where` tells the row's destination (null: none) and position.
template <typename T, int D, bool INTER, int DST_HEAD, typename Where>
__device__ __forceinline__ void move_heads(const RopeParams &o, const T *src, int h0, int H, bool turn, Where where) {
  constexpr int LPR = D / 8, RPP = 32 / LPR, N = heads_per_unit<T, D>() / RPP;
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const Groups g = groups_of(l, o);
  const int h = h0 + lane / LPR, left = H - h;  // this lane's heads: h, h + RPP, ..
  src += (int64_t)h * D;
  Raw<T> raw[N] = {};
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i * RPP < left) raw[i].read(src + i * RPP * D, g);
  int pos = 0;
  T *dst = where(pos);
  if (!dst) return;
  dst += (int64_t)h * DST_HEAD;
  const bool turns = turn && g.turn;
  const Angles t = load_angles(o, pos, l, turns);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float x[8];
    raw[i].get(x);
    if (turn) rotate<INTER>(x, t, turns);
    if (i * RPP < left) {
      store4(dst + i * RPP * DST_HEAD + g.a, x);
      store4(dst + i * RPP * DST_HEAD + g.b, x + 4);
    }
  }
}

__device__ __forceinline__ void copy16(void *dst, const void *src) {  // global to shared, asynchronous
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(dst)), "l"(src) : "memory");
}

// One page of one head of an e4m3 cache, by one warp: slots s0 .. s0 + n - 1 are new rows (the first of them at src,
// at position pos), slots below s0 hold earlier ones.  The rows (of earlier ones the codes) are staged in shared memory and
// read twice, for the scale and for the codes: in registers they would leave an SM a third of its warps.
template <typename T, int D, bool INTER>
__device__ __forceinline__ void quantise_page(const RopeParams &o, T *stage, uint8_t *page, float *scale, const T *src,
                                              int64_t src_row, int s0, int n, int pos, bool turn) {
  constexpr int LPR = D / 8, RPP = 32 / LPR;       // a lane has 8 elements of a row
  constexpr int CPR = D * sizeof(T) / 16;          // 16-byte pieces of a row
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const Groups g = groups_of(l, o);
  const float old_scale = s0 > 0 ? *scale : 1.0f;
  __syncwarp();  // the page before has been read
  for (int c = lane; c < n * CPR; c += 32)
    copy16(stage + (s0 + c / CPR) * D + c % CPR * (16 / sizeof(T)),
           reinterpret_cast<const char *>(src) + (c / CPR) * src_row + c % CPR * 16);
  for (int c = lane; c < s0 * (D / 16); c += 32)
    copy16(reinterpret_cast<uint8_t *>(stage + c / (D / 16) * D) + c % (D / 16) * 16, page + c * 16);
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
  // the values of a slot below s0 + n
  auto values = [&](int slot, float (&x)[8]) {
    const T *row = stage + slot * D;
    if (slot < s0) {
      const uint8_t *codes = reinterpret_cast<const uint8_t *>(row);
      const uint32_t w[2] = {*reinterpret_cast<const uint32_t *>(codes + g.a), *reinterpret_cast<const uint32_t *>(codes + g.b)};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float2 v = h2_to_f2(e4m3x2_to_h2((w[q >> 1] >> (16 * (q & 1))) & 0xffffu));
        x[2 * q] = v.x * old_scale;
        x[2 * q + 1] = v.y * old_scale;
      }
    } else {
      Raw<T> raw;
      raw.read(row, g);
      raw.get(x);
      if (turn) rotate<INTER>(x, load_angles(o, pos + slot - s0, l, g.turn), g.turn);
    }
  };
  float amax = 0.0f;  // the largest finite magnitude
#pragma unroll 2
  for (int slot = lane / LPR; slot < s0 + n; slot += RPP) {
    float x[8];
    values(slot, x);
#pragma unroll
    for (int q = 0; q < 8; ++q) amax = fmaxf(amax, fabsf(x[q]) < INFINITY ? fabsf(x[q]) : 0.0f);
  }
  __syncwarp();
  const int e = scale_exp(ptx::warp_max(amax));
  const float inv = exp2i(-e);
  const int first = old_scale != exp2i(e) ? 0 : s0;  // earlier codes stay where the scale does
#pragma unroll 2
  for (int slot = first / RPP * RPP + lane / LPR; slot < s0 + n; slot += RPP) {
    if (slot < first) continue;
    float x[8];
    values(slot, x);
    *reinterpret_cast<uint32_t *>(page + slot * D + g.a) = e4m3x2(x[0] * inv, x[1] * inv) | e4m3x2(x[2] * inv, x[3] * inv) << 16;
    *reinterpret_cast<uint32_t *>(page + slot * D + g.b) = e4m3x2(x[4] * inv, x[5] * inv) | e4m3x2(x[6] * inv, x[7] * inv) << 16;
  }
  __syncwarp();
  if (lane == 0) *scale = exp2i(e);
}

// A warp per unit.  The first o.q_ctas CTAs rotate queries, the others write K and V: a page of one head, or some heads of one row.
// Nothing is written before the reservation is done, whatever it is: queries may be rotated in place, and those of a request
// that it refuses have to stay as they are.  A warp's first loads are on their way by then.
// What bounds it: the reservation's chain of dependent reads in front (8 to 10 us), then the latency of its loads (8 prompts: 30 us
// alone, DRAM busy half of the time).  Measured, whole calls with the reservation, D = 128, 8 KV and 32 query heads, e4m3 cache:
// 8 prompts of 700-1023 tokens 42 us, 256 requests of 2 to 17 rows 29 us, one row 10.3 us.  (With the queries rotated and stored beside the reservation 38.8, 26.4 and 10.3 us, those of
// refused requests among them.)
template <typename T, bool Q8, int D, bool INTER>
__global__ void __launch_bounds__(kThreads, kCtasPerSM) kv_append_rope_kernel(const KvParams p, const RopeParams o) {
  __shared__ __align__(16) T s_stage[Q8 ? kThreads / 32 * kKvPage * D : 1];
  constexpr int HC = heads_per_unit<T, D>();
  const int lane = threadIdx.x & 31;
  const int64_t T_rows = p.total_rows;
  if ((int)blockIdx.x < o.q_ctas) {
    const int qc = (o.Hq + HC - 1) / HC;
    const int64_t units = T_rows * qc, nwarps = (int64_t)o.q_ctas * (kThreads / 32);
    for (int64_t u = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < units; u += nwarps) {
      const int64_t x = u / qc;
      const int c = (int)(u % qc);
      move_heads<T, D, INTER, D>(o, reinterpret_cast<const T *>(o.q + x * o.q_stride), c * HC, o.Hq, true, [&](int &pos) -> T * {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        pos = p.row_pos[x];
        return p.row_req[x] < 0 ? nullptr : reinterpret_cast<T *>(o.q_out) + x * o.Hq * D;
      });
    }
    return;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent of the reservation
  const int kvc = (p.Hkv + HC - 1) / HC;
  const int64_t groups = Q8 ? (T_rows + o.group - 1) / o.group : T_rows;
  const int64_t units = groups * 2 * (Q8 ? p.Hkv : kvc), nwarps = (int64_t)(gridDim.x - o.q_ctas) * (kThreads / 32);
  for (int64_t u = (int64_t)(blockIdx.x - o.q_ctas) * (kThreads / 32) + (threadIdx.x >> 5); u < units; u += nwarps) {
    if (Q8) {
      const int hv = (int)(u % (2 * p.Hkv));
      const bool is_v = hv >= p.Hkv;
      const int h = is_v ? hv - p.Hkv : hv;
      const int64_t x0 = u / (2 * p.Hkv) * o.group;
      // the rows of the group that start a page or a request: each brings its page's new rows
      int r = -1, pos = 0, n = 0;
      if (lane < o.group && x0 + lane < T_rows) {
        r = p.row_req[x0 + lane];
        if (r >= 0) {
          pos = p.row_pos[x0 + lane];
          const int c = p.context_lens[r], end = c + p.draft_lens[r] + 1;
          n = min(min(kKvPage - pos % kKvPage, end - pos), (int)(T_rows - (x0 + lane)));
          if (pos % kKvPage != 0 && pos != c) n = 0;
        }
      }
      for (unsigned m = __ballot_sync(0xffffffffu, n > 0); m; m &= m - 1) {
        const int src = __ffs(m) - 1;
        const int rr = __shfl_sync(0xffffffffu, r, src), pp = __shfl_sync(0xffffffffu, pos, src);
        const int nn = __shfl_sync(0xffffffffu, n, src);
        const int32_t page = p.block_tables[(int64_t)rr * p.max_blocks + pp / kKvPage];
        if (page < 0 || page >= p.num_blocks) {  // a page id from the free stack outside the pool
          if (lane == 0) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, rr);
          continue;
        }
        const int64_t ph = (int64_t)page * p.Hkv + h;
        const char *rows = (is_v ? p.v_new + (x0 + src) * o.v_stride : p.k_new + (x0 + src) * o.k_stride);
        quantise_page<T, D, INTER>(o, s_stage + (threadIdx.x >> 5) * kKvPage * D, reinterpret_cast<uint8_t *>(is_v ? p.v_cache : p.k_cache) + ph * kKvPage * D,
                            (is_v ? o.v_scale : o.k_scale) + ph, reinterpret_cast<const T *>(rows) + (int64_t)h * D,
                            is_v ? o.v_stride : o.k_stride, pp % kKvPage, nn, pp, !is_v);
      }
    } else {
      const int64_t x = u / (2 * kvc);
      const int cv = (int)(u % (2 * kvc));
      const bool is_v = cv >= kvc;
      move_heads<T, D, INTER, kKvPage * D>(
          o, reinterpret_cast<const T *>(is_v ? p.v_new + x * o.v_stride : p.k_new + x * o.k_stride), (is_v ? cv - kvc : cv) * HC, p.Hkv,
          !is_v, [&](int &pos) -> T * {
            const int r = p.row_req[x];
            if (r < 0) return nullptr;
            pos = p.row_pos[x];
            const int32_t page = p.block_tables[(int64_t)r * p.max_blocks + pos / kKvPage];
            if (page < 0 || page >= p.num_blocks) {
              if (lane == 0) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, r);
              return nullptr;
            }
            return reinterpret_cast<T *>(is_v ? p.v_cache : p.k_cache) + ((int64_t)page * p.Hkv * kKvPage + pos % kKvPage) * D;
          });
    }
  }
}

wisp_status rope_check(const wisp_kv_rope_args *a, bool call) {
  if (!a) return WISP_ERR_INVALID_ARG;
  wisp_status st = kv_check(&a->kv, call, false);
  if (st != WISP_OK) return st;
  const wisp_kv_args &kv = a->kv;
  if (a->cache_dtype != kv.kv_dtype && a->cache_dtype != WISP_E4M3) return WISP_ERR_INVALID_ARG;
  if (a->rot_dim < 0 || a->rot_dim > kv.D || a->Hq < 0) return WISP_ERR_INVALID_ARG;
  if (a->rot_dim % 16 != 0) return WISP_ERR_UNSUPPORTED;
  if (!call || kv.B == 0) return WISP_OK;
  if (a->cache_dtype == WISP_E4M3 && (!a->k_scale || !a->v_scale)) return WISP_ERR_INVALID_ARG;
  if (a->rot_dim > 0 && (!a->rope || !al16(a->rope) || a->rope_positions <= 0)) return WISP_ERR_INVALID_ARG;
  if (a->Hq > 0 && (!a->q || !a->q_out || !al16(a->q) || !al16(a->q_out))) return WISP_ERR_INVALID_ARG;
  const int es = kv.kv_dtype == WISP_BF16 ? 2 : 4;
  auto bad = [&](int64_t stride, int64_t heads) {
    return stride != 0 && (stride < heads * kv.D || stride > INT64_MAX / es / kv.total_q_rows || stride * es % 16 != 0);
  };
  if (bad(a->k_stride, kv.Hkv) || bad(a->v_stride, kv.Hkv) || (a->Hq > 0 && bad(a->q_stride, a->Hq))) return WISP_ERR_INVALID_ARG;
  if (a->Hq > 0) {  // q_out over q: the same packed rows, or none
    const uint64_t row = (uint64_t)a->Hq * kv.D * es, T = kv.total_q_rows, q = (uintptr_t)a->q, out = (uintptr_t)a->q_out;
    const uint64_t step = a->q_stride ? (uint64_t)a->q_stride * es : row;
    const bool in_place = q == out && (step == row || T == 1);
    if (!in_place && q < out + T * row && out < q + (T - 1) * step + row) return WISP_ERR_INVALID_ARG;
  }
  return WISP_OK;
}

// wisp_kv_args' own parameters, with the longest sequence that the rotation's table allows.
KvParams rope_params(const wisp_kv_rope_args *a, void *ws, const KvLayout &L) {
  KvParams p = kv_params(&a->kv, ws, L);
  if (a->rot_dim > 0 && a->rope_positions < p.max_tokens) p.max_tokens = a->rope_positions;
  return p;
}

template <typename T, bool Q8>
cudaError_t launch(const KvParams &p, const RopeParams &o, const cudaLaunchConfig_t &cfg) {
  if (p.D == 128)
    return o.interleaved ? cudaLaunchKernelEx(&cfg, kv_append_rope_kernel<T, Q8, 128, true>, p, o)
                         : cudaLaunchKernelEx(&cfg, kv_append_rope_kernel<T, Q8, 128, false>, p, o);
  return o.interleaved ? cudaLaunchKernelEx(&cfg, kv_append_rope_kernel<T, Q8, 64, true>, p, o)
                       : cudaLaunchKernelEx(&cfg, kv_append_rope_kernel<T, Q8, 64, false>, p, o);
}

}  // namespace

}  // namespace wisp

using namespace wisp;

extern "C" {

size_t wisp_kv_rope_workspace_size(const wisp_kv_rope_args *a) {
  if (rope_check(a, false) != WISP_OK) return 0;
  return kv_layout(&a->kv).total;
}

wisp_status wisp_kv_reserve_append_rope(const wisp_kv_rope_args *a, void *ws, size_t ws_bytes, void *stream) {
  wisp_status st = rope_check(a, true);
  if (st != WISP_OK) return st;
  const wisp_kv_args &kv = a->kv;
  const KvLayout L = kv_layout(&kv);
  if ((st = kv_ws_ok(ws, ws_bytes, L)) != WISP_OK) return st;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const KvParams p = rope_params(a, ws, L);
  if (kv.B == 0)
    return cudaMemsetAsync(p.status, 0, sizeof(DeviceStatus), s) == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
  RopeParams o;
  std::memset(&o, 0, sizeof o);
  o.Hq = a->Hq;
  o.rot8 = a->rot_dim / 8;
  o.interleaved = a->interleaved != 0;
  o.table = a->rope;
  o.q = static_cast<const char *>(a->q);
  o.q_out = static_cast<char *>(a->q_out);
  o.q_stride = (a->q_stride ? a->q_stride : (int64_t)a->Hq * kv.D) * p.esize;
  o.k_stride = (a->k_stride ? a->k_stride : (int64_t)kv.Hkv * kv.D) * p.esize;
  o.v_stride = (a->v_stride ? a->v_stride : (int64_t)kv.Hkv * kv.D) * p.esize;
  o.k_scale = a->k_scale;
  o.v_scale = a->v_scale;
  const bool q8 = a->cache_dtype == WISP_E4M3;
  // A unit has a group of rows and takes the pages that start in it: prompts have one every 16 rows, single tokens one each.  A
  // quarter of a request's rows, so that a warp seldom has two pages in turn.
  o.group = 1;
  while (o.group < kKvPage && 4 * o.group <= kv.total_q_rows / kv.B) o.group *= 2;
  const bool bf = kv.kv_dtype == WISP_BF16;
  const int hc = kv.D == 128 ? (bf ? heads_per_unit<uint16_t, 128>() : heads_per_unit<float, 128>())
                             : (bf ? heads_per_unit<uint16_t, 64>() : heads_per_unit<float, 64>());
  const int64_t T = kv.total_q_rows;
  const int64_t kv_units = q8 ? (T + o.group - 1) / o.group * 2 * kv.Hkv : T * 2 * ((kv.Hkv + hc - 1) / hc);
  const int64_t q_units = T * ((a->Hq + hc - 1) / hc);
  auto ctas = [](int64_t units, int64_t most) {
    const int64_t n = (units + kThreads / 32 - 1) / (kThreads / 32);
    return (int)(n < most ? n : most);
  };
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
    return WISP_ERR_CUDA;
  o.q_ctas = ctas(q_units, (int64_t)sms * 2);  // (8 prompts: with one per SM 51 us, two or four 42, eight 45)
  if (kv_reserve_launch(p, s) != cudaSuccess) return WISP_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)(o.q_ctas + ctas(kv_units, 16384)));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = bf ? (q8 ? launch<uint16_t, true>(p, o, cfg) : launch<uint16_t, false>(p, o, cfg))
                           : (q8 ? launch<float, true>(p, o, cfg) : launch<float, false>(p, o, cfg));
  return e == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
}

wisp_status wisp_kv_commit_rope(const wisp_kv_rope_args *a, void *ws, size_t ws_bytes, void *stream) {
  wisp_status st = rope_check(a, false);
  if (st != WISP_OK) return st;
  if ((st = kv_check(&a->kv, false, true)) != WISP_OK) return st;
  if (a->kv.B > 0 && a->rot_dim > 0 && a->rope_positions <= 0) return WISP_ERR_INVALID_ARG;
  const KvLayout L = kv_layout(&a->kv);
  if ((st = kv_ws_ok(ws, ws_bytes, L)) != WISP_OK) return st;
  return kv_commit_launch(rope_params(a, ws, L), static_cast<cudaStream_t>(stream));
}

}  // extern "C"
