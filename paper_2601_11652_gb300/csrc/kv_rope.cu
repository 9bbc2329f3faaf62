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

constexpr int kThreads = 256;
constexpr int kPasses = 4;  // warp passes over heads per unit of work: so many loads in flight

struct RopeParams {
  int Hq, rot16;         // queries' heads; rotated elements / 16
  int interleaved;
  int group;             // consecutive new rows per K/V unit of an e4m3 cache, at most 16
  const float *table;    // [positions, 16 * rot16]: cosines, then sines
  const char *q;
  char *q_out;
  int64_t q_stride, k_stride, v_stride;  // bytes between rows
  float *k_scale, *v_scale;
};

// 16 elements of one head's row per lane, as two groups of 8: those that rotate into each other (lanes
// below rot16), or two groups that pass.
struct Groups {
  int a, b;
  bool turn;
};
__device__ __forceinline__ Groups groups_of(int l, const RopeParams &o) {
  Groups g;
  g.turn = l < o.rot16;
  if (g.turn) {
    g.a = o.interleaved ? 2 * l : l;
    g.b = o.interleaved ? 2 * l + 1 : l + o.rot16;
  } else {
    g.a = 2 * l;
    g.b = 2 * l + 1;
  }
  return g;
}

__device__ __forceinline__ void load8(const uint16_t *src, float (&x)[16], int at) {
  const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src));
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[at + 2 * i] = __uint_as_float(w[i] << 16);
    x[at + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float *src, float (&x)[16], int at) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float4 v = __ldg(reinterpret_cast<const float4 *>(src) + h);
    x[at + 4 * h] = v.x;
    x[at + 4 * h + 1] = v.y;
    x[at + 4 * h + 2] = v.z;
    x[at + 4 * h + 3] = v.w;
  }
}
__device__ __forceinline__ void store8(uint16_t *dst, const float (&x)[16], int at) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(x[at + 2 * i], x[at + 2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t *>(&v);
  }
  *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float *dst, const float (&x)[16], int at) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
    reinterpret_cast<float4 *>(dst)[h] = make_float4(x[at + 4 * h], x[at + 4 * h + 1], x[at + 4 * h + 2], x[at + 4 * h + 3]);
}

// The lane's 8 cosines and 8 sines of a position.
struct Angles {
  float c[8], s[8];
};
__device__ __forceinline__ void load_angles(const RopeParams &o, int pos, int l, Angles &t) {
  const float4 *p = reinterpret_cast<const float4 *>(o.table + (int64_t)pos * 16 * o.rot16 + 8 * l);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float4 c = __ldg(p + h), s = __ldg(p + 2 * o.rot16 + h);
    t.c[4 * h] = c.x;
    t.c[4 * h + 1] = c.y;
    t.c[4 * h + 2] = c.z;
    t.c[4 * h + 3] = c.w;
    t.s[4 * h] = s.x;
    t.s[4 * h + 1] = s.y;
    t.s[4 * h + 2] = s.z;
    t.s[4 * h + 3] = s.w;
  }
}
__device__ __forceinline__ void turn_pair(float &a, float &b, float c, float s) {
  const float u = __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s));
  b = __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s));
  a = u;
}
__device__ __forceinline__ void rotate(float (&x)[16], const Angles &t, bool interleaved) {
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_pair(x[2 * i], x[2 * i + 1], t.c[i], t.s[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_pair(x[i], x[i + 8], t.c[i], t.s[i]);
  }
}

// Heads [h0, h0 + kPasses * heads per pass) of one row: src -> dst, rotated if `turn`.  dst heads are dst_head
// elements apart.
template <typename T, int D>
__device__ __forceinline__ void move_heads(const RopeParams &o, const T *src, T *dst, int64_t dst_head, int h0, int H, int pos,
                                           bool turn) {
  constexpr int LPR = D / 16, RPP = 32 / LPR;
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const Groups g = groups_of(l, o);
  float x[kPasses][16];
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int h = h0 + i * RPP + lane / LPR;
    if (h < H) {
      load8(src + (int64_t)h * D + 8 * g.a, x[i], 0);
      load8(src + (int64_t)h * D + 8 * g.b, x[i], 8);
    }
  }
  if (turn && g.turn) {
    Angles t;
    load_angles(o, pos, l, t);
#pragma unroll
    for (int i = 0; i < kPasses; ++i) rotate(x[i], t, o.interleaved);
  }
#pragma unroll
  for (int i = 0; i < kPasses; ++i) {
    const int h = h0 + i * RPP + lane / LPR;
    if (h < H) {
      store8(dst + h * dst_head + 8 * g.a, x[i], 0);
      store8(dst + h * dst_head + 8 * g.b, x[i], 8);
    }
  }
}

// One page of one head of an e4m3 cache, by one warp: slots s0 .. s0 + n - 1 are new rows (the first of them at src,
// at position pos), slots below s0 hold earlier ones.
template <typename T, int D>
__device__ __forceinline__ void quantise_page(const RopeParams &o, uint8_t *page, float *scale, const T *src,
                                              int64_t src_row, int s0, int n, int pos, bool turn) {
  constexpr int LPR = D / 16, RPP = 32 / LPR, NP = kKvPage / RPP;
  const int lane = threadIdx.x & 31, l = lane % LPR;
  const Groups g = groups_of(l, o);
  float x[NP][16];
  const float old_scale = s0 > 0 ? *scale : 1.0f;
  float amax = 0.0f;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int slot = i * RPP + lane / LPR;
    if (slot < s0) {
      const uint2 ca = *reinterpret_cast<const uint2 *>(page + slot * D + 8 * g.a);
      const uint2 cb = *reinterpret_cast<const uint2 *>(page + slot * D + 8 * g.b);
      const uint32_t w[4] = {ca.x, ca.y, cb.x, cb.y};
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float2 v = h2_to_f2(e4m3x2_to_h2((w[q >> 1] >> (16 * (q & 1))) & 0xffffu));
        x[i][2 * q] = v.x * old_scale;
        x[i][2 * q + 1] = v.y * old_scale;
      }
    } else if (slot < s0 + n) {
      const T *row = reinterpret_cast<const T *>(reinterpret_cast<const char *>(src) + (slot - s0) * src_row);
      load8(row + 8 * g.a, x[i], 0);
      load8(row + 8 * g.b, x[i], 8);
      if (turn && g.turn) {
        Angles t;
        load_angles(o, pos + slot - s0, l, t);
        rotate(x[i], t, o.interleaved);
      }
    } else {
#pragma unroll
      for (int q = 0; q < 16; ++q) x[i][q] = 0.0f;
    }
#pragma unroll
    for (int q = 0; q < 16; ++q) amax = fmaxf(amax, fabsf(x[i][q]));  // (a NaN loses)
  }
  amax = ptx::warp_max(amax);
  if (amax == INFINITY) {  // the largest finite magnitude decides
    amax = 0.0f;
#pragma unroll
    for (int i = 0; i < NP; ++i)
#pragma unroll
      for (int q = 0; q < 16; ++q) amax = fmaxf(amax, fabsf(x[i][q]) < INFINITY ? fabsf(x[i][q]) : 0.0f);
    amax = ptx::warp_max(amax);
  }
  const int e = scale_exp(amax);
  const float inv = exp2i(-e);
  const bool rewrite = old_scale != exp2i(e);
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int slot = i * RPP + lane / LPR;
    if (slot < s0 + n && (slot >= s0 || rewrite)) {
      uint32_t w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        w[q] = e4m3x2(x[i][4 * q] * inv, x[i][4 * q + 1] * inv) | e4m3x2(x[i][4 * q + 2] * inv, x[i][4 * q + 3] * inv) << 16;
      *reinterpret_cast<uint2 *>(page + slot * D + 8 * g.a) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2 *>(page + slot * D + 8 * g.b) = make_uint2(w[2], w[3]);
    }
  }
  if (lane == 0) *scale = exp2i(e);
}

// A warp per unit: first the K/V units (a page of one head, or some heads of one row), then the queries'.
template <typename T, bool Q8, int D>
__global__ void __launch_bounds__(kThreads) kv_append_rope_kernel(const KvParams p, const RopeParams o) {
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched as a programmatic dependent of the reservation
  constexpr int HC = kPasses * (32 / (D / 16));        // heads per unit of whole rows
  const int lane = threadIdx.x & 31;
  const int64_t T_rows = p.total_rows;
  const int kvc = (p.Hkv + HC - 1) / HC, qc = (o.Hq + HC - 1) / HC;
  const int64_t groups = Q8 ? (T_rows + o.group - 1) / o.group : T_rows;
  const int64_t kv_units = groups * 2 * (Q8 ? p.Hkv : kvc), units = kv_units + T_rows * qc;
  const int64_t nwarps = (int64_t)gridDim.x * (kThreads / 32);
  for (int64_t u = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5); u < units; u += nwarps) {
    if (u >= kv_units) {
      const int64_t x = (u - kv_units) / qc;
      const int c = (int)((u - kv_units) % qc);
      if (p.row_req[x] < 0) continue;
      move_heads<T, D>(o, reinterpret_cast<const T *>(o.q + x * o.q_stride), reinterpret_cast<T *>(o.q_out) + x * o.Hq * D, D,
                       c * HC, o.Hq, p.row_pos[x], true);
      continue;
    }
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
        quantise_page<T, D>(o, reinterpret_cast<uint8_t *>(is_v ? p.v_cache : p.k_cache) + ph * kKvPage * D,
                            (is_v ? o.v_scale : o.k_scale) + ph, reinterpret_cast<const T *>(rows) + (int64_t)h * D,
                            is_v ? o.v_stride : o.k_stride, pp % kKvPage, nn, pp, !is_v);
      }
    } else {
      const int64_t x = u / (2 * kvc);
      const int cv = (int)(u % (2 * kvc));
      const bool is_v = cv >= kvc;
      const int r = p.row_req[x];
      if (r < 0) continue;
      const int pos = p.row_pos[x];
      const int32_t page = p.block_tables[(int64_t)r * p.max_blocks + pos / kKvPage];
      if (page < 0 || page >= p.num_blocks) {
        if (lane == 0) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, r);
        continue;
      }
      T *dst = reinterpret_cast<T *>(is_v ? p.v_cache : p.k_cache) + ((int64_t)page * p.Hkv * kKvPage + pos % kKvPage) * D;
      move_heads<T, D>(o, reinterpret_cast<const T *>(is_v ? p.v_new + x * o.v_stride : p.k_new + x * o.k_stride), dst,
                       kKvPage * D, (is_v ? cv - kvc : cv) * HC, p.Hkv, pos, !is_v);
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
  return WISP_OK;
}

template <typename T, bool Q8>
cudaError_t launch(const KvParams &p, const RopeParams &o, const cudaLaunchConfig_t &cfg) {
  return p.D == 128 ? cudaLaunchKernelEx(&cfg, kv_append_rope_kernel<T, Q8, 128>, p, o)
                    : cudaLaunchKernelEx(&cfg, kv_append_rope_kernel<T, Q8, 64>, p, o);
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
  KvParams p = kv_params(&kv, ws, L);
  if (kv.B == 0)
    return cudaMemsetAsync(p.status, 0, sizeof(DeviceStatus), s) == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
  if (a->rot_dim > 0 && a->rope_positions < p.max_tokens) p.max_tokens = a->rope_positions;
  RopeParams o;
  std::memset(&o, 0, sizeof o);
  o.Hq = a->Hq;
  o.rot16 = a->rot_dim / 16;
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
  // about one page start per group of rows: prompts have one every 16 rows, single tokens one each
  o.group = 1;
  while (o.group < kKvPage && 2 * o.group <= kv.total_q_rows / kv.B) o.group *= 2;
  const int hc = kPasses * (32 / (kv.D / 16));
  const int64_t T = kv.total_q_rows;
  const int64_t units = (q8 ? (T + o.group - 1) / o.group * 2 * kv.Hkv : T * 2 * ((kv.Hkv + hc - 1) / hc)) + T * ((a->Hq + hc - 1) / hc);
  const int64_t blocks = (units + kThreads / 32 - 1) / (kThreads / 32);
  if (kv_reserve_launch(p, s) != cudaSuccess) return WISP_ERR_CUDA;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)(blocks < 4096 ? blocks : 4096));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = kv.kv_dtype == WISP_BF16 ? (q8 ? launch<uint16_t, true>(p, o, cfg) : launch<uint16_t, false>(p, o, cfg))
                                                 : (q8 ? launch<float, true>(p, o, cfg) : launch<float, false>(p, o, cfg));
  return e == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
}

}  // extern "C"
