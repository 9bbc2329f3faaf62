// attn_kv8_f32.cu -- paged GQA attention of the verification forward over an e4m3 cache with fp32 queries, on the CUDA
// cores (the tensor cores would round the queries).
//
// Same contract as attn_f32.cu, with K and V of a page of one head worth code * scale (include/wisp_kv8.h).
//
// Persistent CTAs (one per SM) of eight warps take work items from the plan's counter.  A warp keeps four of
// an item's rows: their scores against a page of 16 keys (lane: one key, two rows), running maxima and sums, and O
// (lane: D / 32 columns of the four rows).  The CTA decodes each page into shared memory once.
#include "attn_merge.cuh"
#include "fp8.cuh"

#include <cstring>

namespace wisp {

namespace {

constexpr int kWarps = 8;
constexpr int kThreads = kWarps * 32;
constexpr int kPage = 16;
constexpr int kRowsPerWarp = kF32RowsPerItem / kWarps;
static_assert(kRowsPerWarp == 4, "rows of an item");

}  // namespace

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attn_kv8_f32_kernel(const __grid_constant__ AttnParams p) {
  constexpr int LD = D + 4, CPL = D / 32;
  __shared__ __align__(16) float s_q[kF32RowsPerItem * LD];
  extern __shared__ __align__(16) float s_kv[];  // K [16][LD], V [16][LD]
  __shared__ float s_p[kWarps][kRowsPerWarp][kPage];
  __shared__ int s_item, s_last;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int key = lane & 15, half = lane >> 4;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n_items = p.header->n_items;
  if ((int)blockIdx.x >= p.header->attn_ctas) return;  // the SM is left to the acceptance pass of the same step
  const int g = p.Hq / p.Hkv;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  for (;;) {
    __syncthreads();
    if (tid == 0) {
      int it;
      do {
        it = atomicAdd(&p.header_mut->next_item, 1);
        if (it >= n_items) it = -1;
      } while (it >= 0 && p.items[it].t1 <= p.items[it].t0);  // (a refused request's items are empty)
      s_item = it;
    }
    __syncthreads();
    const int it = s_item;
    if (it < 0) break;
    const WorkItem w = p.items[it];
    for (int c = tid; c < kF32RowsPerItem * D; c += kThreads) {
      const int row = c / D, d = c % D, rj = w.row0 + row;
      s_q[row * LD + d] =
          row < w.rows ? static_cast<const float *>(p.q)[((int64_t)(w.q0 + rj / g) * p.Hq + w.h * g + rj % g) * D + d] : 0.0f;
    }
    float o[kRowsPerWarp][CPL], m[2], l[2];
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i)
#pragma unroll
      for (int q = 0; q < CPL; ++q) o[i][q] = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.0f;
    }
    const int32_t *bt = p.block_tables + (int64_t)w.r * p.max_blocks_per_seq;
    for (int t = w.t0; t < w.t1; t += kPage) {
      const int32_t b = bt[t / kPage];
      const bool bad = b < 0 || b >= p.num_blocks;
      if (bad && tid == 0) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, w.r);
      const int64_t ph = (int64_t)(bad ? 0 : b) * p.Hkv + w.h;
      const float ks = p.k_scale[ph], vs = p.v_scale[ph];
      __syncthreads();  // the page before is no longer read
      for (int c = tid; c < 2 * kPage * D / 16; c += kThreads) {  // 16 codes of K or V
        const int slot = c % (kPage * D / 16) / (D / 16), d = c % (D / 16) * 16;
        const bool v = c >= kPage * D / 16;
        const uint8_t *src = static_cast<const uint8_t *>(v ? p.v_cache : p.k_cache) + (ph * kPage + slot) * D + d;
        float *dst = s_kv + ((v ? kPage : 0) + slot) * LD + d;
        // slots past the item hold anything: zeros in their place
        const uint4 x = bad || t + slot >= w.t1 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4 *>(src);
        const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 f = h2_to_f2(e4m3x2_to_h2((u[i >> 1] >> (16 * (i & 1))) & 0xffffu));
          dst[2 * i] = f.x * (v ? vs : ks);
          dst[2 * i + 1] = f.y * (v ? vs : ks);
        }
      }
      __syncthreads();
      const int tok = t + key;
      float al[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int row = warp * kRowsPerWarp + half * 2 + i;
        float s = 0.0f;
        for (int d = 0; d < D; d += 4) {
          const float4 a = *reinterpret_cast<const float4 *>(s_q + row * LD + d);
          const float4 k = *reinterpret_cast<const float4 *>(s_kv + key * LD + d);
          s = fmaf(a.x, k.x, fmaf(a.y, k.y, fmaf(a.z, k.z, fmaf(a.w, k.w, s))));
        }
        const bool seen = tok < w.t1 && w.row0 + row >= g * max(tok - w.ctx, 0);
        s = seen ? s * scale_log2 : -INFINITY;
        float mx = s;
        for (int x = 1; x < 16; x <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
        const float mn = fmaxf(m[i], mx);
        al[i] = mn == m[i] ? 1.0f : exp2f(m[i] - mn);
        m[i] = mn;
        const float e = s == -INFINITY ? 0.0f : exp2f(s - mn);
        l[i] = fmaf(l[i], al[i], e);
        s_p[warp][half * 2 + i][key] = e;
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < kRowsPerWarp; ++i) {
        const float a = __shfl_sync(0xffffffffu, al[i & 1], (i >> 1) * 16);
#pragma unroll
        for (int q = 0; q < CPL; ++q) o[i][q] *= a;
        for (int x = 0; x < kPage; ++x) {
          const float e = s_p[warp][i][x];
          if (e != 0.0f) {  // (a key that the row does not see adds nothing, whatever it holds)
#pragma unroll
            for (int q = 0; q < CPL; ++q) o[i][q] = fmaf(e, s_kv[(kPage + x) * LD + lane * CPL + q], o[i][q]);
          }
        }
      }
      __syncwarp();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      for (int x = 1; x < 16; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
      const int row = warp * kRowsPerWarp + i;
      const float den = __shfl_sync(0xffffffffu, l[i & 1], (i >> 1) * 16), mx = __shfl_sync(0xffffffffu, m[i & 1], (i >> 1) * 16);
      if (row >= w.rows) continue;
      if (w.poff < 0) {
        const int rj = w.row0 + row;
        st_cols<CPL>(static_cast<float *>(p.out) + ((int64_t)(w.q0 + rj / g) * p.Hq + w.h * g + rj % g) * D + lane * CPL, o[i], 1.0f / den);
      } else {
        float *part = p.partials + w.poff;
#pragma unroll
        for (int q = 0; q < CPL; ++q) __stcg(part + (int64_t)row * D + lane * CPL + q, o[i][q]);
        if (lane == 0) {
          __stcg(part + w.rows * D + row, mx);
          __stcg(part + w.rows * D + w.rows + row, den);
        }
      }
    }
    if (w.poff >= 0) {
      // split: the last chunk of this (request, head, row group) to finish merges all
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const int chunks = p.req_chunks[w.r];
        const int done = atomicAdd(p.pair_done + ((int64_t)w.r * p.Hkv + w.h) * p.row_groups + w.rg, 1);
        s_last = done == chunks - 1 ? chunks : 0;
        __threadfence();
      }
      __syncthreads();
      if (s_last > 0) merge_chunks<D, float>(p, w, g, s_last, warp, kWarps);
    }
  }
}

cudaError_t attn_kv8_f32_launch(const AttnParams &p, int grid, cudaStream_t s) {
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cfg.dynamicSmemBytes = 2 * kPage * (p.D + 4) * 4;
  return p.D == 128 ? cudaLaunchKernelEx(&cfg, attn_kv8_f32_kernel<128>, p) : cudaLaunchKernelEx(&cfg, attn_kv8_f32_kernel<64>, p);
}

}  // namespace wisp
