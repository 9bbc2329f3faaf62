// prompt_row.cuh -- one row of the attention of prompt.cuh by one warp in plain fp32, for the rare rows that the tensor-core kernels hand on:
// values near the ends of fp32, where their scaled operands or their unnormalised sums leave what they can hold.
#pragma once

#include "attn_merge.cuh"
#include "fp8.cuh"
#include "prompt.cuh"

namespace wisp {

// CPL (2 or 4) consecutive elements, in fp32.  Codes of e4m3 times `sc`, and that in bf16 where the queries are bf16 (as prompt_tc.cu).
template <int CPL>
__device__ __forceinline__ void row_values(const float *src, float (&v)[CPL]) {
  if (CPL == 4) {
    const float4 t = __ldg(reinterpret_cast<const float4 *>(src));
    v[0] = t.x;
    v[1] = t.y;
    v[CPL - 2] = t.z;
    v[CPL - 1] = t.w;
  } else {
    const float2 t = __ldg(reinterpret_cast<const float2 *>(src));
    v[0] = t.x;
    v[1] = t.y;
  }
}
template <int CPL>
__device__ __forceinline__ void row_values(const uint16_t *src, float (&v)[CPL]) {
#pragma unroll
  for (int i = 0; i < CPL; i += 2) {
    const uint32_t u = __ldg(reinterpret_cast<const uint32_t *>(src + i));
    v[i] = __uint_as_float(u << 16);
    v[i + 1] = __uint_as_float(u & 0xffff0000u);
  }
}
template <int CPL, bool BF16>
__device__ __forceinline__ void row_codes(const uint8_t *src, float sc, float (&v)[CPL]) {
#pragma unroll
  for (int i = 0; i < CPL; i += 2) {
    const float2 t = h2_to_f2(e4m3x2_to_h2(__ldg(reinterpret_cast<const uint16_t *>(src + i))));
    v[i] = t.x * sc;
    v[i + 1] = t.y * sc;
    if (BF16) {
      const uint32_t u = bf16x2_sat(v[i], v[i + 1]);
      v[i] = __uint_as_float(u << 16);
      v[i + 1] = __uint_as_float(u & 0xffff0000u);
    }
  }
}

// Output row `row` (of all query rows), query head `head`.  Keys in turn, eight at a time; the output is kept
// normalised, o' = o (l a / l') + sum_i v_i (w_i / l'), so that it never leaves the range of the values.  Reads K and V once per row from L2,
// about 35 instructions a key: a whole prompt of 16384 tokens this way would take some tenths of a second, a thousand times the tensor cores' time.
// only_not_finite: only the elements whose output is not finite (others keep what they have).
template <int D, typename T>
__device__ __forceinline__ void prompt_row(const PromptPlan &p, const AttnParams &a, int row, int head, bool only_not_finite) {
  constexpr bool kBf = sizeof(T) == 2;
  constexpr int CPL = D / 32, kKeys = 8;
  const int lane = threadIdx.x & 31, hk = head / (p.Hq / p.Hkv);
  int r = 0;  // its request: the last one whose first row is not behind it
  for (int hi = p.B - 1; r < hi;) {
    const int mid = (r + hi + 1) >> 1;
    if (p.q_row_start[mid] <= row) r = mid;
    else hi = mid - 1;
  }
  const Segment &own = p.segs[r];
  const int run = p.req_run[r], shared = own.t0 / 16;  // pages that the run's first request names
  const int32_t *bt = a.block_tables + (int64_t)r * a.max_blocks_per_seq;
  const int32_t *bt0 = a.block_tables + (int64_t)(run >= 0 ? p.segs[p.B + run].r : r) * a.max_blocks_per_seq;
  const int seen = own.ctx + (row - own.q0) + 1;
  const int64_t at = ((int64_t)row * p.Hq + head) * D + lane * CPL;
  float q[CPL], o[CPL];
  row_values<CPL>(static_cast<const T *>(a.q) + at, q);
  float amax = 0.0f;
#pragma unroll
  for (int c = 0; c < CPL; ++c) {
    amax = fmaxf(amax, fabsf(q[c]));
    o[c] = 0.0f;
  }
  // codes times their scale may be past fp32 where the scores are not: 2^-16 of the scale goes to the queries, if they have room
  const bool move = !kBf && a.k_scale && ptx::warp_max(amax) < 0x1p100f;
  const float down = move ? 0x1p-16f : 1.0f;
#pragma unroll
  for (int c = 0; c < CPL; ++c) q[c] *= move ? 0x1p16f : 1.0f;
  const float scale = 1.4426950408889634f / sqrtf((float)D);
  float m = -INFINITY, l = 0.0f;
  for (int t = 0; t < seen; t += kKeys) {
    const int page = t / 16, bid = __ldg((page < shared ? bt0 : bt) + page);
    const bool valid = bid >= 0 && bid < a.num_blocks;  // (else its keys and values count as zeros, as in the tensor-core kernels)
    const int64_t head0 = (int64_t)(valid ? bid : 0) * a.Hkv + hk, src = (head0 * 16 + t % 16) * D + lane * CPL;
    float s[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      float k[CPL];
      if (a.k_scale) row_codes<CPL, kBf>(static_cast<const uint8_t *>(a.k_cache) + src + i * D, __ldg(a.k_scale + head0) * down, k);
      else row_values<CPL>(static_cast<const T *>(a.k_cache) + src + i * D, k);
      s[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) s[i] = fmaf(q[c], k[c], s[i]);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
#pragma unroll
      for (int i = 0; i < kKeys; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], d);
    float mn = m;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      s[i] = t + i < seen ? (valid ? __fmul_rn(s[i], scale) : 0.0f) : -INFINITY;
      mn = fmaxf(mn, s[i]);
    }
    const float ref = mn == -INFINITY ? 0.0f : mn;
    float ln = l * (m == mn ? 1.0f : ptx::ex2(m - ref));
    const float old = ln;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      s[i] = ptx::ex2(__fadd_rn(s[i], -ref));
      ln += s[i];
    }
    m = mn;
    l = ln;
    if (ln == 0.0f) continue;  // (scores of -inf so far)
    const float inv = 1.0f / ln, keep = old * inv;
#pragma unroll
    for (int c = 0; c < CPL; ++c) o[c] *= keep;
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      if (t + i >= seen || !valid) continue;
      float v[CPL];
      if (a.k_scale) row_codes<CPL, kBf>(static_cast<const uint8_t *>(a.v_cache) + src + i * D, __ldg(a.v_scale + head0), v);
      else row_values<CPL>(static_cast<const T *>(a.v_cache) + src + i * D, v);
#pragma unroll
      for (int c = 0; c < CPL; ++c) o[c] = fmaf(s[i] * inv, v[c], o[c]);
    }
  }
  T *out = static_cast<T *>(p.out) + at;
  if (only_not_finite) {  // (l is finite, and so are the elements that stay)
    float had[CPL];
#pragma unroll
    for (int c = 0; c < CPL; ++c) had[c] = sizeof(T) == 2 ? __uint_as_float((uint32_t)out[c] << 16) : (float)out[c];
#pragma unroll
    for (int c = 0; c < CPL; ++c) o[c] = fabsf(had[c]) < INFINITY ? had[c] : o[c];
  }
  st_cols<CPL>(out, o, l == 0.0f ? __uint_as_float(0x7fffffffu) : 1.0f);
}

}  // namespace wisp
