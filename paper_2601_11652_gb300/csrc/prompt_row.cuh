// prompt_row.cuh -- one row of the attention of prompt.cuh by one warp in plain fp32, for the rare rows that the tensor-core kernels hand on
// (prompt.cuh): scores so far from zero that their steps are powers of two of their weights, and fp32 operands too far apart.
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

// Output rows row[i] (of all query rows), query heads head[i], i in the mask `use`: of request r and KV head hk.  Keys in turn, eight at a time; lane
// 8 i + k (modulo kSums) has row i's score of the k-th, its softmax is among eight lanes.  Outputs are kept normalised, o' = o (l a / l') + sum_k v_k (w_k / l'), so
// that they never leave the range of the values.  Bound by instructions: all rows of a prompt of 8192 tokens, 32 heads over 8
// of 128, 130 ms (the tensor cores 0.3).  Four rows at once took 82, but with 13 KB more code the merge took 1.3 us more where nothing is handed on.
constexpr int kRowsAtOnce = 2;
template <int D, typename T, bool KV8>
__device__ __forceinline__ void prompt_rows(const PromptPlan &p, const AttnParams &a, int r, const int (&row)[kRowsAtOnce], const int (&head)[kRowsAtOnce],
                                            int hk, uint32_t use) {
  constexpr bool kBf = sizeof(T) == 2;
  constexpr int CPL = D / 32, kKeys = 8, kSums = kRowsAtOnce * kKeys;
  const int lane = threadIdx.x & 31;
  const Segment &own = p.segs[r];
  const int run = p.req_run[r], shared = own.t0 / 16;  // pages that the run's first request names
  const int32_t *bt = a.block_tables + (int64_t)r * a.max_blocks_per_seq;
  const int32_t *bt0 = a.block_tables + (int64_t)(run >= 0 ? p.segs[p.B + run].r : r) * a.max_blocks_per_seq;
  float q[kRowsAtOnce][CPL], o[kRowsAtOnce][CPL];
  int64_t at[kRowsAtOnce];
  int seen[kRowsAtOnce], most = 0;
#pragma unroll
  for (int i = 0; i < kRowsAtOnce; ++i) {
    const bool has = use >> i & 1;
    at[i] = has ? ((int64_t)row[i] * p.Hq + head[i]) * D + lane * CPL : 0;
    seen[i] = has ? own.ctx + (row[i] - own.q0) + 1 : 0;
    most = max(most, seen[i]);
#pragma unroll
    for (int c = 0; c < CPL; ++c) q[i][c] = o[i][c] = 0.0f;
    if (has) row_values<CPL>(static_cast<const T *>(a.q) + at[i], q[i]);
  }
  int mine = 0;  // keys that this lane's row sees
#pragma unroll
  for (int i = 0; i < kRowsAtOnce; ++i) mine = lane % kSums / kKeys == i ? seen[i] : mine;
  const float scale = 1.4426950408889634f / sqrtf((float)D);
  float m = -INFINITY, l = 0.0f;  // of this lane's row
  for (int t = 0; t < most; t += kKeys) {
    const int page = t / 16, bid = __ldg((page < shared ? bt0 : bt) + page);
    const bool valid = bid >= 0 && bid < a.num_blocks;  // (else its keys and values count as zeros, as in the tensor-core kernels)
    const int64_t head0 = (int64_t)(valid ? bid : 0) * a.Hkv + hk, src = (head0 * 16 + t % 16) * D + lane * CPL;
    // codes times their scale may be past fp32 where the scores are not
    const float ks = KV8 ? __ldg(a.k_scale + head0) : 1.0f, down = !kBf && ks > 0x1p60f ? 0x1p-16f : 1.0f;
    float s[kSums], v[kKeys][CPL];
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {  // (a page's slots behind the rows' keys may hold anything, but they are there)
      float x[CPL];
      if (KV8) {
        row_codes<CPL, kBf>(static_cast<const uint8_t *>(a.k_cache) + src + k * D, ks * down, x);
        row_codes<CPL, kBf>(static_cast<const uint8_t *>(a.v_cache) + src + k * D, __ldg(a.v_scale + head0), v[k]);
      } else {
        row_values<CPL>(static_cast<const T *>(a.k_cache) + src + k * D, x);
        row_values<CPL>(static_cast<const T *>(a.v_cache) + src + k * D, v[k]);
      }
#pragma unroll
      for (int i = 0; i < kRowsAtOnce; ++i) {
        float y = 0.0f;
#pragma unroll
        for (int c = 0; c < CPL; ++c) y = fmaf(q[i][c], x[c], y);
        s[i * kKeys + k] = y;
      }
    }
    // kSums sums over the lanes: every lane ends with the one of its number (modulo kSums)
#pragma unroll
    for (int d = 16; d >= kSums; d >>= 1)
#pragma unroll
      for (int i = 0; i < kSums; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], d);
#pragma unroll
    for (int d = kSums / 2; d > 0; d >>= 1)
#pragma unroll
      for (int i = 0; i < d; ++i) {
        const float keep = lane & d ? s[i + d] : s[i], give = lane & d ? s[i] : s[i + d];
        s[i] = keep + __shfl_xor_sync(0xffffffffu, give, d);
      }
    const float x = t + (lane & 7) < mine ? (valid ? __fmul_rn(s[0], scale / down) : 0.0f) : -INFINITY;
    float mn = x;
#pragma unroll
    for (int d = 1; d < kKeys; d <<= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
    mn = fmaxf(mn, m);
    const float ref = mn == -INFINITY ? 0.0f : mn, e = ptx::ex2(__fadd_rn(x, -ref));
    float sum = e;
#pragma unroll
    for (int d = 1; d < kKeys; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    const float old = l * (m == mn ? 1.0f : ptx::ex2(m - ref));
    m = mn;
    l = old + sum;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;  // (0: scores of -inf so far)
    const float keep = t < mine ? old * inv : 1.0f, w = t < mine ? e * inv : 0.0f;  // (behind its last key a row stays as it is: what goes with it has no say)
#pragma unroll
    for (int i = 0; i < kRowsAtOnce; ++i) {
      const float f = __shfl_sync(0xffffffffu, keep, i * kKeys);
#pragma unroll
      for (int c = 0; c < CPL; ++c) o[i][c] *= f;
#pragma unroll
      for (int k = 0; k < kKeys; ++k) {
        const float g = __shfl_sync(0xffffffffu, w, i * kKeys + k);
        if (t + k < seen[i] && valid)
#pragma unroll
          for (int c = 0; c < CPL; ++c) o[i][c] = fmaf(g, v[k][c], o[i][c]);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kRowsAtOnce; ++i) {
    const float sum = __shfl_sync(0xffffffffu, l, i * kKeys);
    if (use >> i & 1) st_cols<CPL>(static_cast<T *>(p.out) + at[i], o[i], sum == 0.0f ? __uint_as_float(0x7fffffffu) : 1.0f);
  }
}

// The request of a row: the last one whose first row is not behind it.
__device__ __forceinline__ int request_of(const PromptPlan &p, int row) {
  int r = 0;
  for (int hi = p.B - 1; r < hi;) {
    const int mid = (r + hi + 1) >> 1;
    if (p.q_row_start[mid] <= row) r = mid;
    else hi = mid - 1;
  }
  return r;
}

}  // namespace wisp
