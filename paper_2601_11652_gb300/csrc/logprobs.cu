// logprobs.cu -- log probabilities of given tokens with the rows' entropies and top alternatives
// (include/wisp_logprobs.h), and the tokens that a verified batch committed.
//
// With m = max z, s = sum exp(z - m) and w = sum exp(z - m) (z - m): log p(y) = z_y - m - log s and
// entropy = log s - w / s.
#include "common.cuh"
#include "sm100_ptx.cuh"
#include "wisp_logprobs.h"

#include <cmath>
#include <cstring>

namespace wisp {

namespace {

constexpr int kThreads = 512;
constexpr int kMaxTop = 32;
constexpr int kTokThreads = 1024;

struct LogprobParams {
  int rows, V, top_n;
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
__device__ __forceinline__ int id_of(uint64_t key) { return (int)(0xffffffffu - (uint32_t)key); }
__device__ __forceinline__ float logit_of(uint64_t key) {
  const uint32_t o = (uint32_t)(key >> 32);
  return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

__global__ void status_clear_kernel(DeviceStatus *st) {
  st->code = 0;
  st->pad = 0;
  st->request_id = 0;
}

// One CTA per row: the maximum, then the sums, then the alternatives one by one.
template <typename T>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const LogprobParams p) {
  __shared__ float s_f[2][kThreads / 32];
  __shared__ uint64_t s_k[kThreads / 32];
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int tok = p.tokens[row];
  const T *z = static_cast<const T *>(p.logits) + (int64_t)row * p.stride;
  auto write_all = [&](float v, int id) {
    if (tid == 0) {
      p.logprob[row] = v;
      if (p.entropy) p.entropy[row] = v;
    }
    if (tid < p.top_n) {
      p.top_tokens[(int64_t)row * p.top_n + tid] = id;
      p.top_logprobs[(int64_t)row * p.top_n + tid] = v;
    }
  };
  if (tok < 0) return write_all(0.0f, -1);
  if (tok >= p.V) {
    if (tid == 0) report(p.status, WISP_DEV_BAD_TOKEN, nullptr, row);
    return write_all(NAN, -1);
  }
  float m = -INFINITY;
  bool bad = false;
  for (int i = tid; i < p.V; i += kThreads) {
    const float v = element(z, i);
    bad |= !(v < INFINITY);
    m = fmaxf(m, v);
  }
  m = ptx::warp_max(m);
  if (lane == 0) s_f[0][warp] = m;
  bad = __syncthreads_or(bad);
  for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, s_f[0][w]);
  if (bad || m == -INFINITY) {
    if (tid == 0) report(p.status, WISP_DEV_BAD_PROB, nullptr, row);
    return write_all(NAN, -1);
  }
  __syncthreads();
  float s = 0.0f, a = 0.0f;
  for (int i = tid; i < p.V; i += kThreads) {
    const float d = element(z, i) - m, e = expf(d);
    s += e;
    if (d > -INFINITY) a += e * d;
  }
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    a += __shfl_xor_sync(0xffffffffu, a, o);
  }
  if (lane == 0) {
    s_f[0][warp] = s;
    s_f[1][warp] = a;
  }
  __syncthreads();
  s = a = 0.0f;
  for (int w = 0; w < kThreads / 32; ++w) {
    s += s_f[0][w];
    a += s_f[1][w];
  }
  const float ls = logf(s);
  if (tid == 0) {
    p.logprob[row] = element(z, tok) - m - ls;
    if (p.entropy) p.entropy[row] = ls - a / s;
  }
  uint64_t last = ~0ull;
  for (int t = 0; t < p.top_n; ++t) {
    uint64_t best = 0;
    for (int i = tid; i < p.V; i += kThreads) {
      const uint64_t k = key_of(element(z, i), i);
      if (k < last && k > best) best = k;
    }
    for (int o = 16; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
    if (lane == 0) s_k[warp] = best;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) best = max(best, s_k[w]);
    __syncthreads();
    if (tid == 0) {
      p.top_tokens[(int64_t)row * p.top_n + t] = best ? id_of(best) : -1;
      p.top_logprobs[(int64_t)row * p.top_n + t] = best ? logit_of(best) - m - ls : -INFINITY;
    }
    last = best;
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
  status_clear_kernel<<<1, 1, 0, s>>>(p.status);
  if (a->rows > 0) {
    if (a->logits_dtype == WISP_BF16)
      logprobs_kernel<uint16_t><<<a->rows, kThreads, 0, s>>>(p);
    else
      logprobs_kernel<float><<<a->rows, kThreads, 0, s>>>(p);
  }
  return cudaGetLastError() == cudaSuccess ? WISP_OK : WISP_ERR_CUDA;
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
