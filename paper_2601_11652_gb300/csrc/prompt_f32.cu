// prompt_f32.cu -- the attention of prompt_tc.cu for fp32 queries (fp32 cache, or e4m3 with scales; include/wisp_prompt.h), on the tensor cores.
//
// An fp32 value x of a row with largest magnitude 2^e' is 2^e (h + l): h and l halves (fp16), e = e' - 14, so that x is off by 2^-23 of itself, or
// 2^-38 of the row's largest where it is far below that.  A product of two such rows is 2^(e + e) (h h + h l + l h), three tensor-core products
// accumulated in fp32, the small ones first; what l l would add is 2^-24 of it.  So per tile of 64 keys:
//   S = Q K^T      M = 128 rows, N = 64 keys, K = D; a row's and a key's power of two are factors of its scores
//   P = 2^(S - m)  by 128 threads, a row each; a key's power of two (or scale) in V rides on P; again as h + l, in TMEM
//   O_t = P V      into TMEM from zero for every tile, and added to the row's O in registers in fp32.  (The tensor core's accumulation cuts
//                  bits off rather than rounding, a bias of up to 2^-24 per step: over a tile's 12 steps it stays at fp32's own error, over a
//                  long sequence it would not.)
// e4m3 codes are halves already: h alone, and two products instead of three.
// P is at most 2^14 (m moves where a tile's maximum is above that, which is 2^11 to 2^12 then), so that a weight's absolute steps, 2^-25 of
// these units, are 2^-36 of the row's largest.
//
// An item is one tile of 128 rows.  Persistent CTAs, 16 warps: 0-3 softmax and epilogue; 4-7 and 8-11 turn a K and a V tile into halves, in
// place; 12 and 13 issue S and P V; 14 takes items and loads K and V.  Every wait is bounded.
// Bound: the softmax warps, one per scheduler: with heads of 64 a tile's way through them (scores, weights, halves, the O before) is 2400 cycles
// alone and 3100 beside the warps that convert.  4096 tokens, 32 heads over 8 of 128: 588 us, 234 TFLOP/s of the definition's products (three
// times that on the tensor cores); over e4m3 409 us, 336 TFLOP/s; heads of 64 371 us, 185 TFLOP/s.
// Q by the warps that convert V, one item ahead, was no faster (609 to 612, over e4m3 400 to 415 us).  The instruction cache counts: the epilogue's way for V
// that is not finite as a loop instead of D copies of it took 42 KB of code and (D = 128) 43 us of 635.
#include "attn_merge.cuh"
#include "fp8.cuh"
#include "prompt.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>
#include <cstring>

namespace wisp {

namespace {

constexpr int kBT = 64;       // keys per tile
constexpr int kM = 128;       // rows
constexpr int kThreads = 512;
constexpr uint32_t kTmemCols = 512;  // S at 0 and 64, P at 128 and 192 (h, then l), O at 256 and 384
constexpr uint32_t kWaitCycles = 3000000000u;  // about one and a half seconds: a wait that long is a failure
// Sums of weights stay below 1, so that O never leaves the values' range: a tile adds 1/2 at most, as its largest score lies kRoom or more below the
// reference (log2), and with 1/2 in it the reference moves up by kRoom.  A new one lies kAbove above the largest score, a whole number, so that it
// differs from a tile to the next by d (see there) exactly.
constexpr float kRoom = 7.0f, kAbove = 10.0f;
constexpr int kUp = 21;       // P is weights times 2^kUp: at most 2^14
constexpr int kDown = 31;     // of keys' factors (log2)
constexpr int kLeast = -78;   // of d (see there): rows beyond are handed on, as their small weights times 2^d are no normal numbers
constexpr int kItemRing = 2;
constexpr int kSlots = 8;     // of the keys' factors, by tile: the eighth next tile is converted after this one's softmax is done

template <int D>
struct Cfg {
  static constexpr int HALVES = D / 64;
  static constexpr int QHALF = kM * 128, KHALF = kBT * 128;  // 64 elements of each row: [rows][128 B], swizzled
  static constexpr int QPART = HALVES * QHALF, KPART = HALVES * KHALF;  // h or l
  static constexpr int TILE = 2 * KPART;          // of K or V: fp32, then h and l
  static constexpr int NS = D == 128 ? 2 : 4;     // stages of K, and of V
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = 2 * QPART;
  static constexpr int OFF_V = OFF_K + NS * TILE;
  static constexpr int OFF_ST = OFF_V + NS * TILE;  // the epilogue's rows on their way out: 2 KB a warp
  static constexpr int OFF_BAR = OFF_ST + 4 * 2048;
  static constexpr int N_BAR = 56;
  static constexpr int OFF_RING = OFF_BAR + N_BAR * 8;
  static constexpr int OFF_MISC = OFF_RING + kItemRing * 64;
  static constexpr int OFF_KF = OFF_MISC + 64;             // float [kSlots][64]: factors of the keys' scores
  static constexpr int OFF_VF = OFF_KF + kSlots * kBT * 4; // float [kSlots][64]: factors of the keys' weights
  static constexpr int OFF_VE = OFF_VF + kSlots * kBT * 4; // int [kSlots]: exponent that the tile's factors are relative to
  static constexpr int OFF_VM = OFF_VE + kSlots * 4;       // float [2][4]: largest factors of the warps that convert V (or the first one's that is not zero), by tile
  static constexpr int OFF_KX = OFF_VM + 32;      // uint32 [kSlots][4]: keys with values that are not finite, 16 a warp (two bits each)
  static constexpr int OFF_ODD = OFF_KX + kSlots * 16;     // int [2][3][D] first positions that see NaN, +inf, -inf
  static constexpr int OFF_FAR = OFF_ODD + 2 * 3 * D * 4;  // uint8 [128]: the row has had a reference far from zero
  static constexpr int SMEM = OFF_FAR + kM + 1024;         // + slack to align the base to 1024
  static_assert(SMEM <= 227 * 1024, "shared memory of one CTA on sm_103a");
};

template <int D>
struct Bars {
  using C = Cfg<D>;
  static constexpr int KR_FULL = 0, K_FULL = C::NS, K_EMPTY = 2 * C::NS;  // raw, converted, free again
  static constexpr int VR_FULL = 3 * C::NS, V_FULL = 4 * C::NS, V_EMPTY = 5 * C::NS;
  static constexpr int Q_FULL = 6 * C::NS, Q_EMPTY = Q_FULL + 1;
  static constexpr int S_FULL = Q_EMPTY + 1, S_EMPTY = S_FULL + 2, P_FULL = S_EMPTY + 2, O_FULL = P_FULL + 2, O_EMPTY = O_FULL + 2;  // [2]
  static constexpr int IT_FULL = O_EMPTY + 2, IT_EMPTY = IT_FULL + kItemRing;
  static constexpr int ODD_FREE = IT_EMPTY + kItemRing;  // [2]
  static constexpr int CONV = ODD_FREE + 2;              // [2] the warps that convert K, V: a tile is in registers
  static constexpr int MMA_DONE = CONV + 2, FIN = MMA_DONE + 1;
  static_assert(FIN + 1 <= C::N_BAR, "barrier count");
};

__device__ __forceinline__ bool wait_bar(uint32_t b, uint32_t parity, volatile int *abort) {
  const uint32_t t0 = clock();
#pragma unroll 1
  while (!ptx::mbar_try_wait(b, parity)) {
    if (*abort) return false;
    if ((uint32_t)clock() - t0 > kWaitCycles) {
      *abort = 1;
      return false;
    }
  }
  return true;
}

// Instruction descriptor, kind::f16: fp32 accumulate, fp16 A (K-major) and B.
__device__ constexpr uint32_t idesc_f16(int N, bool b_mn_major) {
  return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kM >> 4) << 24);
}

// The exponent e of a row whose largest finite magnitude is `amax`: values times 2^-e stay below 2^15.  (2^-e and 2^e are normal numbers.)
__device__ __forceinline__ int row_exp(float amax) { return max((int)(__float_as_uint(amax) >> 23) - 127 - 14, -126); }
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
// The exponent of a factor (0 of 0).
__device__ __forceinline__ int exp_of(float x) { return x > 0.0f ? max((int)(__float_as_uint(x) >> 23) - 127, -126) : 0; }

__device__ __forceinline__ uint32_t h2(float a, float b) {
  const __half2 v = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t *>(&v);
}
// a, b as halves, and what is left of them
__device__ __forceinline__ void split2(float a, float b, uint32_t &h, uint32_t &l) {
  h = h2(a, b);
  const float2 f = h2_to_f2(h);
  l = h2(a - f.x, b - f.y);
}

}  // namespace

template <int D, bool KV8>
__global__ void __launch_bounds__(kThreads, 1)
    prompt_f32_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv,
                      const __grid_constant__ CUtensorMap tmk4, const __grid_constant__ CUtensorMap tmv4) {
  using C = Cfg<D>;
  using B = Bars<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = ptx::smem_u32(smem);
  const uint32_t bars = sbase + C::OFF_BAR;
  auto bar = [&](int i) -> uint32_t { return bars + 8 * i; };
  struct RingSlot {
    int it;
    int pad[3];
    WorkItem w;
  };
  static_assert(sizeof(RingSlot) <= 64, "item ring slot");
  RingSlot *s_ring = reinterpret_cast<RingSlot *>(smem + C::OFF_RING);
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + C::OFF_MISC);
  volatile int *s_abort = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 4);
  volatile int *s_isodd = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 8);  // [2]
  float *s_kf = reinterpret_cast<float *>(smem + C::OFF_KF), *s_vf = reinterpret_cast<float *>(smem + C::OFF_VF);
  int *s_ve = reinterpret_cast<int *>(smem + C::OFF_VE);
  float *s_vm = reinterpret_cast<float *>(smem + C::OFF_VM);
  uint32_t *s_kx = reinterpret_cast<uint32_t *>(smem + C::OFF_KX);
  int *s_odd = reinterpret_cast<int *>(smem + C::OFF_ODD);
  uint8_t *s_far = smem + C::OFF_FAR;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NS; ++i) {
      ptx::mbar_init(bar(B::KR_FULL + i), 1);
      ptx::mbar_init(bar(B::K_FULL + i), 4);
      ptx::mbar_init(bar(B::K_EMPTY + i), 1);
      ptx::mbar_init(bar(B::VR_FULL + i), 1);
      ptx::mbar_init(bar(B::V_FULL + i), 4);
      ptx::mbar_init(bar(B::V_EMPTY + i), 1);
    }
    ptx::mbar_init(bar(B::Q_FULL), 4);
    ptx::mbar_init(bar(B::Q_EMPTY), 1);
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(bar(B::S_FULL + b), 1);
      ptx::mbar_init(bar(B::S_EMPTY + b), 4);
      ptx::mbar_init(bar(B::P_FULL + b), 4);
      ptx::mbar_init(bar(B::O_FULL + b), 1);
      ptx::mbar_init(bar(B::O_EMPTY + b), 4);
      ptx::mbar_init(bar(B::ODD_FREE + b), 4);
      ptx::mbar_init(bar(B::CONV + b), 4);
    }
    for (int i = 0; i < kItemRing; ++i) {
      ptx::mbar_init(bar(B::IT_FULL + i), 1);
      ptx::mbar_init(bar(B::IT_EMPTY + i), 4 + 8 + 2);  // softmax, converting warps, MMA issuers
    }
    ptx::mbar_init(bar(B::MMA_DONE), 2);
    ptx::mbar_init(bar(B::FIN), kThreads / 32);
    *s_abort = 0;
    s_isodd[0] = s_isodd[1] = 0;
    ptx::fence_mbar_init();
  }
  for (int i = threadIdx.x; i < 2 * 3 * D; i += kThreads) s_odd[i] = INT32_MAX;
  if (threadIdx.x < kM) s_far[threadIdx.x] = 0;
  if (warp == 14 && lane == 0) {
    ptx::prefetch_tmap(&tmk);
    ptx::prefetch_tmap(&tmv);
    ptx::prefetch_tmap(&tmk4);
    ptx::prefetch_tmap(&tmv4);
  }
  __syncwarp();
  if (warp == 12) {
    ptx::tmem_alloc(s_tmem, kTmemCols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *s_tmem;
  // everything above may overlap the planner (programmatic dependent launch)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int g = p.Hq / p.Hkv;
  const int tile_pos = kM / g;  // positions of a tile

  // takes the next item from the ring: false at the end
  auto next_item = [&](uint32_t j, WorkItem &w, bool &ok) -> bool {
    const int slot = j % kItemRing;
    if (!wait_bar(bar(B::IT_FULL + slot), (j / kItemRing) & 1, s_abort)) { ok = false; return false; }
    const int it = s_ring[slot].it;
    w = s_ring[slot].w;
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bar(B::IT_EMPTY + slot));
    return it >= 0;
  };
  auto tiles_of = [](const WorkItem &w) { return (w.t1 - w.t0 + kBT - 1) / kBT; };

  bool ok = true;
  if (warp < 4) {
    // registers: 16 warps launch with 128 each, 512 a lane and warp of a scheduler = 248 + 104 + 104 + 56.  (Each split stands at the head of its
    // own branch: after a join the compiler counts with the least.)
    asm volatile("setmaxnreg.inc.sync.aligned.u32 248;");
    // ------------------------------------------------------------------ softmax and epilogue, a row per thread
    const int row = threadIdx.x;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const float scale = 1.4426950408889634f / sqrtf((float)D);
    const int pos0 = row / g, hh0 = row - pos0 * g;  // of this row within its tile
    uint32_t n = 0;   // tiles so far
    WorkItem w;
    for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
      const int nt = tiles_of(w);
      const bool mine = row < w.rows;
      const int pos = w.rg * tile_pos + pos0;
      const int end = min(w.t1, w.ctx + pos + 1);  // keys that it sees
      // ---- the row of Q as halves
      const float *qrow = static_cast<const float *>(p.q) + ((int64_t)(w.q0 + pos) * p.Hq + w.h * g + hh0) * D;
      float fq = 0.0f;
      if (!wait_bar(bar(B::Q_EMPTY), (j & 1) ^ 1, s_abort)) { ok = false; break; }
      {
        float4 v[D / 4];  // (all of its loads at once)
#pragma unroll
        for (int c = 0; c < D / 4; ++c) v[c] = mine ? __ldg(reinterpret_cast<const float4 *>(qrow) + c) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < D / 4; ++c) amax = fmaxf(fmaxf(fmaxf(amax, fabsf(v[c].x)), fmaxf(fabsf(v[c].y), fabsf(v[c].z))), fabsf(v[c].w));
        const int e = amax < INFINITY ? row_exp(amax) : 0;  // (a row with an infinity or a NaN becomes NaN in any case)
        // (a product of halves is below 2^37, a key's factor has 2^-kDown of it: up to fq, which has it back, nothing leaves fp32 that the score
        // does not.  Rows of a factor past 2^30, and keys of 2^-113, cannot be held so.)
        fq = pow2(min(e, 30) + kDown) * scale;
        if (e > 30) s_far[row] = 1;
        const float s = pow2(-e);
        uint8_t *line = smem + C::OFF_Q + row * 128;
#pragma unroll
        for (int c = 0; c < D; c += 8) {
          const float4 a = v[c / 4], b = v[c / 4 + 1];
          uint4 h, l;
          split2(a.x * s, a.y * s, h.x, l.x);
          split2(a.z * s, a.w * s, h.y, l.y);
          split2(b.x * s, b.y * s, h.z, l.z);
          split2(b.z * s, b.w * s, h.w, l.w);
          uint8_t *at = line + (c >> 6) * C::QHALF + ((((c >> 3) & 7) ^ (row & 7)) << 4);
          *reinterpret_cast<uint4 *>(at) = h;
          *reinterpret_cast<uint4 *>(at + C::QPART) = l;
        }
      }
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(B::Q_FULL));

      float m = -INFINITY, l = 0.0f;
      int ev = 0;  // of the tile before
      float2 o[D / 2];
#pragma unroll
      for (int i = 0; i < D / 2; ++i) o[i] = make_float2(0.0f, 0.0f);
      // adds tile k's P V
      auto collect = [&](uint32_t k) -> bool {
        const int b = k & 1;
        if (!wait_bar(bar(B::O_FULL + b), (k >> 1) & 1, s_abort)) return false;
        ptx::tc_fence_after();
        const float f = ev >= -126 ? pow2(ev) : __int_as_float(1 << (ev + 149));  // (no normal number)
        const float2 f2 = make_float2(f, f);
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          uint32_t x[32];
          ptx::tmem_ld32(tmem + lanes + 256 + b * 128 + c, x);
          ptx::tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 32; i += 2)
            o[(c + i) / 2] = __ffma2_rn(make_float2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), f2, o[(c + i) / 2]);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B::O_EMPTY + b));
        return true;
      };
      const int all = min(w.t1, w.ctx + w.rg * tile_pos + 1);  // keys that the first row sees
      for (int t = 0; t < nt; ++t, ++n) {
        const int b = n & 1, slot = n % kSlots;
        if (!wait_bar(bar(B::S_FULL + b), (n >> 1) & 1, s_abort)) { ok = false; break; }
        ptx::tc_fence_after();
        const int base = w.t0 + t * kBT;
        const float *vf = s_vf + slot * kBT;
        int d = 0;
        // Scores that are not those of the product are put right where they lie, in TMEM: the code of a tile's usual way, and of the other roles beside
        // it, has to stay in the instruction cache (with this in registers 4096 tokens took 668 us, 635 so; heads of 64 423 and 378).
        const uint4 kx = KV8 ? make_uint4(0, 0, 0, 0) : *reinterpret_cast<const uint4 *>(s_kx + slot * 4);
        if ((kx.x | kx.y | kx.z | kx.w) || base + kBT > all) {
          const uint32_t t_s = tmem + lanes + b * kBT;
          if (kx.x | kx.y | kx.z | kx.w) {
            // scores of keys with values that are not finite, from the values themselves
#pragma unroll 1
            for (int k = 0; k < kBT; ++k) {
              const uint32_t word = k < 16 ? kx.x : k < 32 ? kx.y : k < 48 ? kx.z : kx.w;
              if (!((word >> (2 * (k & 15))) & 3u) || base + k >= w.t1) continue;
              const int bid = __ldg(p.block_tables + (int64_t)w.r * p.max_blocks_per_seq + (base + k) / 16);
              const float *kr = static_cast<const float *>(p.k_cache) + (((int64_t)bid * p.Hkv + w.h) * 16 + (base + k) % 16) * D;
              float s = 0.0f;
              if (mine)
                for (int c = 0; c < D; ++c) s = fmaf(__ldg(qrow + c), __ldg(kr + c), s);
              __syncwarp();
              ptx::tmem_st1(t_s + k, __float_as_uint(s * (scale / fq)));
            }
            ptx::tmem_wait_st();
          }
          if (base + kBT > all) {
            const int seen = end - base;
#pragma unroll 1
            for (int c = 0; c < kBT; c += 16) {
              uint32_t y[16];
              ptx::tmem_ld16(t_s + c, y);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i)
                if (c + i >= seen) y[i] = 0xff800000u;
              ptx::tmem_st16(t_s + c, y);
            }
            ptx::tmem_wait_st();
            // Here V's factors are relative to the first that is not zero (elsewhere to the largest), and a row's weights are computed with 2^d, d the distance to
            // the largest factor that it sees (d goes back into their sum and into P V): what it does not see has no say in its bits.
            if (!wait_bar(bar(B::V_FULL + n % C::NS), (n / C::NS) & 1, s_abort)) { ok = false; break; }
            float most = 0.0f;
#pragma unroll 4
            for (int i = 0; i < kBT; ++i) most = fmaxf(most, i < seen ? vf[i] : 0.0f);
            d = most > 0.0f ? kUp - exp_of(most) : 0;
            if (d < kLeast) s_far[row] = 1;
          }
        }
        uint32_t x[2][32];
        ptx::tmem_ld32(tmem + lanes + b * kBT, x[0]);
        ptx::tmem_ld32(tmem + lanes + b * kBT + 32, x[1]);
        ptx::tmem_wait_ld();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B::S_EMPTY + b));
        const float *kf = s_kf + slot * kBT;
#pragma unroll
        for (int i = 0; i < kBT; i += 4) {
          const float4 f = *reinterpret_cast<const float4 *>(kf + i);
          uint32_t *y = &x[i >> 5][i & 31];
          const float2 u = __fmul2_rn(make_float2(__uint_as_float(y[0]), __uint_as_float(y[1])), make_float2(f.x, f.y));
          const float2 v = __fmul2_rn(make_float2(__uint_as_float(y[2]), __uint_as_float(y[3])), make_float2(f.z, f.w));
          y[0] = __float_as_uint(u.x);
          y[1] = __float_as_uint(u.y);
          y[2] = __float_as_uint(v.x);
          y[3] = __float_as_uint(v.y);
        }
        float mx[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          mx[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]));
#pragma unroll
          for (int i = 2; i < 32; i += 2) mx[c] = ptx::max3(mx[c], __uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1]));
        }
        const float top = fmaxf(mx[0], mx[1]) * fq;
        bool collected = t == 0;
        if (t == 0) {
          m = floorf(top) + kAbove;
        } else {
          const bool move = mine && (top > m - kRoom || l > 0.5f);
          if (__any_sync(0xffffffffu, move)) {
            // (the tile before still has the reference from before)
            collected = true;
            if (!collect(n - 1)) { ok = false; break; }
            const float to = top > m - kRoom ? floorf(top) + kAbove : m + kRoom;
            const float a = move ? ptx::ex2(m - to) : 1.0f;
            if (move && is_far(m)) s_far[row] = 1;
            if (move) m = to;
            l *= a;
#pragma unroll
            for (int i = 0; i < D / 2; ++i) o[i] = __fmul2_rn(o[i], make_float2(a, a));
          }
        }
        float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        if (!wait_bar(bar(B::V_FULL + n % C::NS), (n / C::NS) & 1, s_abort)) { ok = false; break; }  // (its factors)
        const float mm = (m == -INFINITY ? 0.0f : -m) + (float)d;  // (nothing seen so far: every weight is zero)
        const float2 m2 = make_float2(mm, mm), fq2 = make_float2(fq, fq);
#pragma unroll
        for (int c = 0; c < kBT; c += 16) {
          uint32_t ph[8], pl[8];
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const float4 f = *reinterpret_cast<const float4 *>(vf + c + i);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              const uint32_t *y = &x[(c + i) >> 5][((c + i) & 31) + 2 * q];
              const float2 a = __ffma2_rn(make_float2(__uint_as_float(y[0]), __uint_as_float(y[1])), fq2, m2);
              const float2 p2 = make_float2(ptx::ex2(a.x), ptx::ex2(a.y));
              sum[q] = __fadd2_rn(sum[q], p2);
              const float2 u = __fmul2_rn(p2, q == 0 ? make_float2(f.x, f.y) : make_float2(f.z, f.w));
              split2(u.x, u.y, ph[i / 2 + q], pl[i / 2 + q]);
            }
          }
          ptx::tmem_st8(tmem + lanes + 128 + b * 64 + c / 2, ph);
          ptx::tmem_st8(tmem + lanes + 128 + b * 64 + 32 + c / 2, pl);
        }
        l = fmaf((sum[0].x + sum[0].y) + (sum[1].x + sum[1].y), pow2(-d), l);
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B::P_FULL + b));
        if (!collected && !collect(n - 1)) { ok = false; break; }
        ev = s_ve[slot] - d;
      }
      if (!ok || !collect(n - 1)) { ok = false; break; }
      const bool far = is_far(m) || s_far[row];
      s_far[row] = 0;
      // ---- epilogue: the row through the warp's 2 KB in pieces of 64 bytes, so that four lanes store a row's piece together
      const bool part = w.poff >= 0;
      const float inv = part ? 1.0f : 1.0f / l;
      uint8_t *stage = smem + C::OFF_ST + warp * 2048;
      const int warp_rows = min(w.rows - warp * 32, 32);
      float *dst[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int r = warp * 32 + 8 * x + (lane >> 2), pj = r / g;
        dst[x] = (part ? p.partials + w.poff + (int64_t)r * D
                       : static_cast<float *>(p.out) + ((int64_t)(w.q0 + w.rg * tile_pos + pj) * p.Hq + w.h * g + (r - pj * g)) * D) +
                 (lane & 3) * 4;
      }
#pragma unroll
      for (int c = 0; c < D; c += 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float2 c1 = __fmul2_rn(o[(c + 4 * i) / 2], make_float2(inv, inv)), c2 = __fmul2_rn(o[(c + 4 * i) / 2 + 1], make_float2(inv, inv));
          *reinterpret_cast<float4 *>(stage + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) = make_float4(c1.x, c1.y, c2.x, c2.y);
        }
        __syncwarp();
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int r = 8 * x + (lane >> 2);
          if (r < warp_rows)
            __stcg(reinterpret_cast<float4 *>(dst[x] + c),
                   *reinterpret_cast<const float4 *>(stage + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4)));
        }
        __syncwarp();
      }
      if (s_isodd[j & 1]) {  // V held values that are not finite: what they make of the rows that see them (short code: see the scores)
        const int *so = s_odd + (j & 1) * 3 * D;
        float *at = part ? p.partials + w.poff + (int64_t)row * D : static_cast<float *>(p.out) + ((int64_t)(w.q0 + pos) * p.Hq + w.h * g + hh0) * D;
#pragma unroll 1
        for (int i = 0; i < D; ++i) {
          const bool nan = pos >= so[i], up = pos >= so[D + i], down = pos >= so[2 * D + i];
          if (mine && (nan || up || down)) at[i] = __ldcg(at + i) + (nan || (up && down) ? __uint_as_float(0x7fffffffu) : up ? INFINITY : -INFINITY);
        }
      }
      if (part && mine) {
        float *stat = p.partials + w.poff + (int64_t)w.rows * D + row;
        __stcg(stat, m);
        __stcg(stat + w.rows, far ? marked(l) : l);
      }
      if (far && mine) hand_on(p, w.q0 + pos, w.h * g + hh0);
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(B::ODD_FREE + (j & 1)));
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
    // ------------------------------------------------------------------ tiles into halves: K by warps 4-7, V by 8-11, two threads per key
    const bool is_k = warp < 8;
    const int id = (threadIdx.x & 127), key = id >> 1, half = id & 1;
    constexpr int E = D / 2;  // elements of a thread
    const int off = is_k ? C::OFF_K : C::OFF_V;
    const int full = is_k ? B::KR_FULL : B::VR_FULL, done = is_k ? B::K_FULL : B::V_FULL, conv = bar(B::CONV + (is_k ? 0 : 1));
    uint32_t n = 0, nb = 0;
    auto together = [&]() -> bool {  // the four warps
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(conv);
      return wait_bar(conv, nb++ & 1, s_abort);
    };
    WorkItem w;
    for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
      const int nt = tiles_of(w), ob = j & 1;
      const int all = min(w.t1, w.ctx + w.rg * tile_pos + 1);  // keys that the first row sees
      if (!is_k) {
        // this item's buffer of odd values: free, and cleared where it was used
        if (!wait_bar(bar(B::ODD_FREE + ob), ((j >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
        const bool used = s_isodd[ob] != 0;
        if (!together()) { ok = false; break; }  // (all have read the flag before one sets it)
        if (used) {
          for (int i = id; i < 3 * D; i += 128) s_odd[ob * 3 * D + i] = INT32_MAX;
          s_isodd[ob] = 0;
          if (!together()) { ok = false; break; }
        }
      }
      const int32_t *bt = p.block_tables + (int64_t)w.r * p.max_blocks_per_seq + w.t0 / 16;
      const int nblk = (w.t1 - w.t0 + 15) / 16;
      const float *scales = is_k ? p.k_scale : p.v_scale;
      auto page = [&](int t) -> int {
        const int rel = (kBT / 16) * t + key / 16;
        return KV8 && rel < nblk ? __ldg(bt + rel) : -1;
      };
      auto scale_of = [&](int b) { return KV8 && b >= 0 && b < p.num_blocks ? __ldg(scales + (int64_t)b * p.Hkv + w.h) : 0.0f; };
      float sc = scale_of(page(0));
      int b2 = page(1);
      for (int t = 0; t < nt; ++t, ++n) {
        const int st = n % C::NS, slot = n % kSlots;
        const float sc1 = scale_of(b2);
        b2 = page(t + 2);
        if (!wait_bar(bar(full + st), (n / C::NS) & 1, s_abort)) { ok = false; break; }
        uint8_t *tile = smem + off + st * C::TILE;
        const int at_key = w.t0 + t * kBT + key;
        const bool real = at_key < w.t1;  // (others are nobody's and count as zeros)
        const bool part = w.t0 + (t + 1) * kBT > all;
        uint32_t h[E / 2], l[KV8 ? 1 : E / 2];
        float f;  // the key's factor
        bool nonfinite = false;
        constexpr int G = E / 8;  // groups of eight elements, from one of its own on (so that lanes read different banks)
        constexpr int ES = KV8 ? 1 : 4;
        uint8_t *src = tile + key * (D * ES) + half * (E * ES);
        // Values that are not finite become zeros, remembered with the first position that sees them; the row is then read once more.
        // (A NaN code of K stays: its scores are NaN.)
        auto patch = [&]() {
          nonfinite = true;
#pragma unroll 1
          for (int i = 0; i < E; ++i) {
            int kind;
            if (KV8) {
              if ((src[i] & 0x7f) != 0x7f) continue;
              src[i] = 0;
              kind = 0;
            } else {
              float *x = reinterpret_cast<float *>(src) + i;
              if (fabsf(*x) < INFINITY) continue;
              kind = *x != *x ? 0 : *x > 0.0f ? 1 : 2;
              *x = 0.0f;
            }
            if (!is_k && real) {
              atomicMin(&s_odd[(ob * 3 + kind) * D + half * E + i], max(at_key - w.ctx, 0));
              s_isodd[ob] = 1;
            }
          }
        };
        if constexpr (KV8) {
#pragma unroll 1
          for (int pass = 0; pass < 2; ++pass) {
            __half2 any = __floats2half2_rn(0.0f, 0.0f);
            const __half2 zero = any;
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const uint2 u = *reinterpret_cast<const uint2 *>(src + ((i + id) % G) * 8);
              h[4 * i] = e4m3x2_to_h2(u.x & 0xffffu);
              h[4 * i + 1] = e4m3x2_to_h2(u.x >> 16);
              h[4 * i + 2] = e4m3x2_to_h2(u.y & 0xffffu);
              h[4 * i + 3] = e4m3x2_to_h2(u.y >> 16);
#pragma unroll
              for (int q = 0; q < 4; ++q) any = __hfma2(*reinterpret_cast<const __half2 *>(&h[4 * i + q]), zero, any);
            }
            if (is_k || __low2float(any) + __high2float(any) == 0.0f) break;
            patch();
          }
          f = sc;
        } else {
          float v[E], amax;
#pragma unroll 1
          for (int pass = 0; pass < 2; ++pass) {
            float any[4], am[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) any[i] = am[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < G; ++i) {
              const float4 a = *reinterpret_cast<const float4 *>(src + ((i + id) % G) * 32);
              const float4 b = *reinterpret_cast<const float4 *>(src + ((i + id) % G) * 32 + 16);
              v[8 * i] = a.x; v[8 * i + 1] = a.y; v[8 * i + 2] = a.z; v[8 * i + 3] = a.w;
              v[8 * i + 4] = b.x; v[8 * i + 5] = b.y; v[8 * i + 6] = b.z; v[8 * i + 7] = b.w;
            }
#pragma unroll
            for (int i = 0; i < E; i += 8)
#pragma unroll
              for (int q = 0; q < 4; ++q) {  // (NaN where a value is not finite)
                any[q] = fmaf(v[i + 2 * q], 0.0f, fmaf(v[i + 2 * q + 1], 0.0f, any[q]));
                am[q] = ptx::max3(am[q], fabsf(v[i + 2 * q]), fabsf(v[i + 2 * q + 1]));
              }
            amax = fmaxf(fmaxf(am[0], am[1]), fmaxf(am[2], am[3]));
            if ((any[0] + any[1]) + (any[2] + any[3]) == 0.0f) break;
            patch();
          }
          amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
          const int e = row_exp(amax);
          const float s = pow2(-e);
          f = is_k || amax > 0.0f ? pow2(e) : 0.0f;
#pragma unroll
          for (int i = 0; i < E; i += 2) {
            const float2 y = __fmul2_rn(make_float2(v[i], v[i + 1]), make_float2(s, s));
            split2(y.x, y.y, h[i / 2], l[i / 2]);
          }
        }
        if (!real) f = 0.0f;
        if (is_k) {
          if (half == 0) s_kf[slot * kBT + key] = real ? fmaxf(f * pow2(-kDown), 0x1p-149f) : 1.0f;  // (not zero: masked scores are -inf before)
          if (!KV8) {
            const uint32_t odd = __ballot_sync(0xffffffffu, nonfinite && real);
            if (lane == 0) s_kx[slot * 4 + warp - 4] = odd;
          }
        } else {
          // what the tile's factors are relative to: the power of two of the largest, or where some row does not see all keys, of
          // the first key whose V is not zero (rows that do not see it have nothing from this tile)
          const uint32_t some = __ballot_sync(0xffffffffu, f > 0.0f);
          const float wm = part ? __shfl_sync(0xffffffffu, f, some ? __ffs(some) - 1 : 0) : ptx::warp_max(f);
          if (lane == 0) s_vm[(n & 1) * 4 + warp - 8] = wm;
        }
        if (!together()) { ok = false; break; }  // the tile is in registers
        if (!is_k && half == 0) {
          // (a factor that is 2^120 of it or more counts for rows that do not see it)
          const float4 m4 = *reinterpret_cast<const float4 *>(s_vm + (n & 1) * 4);
          const float first = m4.x > 0.0f ? m4.x : m4.y > 0.0f ? m4.y : m4.z > 0.0f ? m4.z : m4.w;
          const int e = exp_of(part ? first : fmaxf(fmaxf(m4.x, m4.y), fmaxf(m4.z, m4.w))), e2 = e / 2;
          s_vf[slot * kBT + key] = fminf(f * pow2(-e2) * pow2(e2 - e + kUp), 0x1p120f);
          if (id == 0) s_ve[slot] = e - kUp;
        }
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const int c = half * G + (i + id) % G;  // chunk of the row
          uint8_t *at = tile + (c >> 3) * C::KHALF + key * 128 + (((c & 7) ^ (key & 7)) << 4);
          *reinterpret_cast<uint4 *>(at) = make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
          if constexpr (!KV8) *reinterpret_cast<uint4 *>(at + C::KPART) = make_uint4(l[4 * i], l[4 * i + 1], l[4 * i + 2], l[4 * i + 3]);
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(done + st));
        sc = sc1;
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 14) {
      // ------------------------------------------------------------------ items, K, V
      const int n_items = p.header->n_items;
      int claimed = (int)blockIdx.x < n_items ? (int)blockIdx.x : -1;  // the first item is this CTA's by its index
      auto claim = [&]() {
        if (lane == 0 && claimed == -2) {
          claimed = atomicAdd(&p.header_mut->next_item, 1);
          if (claimed >= n_items) claimed = -1;
        }
      };
      constexpr uint32_t kRaw = KV8 ? kBT * D : kBT * D * 4;
      uint32_t nk = 0, nv = 0;
      for (uint32_t j = 0;; ++j) {
        const int slot = j % kItemRing;
        if (!wait_bar(bar(B::IT_EMPTY + slot), ((j / kItemRing) & 1) ^ 1, s_abort)) { ok = false; break; }
        claim();
        int it = 0;
        if (lane == 0) {
          it = claimed;
          claimed = -2;
          s_ring[slot].it = it;
          if (it >= 0) s_ring[slot].w = item_at(p, it);
        }
        it = __shfl_sync(0xffffffffu, it, 0);
        __syncwarp();
        const WorkItem w = s_ring[slot].w;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B::IT_FULL + slot));
        if (it < 0) break;
        const int32_t *bt = p.block_tables + (int64_t)w.r * p.max_blocks_per_seq + w.t0 / 16;
        const int nblk = (w.t1 - w.t0 + 15) / 16, nt = tiles_of(w);
        auto fetch = [&](int tile8) -> int {  // block ids of eight tiles, a lane each
          const int i = tile8 * 32 + lane;
          return i < nblk ? __ldg(bt + i) : -1;
        };
        int cur = -1, next = fetch(0);
        auto load = [&](bool is_k, int t) -> bool {
          const uint32_t n = is_k ? nk : nv;
          const int s = n % C::NS;
          const int full = (is_k ? B::KR_FULL : B::VR_FULL) + s, empty = (is_k ? B::K_EMPTY : B::V_EMPTY) + s;
          const int rel = 4 * t + (lane & 3);
          int bid = __shfl_sync(0xffffffffu, cur, rel & 31);
          if (!wait_bar(bar(empty), ((n / C::NS) & 1) ^ 1, s_abort)) return false;
          const bool valid = bid >= 0 && bid < p.num_blocks;
          if (is_k && lane < 4 && rel < nblk && !valid) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, w.r);
          ++(is_k ? nk : nv);
          const uint32_t dst = sbase + (is_k ? C::OFF_K : C::OFF_V) + s * C::TILE;
          const int b0 = __shfl_sync(0xffffffffu, bid, 0);
          const bool row4 = __ballot_sync(0xffffffffu, lane < 4 && valid && bid == b0 + lane) == 0xfu;
          if (!valid) bid = p.num_blocks;  // past the item (or invalid): out-of-range box, reads zeros
          int bids[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) bids[x] = __shfl_sync(0xffffffffu, bid, x);
          if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(bar(full), kRaw);
            if (row4) {
              ptx::tma_load_4d(dst, is_k ? &tmk4 : &tmv4, bar(full), 0, 0, w.h, b0);
            } else {
#pragma unroll
              for (int x = 0; x < 4; ++x) ptx::tma_load_4d(dst + x * (kRaw / 4), is_k ? &tmk : &tmv, bar(full), 0, 0, w.h, bids[x]);
            }
          }
          __syncwarp();
          return true;
        };
        for (int t = 0; t < nt && ok; ++t) {
          if ((t & 7) == 0) {
            cur = next;
            next = fetch((t >> 3) + 1);
          }
#pragma unroll 1
          for (int kv = 0; kv < 2 && ok; ++kv) ok = load(kv == 0, t);
          if (t == max(nt - 4, 0)) claim();  // the next item, early enough to hide the way to it
        }
        if (!ok) break;
      }
      asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      // drain: what was issued must land before the CTA's shared memory goes away
      if (lane == 0) {
#pragma unroll 1
        for (int x = 0; x < 2; ++x) {
          const int full = x ? B::VR_FULL : B::KR_FULL;
          const uint32_t n = x ? nv : nk;
#pragma unroll 1
          for (uint32_t k = 0; k < C::NS && k < n; ++k) {
            const uint32_t t0 = clock();
            while (!ptx::mbar_try_wait(bar(full + (n - 1 - k) % C::NS), ((n - 1 - k) / C::NS) & 1) && (uint32_t)clock() - t0 < kWaitCycles) {
            }
          }
        }
      }
    } else if (warp == 12 || warp == 13) {
      // ------------------------------------------------------------------ MMA issuers: 12 S, 13 P V
      const bool is_s = warp == 12;
      const uint32_t idesc = is_s ? idesc_f16(kBT, false) : idesc_f16(D, true);
      uint32_t n = 0;
      WorkItem w;
      for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
        const int nt = tiles_of(w);
        if (is_s && !wait_bar(bar(B::Q_FULL), j & 1, s_abort)) { ok = false; break; }
        for (int t = 0; t < nt; ++t, ++n) {
          const int st = n % C::NS, b = n & 1;
          const uint32_t round = (n / C::NS) & 1, half = (n >> 1) & 1;
          if (is_s) {
            if (!wait_bar(bar(B::K_FULL + st), round, s_abort) || !wait_bar(bar(B::S_EMPTY + b), half ^ 1, s_abort)) { ok = false; break; }
            if (ptx::elect_one()) {
              ptx::tc_fence_after();
              const uint64_t qd = ptx::sdesc_sw128(sbase + C::OFF_Q, 16, 1024);
              const uint64_t kd = ptx::sdesc_sw128(sbase + C::OFF_K + st * C::TILE, 16, 1024);
              // l h, h l, h h
#pragma unroll
              for (int x = 0; x < 3; ++x) {
                if (KV8 && x == 1) continue;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
                  ptx::umma_f16(tmem + b * kBT, qd + (((x == 0 ? C::QPART : 0) + (ks >> 2) * C::QHALF + (ks & 3) * 32) >> 4),
                                kd + (((x == 1 ? C::KPART : 0) + (ks >> 2) * C::KHALF + (ks & 3) * 32) >> 4), idesc, x > 0 || ks > 0);
              }
              ptx::umma_commit(bar(B::S_FULL + b));
              ptx::umma_commit(bar(B::K_EMPTY + st));
              if (t == nt - 1) ptx::umma_commit(bar(B::Q_EMPTY));
            }
          } else {
            if (!wait_bar(bar(B::V_FULL + st), round, s_abort) || !wait_bar(bar(B::O_EMPTY + b), half ^ 1, s_abort) ||
                !wait_bar(bar(B::P_FULL + b), half, s_abort)) {
              ok = false;
              break;
            }
            if (ptx::elect_one()) {
              ptx::tc_fence_after();
              const uint64_t vd = ptx::sdesc_sw128(sbase + C::OFF_V + st * C::TILE, C::KHALF, 1024);
#pragma unroll
              for (int x = 0; x < 3; ++x) {
                if (KV8 && x == 1) continue;
#pragma unroll
                for (int ks = 0; ks < kBT / 16; ++ks)
                  ptx::umma_f16_ts(tmem + 256 + b * 128, tmem + 128 + b * 64 + (x == 0 ? 32 : 0) + ks * 8,
                                   vd + (((x == 1 ? C::KPART : 0) + ks * 16 * 128) >> 4), idesc, x > 0 || ks > 0);
              }
              ptx::umma_commit(bar(B::O_FULL + b));
              ptx::umma_commit(bar(B::V_EMPTY + st));
            }
          }
          __syncwarp();
        }
      }
      if (ptx::elect_one()) {
        // every MMA issued must finish before the TMEM is released
        ptx::umma_commit(bar(B::MMA_DONE));
        const uint32_t t0 = clock();
        while (!ptx::mbar_try_wait(bar(B::MMA_DONE), 0) && (uint32_t)clock() - t0 < kWaitCycles) {
        }
      }
    }
  }

  if (!ok && lane == 0) report(p.status, WISP_DEV_TIMEOUT, p.request_ids, -1);
  // teardown: the TMEM is freed once every warp has said that it is done with it
  __syncwarp();
  ptx::tc_fence_before();
  if (lane == 0) ptx::mbar_arrive(bar(B::FIN));
  if (warp == 12) {
    const uint32_t t0 = clock();
    while (!ptx::mbar_try_wait(bar(B::FIN), 0) && (uint32_t)clock() - t0 < kWaitCycles) {
    }
    __syncwarp();
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------------------- host side
namespace {

PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;

cudaError_t get_encode() {
  if (g_encode) return cudaSuccess;
  void *fn = nullptr;
  cudaDriverEntryPointQueryResult q;
  const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
  if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
  g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  return cudaSuccess;
}

// The paged pool [num_blocks, Hkv, 16, D] as it is, in boxes of `pages` pages of one head.
cudaError_t encode(CUtensorMap *map, const AttnParams &p, const void *base, int pages) {
  const bool codes = p.k_scale != nullptr;
  const cuuint64_t es = codes ? 1 : 4, D = p.D;
  const cuuint64_t dims[4] = {D, 16, (cuuint64_t)p.Hkv, (cuuint64_t)p.num_blocks};
  const cuuint64_t strides[3] = {D * es, 16 * D * es, (cuuint64_t)p.Hkv * 16 * D * es};
  const cuuint32_t box[4] = {(cuuint32_t)p.D, 16, 1, (cuuint32_t)pages}, ones[4] = {1, 1, 1, 1};
  const CUresult r = g_encode(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 4, const_cast<void *>(base), dims,
                              strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, bool KV8>
cudaError_t launch(const AttnParams &p, int grid, cudaStream_t s) {
  CUtensorMap tk, tv, tk4, tv4;
  cudaError_t e = encode(&tk, p, p.k_cache, 1);
  if (e == cudaSuccess) e = encode(&tv, p, p.v_cache, 1);
  if (e == cudaSuccess) e = encode(&tk4, p, p.k_cache, 4);
  if (e == cudaSuccess) e = encode(&tv4, p, p.v_cache, 4);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = Cfg<D>::SMEM;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, prompt_f32_kernel<D, KV8>, p, tk, tv, tk4, tv4);
}

template <int D, bool KV8>
cudaError_t setup() {
  return cudaFuncSetAttribute(prompt_f32_kernel<D, KV8>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::SMEM);
}

}  // namespace

cudaError_t prompt_f32_setup() {
  cudaError_t e = get_encode();
  if (e == cudaSuccess) e = setup<128, false>();
  if (e == cudaSuccess) e = setup<128, true>();
  if (e == cudaSuccess) e = setup<64, false>();
  return e == cudaSuccess ? setup<64, true>() : e;
}

cudaError_t prompt_f32_launch(const AttnParams &p, int grid, cudaStream_t s) {
  if (p.k_scale) return p.D == 128 ? launch<128, true>(p, grid, s) : launch<64, true>(p, grid, s);
  return p.D == 128 ? launch<128, false>(p, grid, s) : launch<64, false>(p, grid, s);
}

}  // namespace wisp
