// attn_kv8_tc.cu -- tensor-core paged GQA attention of the verification forward over an e4m3 cache, bf16 queries.
//
// Same contract as attn_tc.cu (request r's k+1 new queries over its L_total paged keys, query j seeing keys
// 0..c_r + j), with K and V of a page of one head worth code * scale (include/wisp_kv8.h).  K and V go from HBM to the
// tensor core as they are:
//   S^T = K Q^T       (M = 128 keys of a tile, N = the item's rows, K = D),     kind::f8f6f4
//   O^T = V^T P^T     (M = D, N = rows, K = 128 keys)
// The other operand of each product is split into two e4m3 parts, x = (hi + lo / 16) 2^e, that lie side by side along
// N: 4 + 4 significant bits, what a bf16 value has, for one pass over K or V in shared memory; the reader of an
// accumulator adds its two halves.  e is a power of two per query row, and for P per row and tile: P = 2^(s - m + 8)
// with m the row's maximum over the tile's 128 keys, so that each tile keeps 8 bits down to 2^-13 of its own largest
// weight and 2^-22 absolutely, whatever other tiles hold (with one exponent for a whole sequence, a key that outweighs the
// others by 2^17 would cost them their bits).  The key's page scales enter as a factor of S and, as log2, in s,
// so that V's scale rides on P.  PV products of different tiles have different exponents: each goes to a TMEM
// accumulator of its own and the correction warps add it to their running sums with 2^(m - M).
//
// Persistent CTAs (one per SM) take work items (request, KV head, key chunk, row group) from the plan's counter,
// longest first.  Warp roles:
//   * warp 2 takes items just in time and publishes them in a 4-slot ring; warps 17-19 split an item's query rows into
//     one of two Q buffers;
//   * warps 0 and 3 (K and V producers) stream tiles of 128 tokens with TMA, one 16 KB box when the tile's eight pages
//     are consecutive in the pool, else one box per page; warp 0 also brings the pages' scales;
//   * warps 1 and 16 issue the MMAs: S^T and PV;
//   * warps 4-7 and 12-15 (softmax): two groups that take turns by tile, one warp per TMEM lane quadrant: a thread
//     holds one key's scores for all rows.  A group's four warps agree on the tile's row maxima through shared memory;
//   * warps 8-11 (correction): thread d keeps head-dim index d of every row's O; they also write the outputs or the
//     (O, m, l) partials of a split item, whose last chunk merges all.
//
// Every mbarrier wait is bounded in time; an expired wait records WISP_DEV_TIMEOUT and the CTA drains.
#include "attn_merge.cuh"
#include "fp8.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>
#include <cstring>
#include <mutex>
#include <type_traits>

namespace wisp {

namespace {

constexpr int kBT = 128;            // KV tokens per tile (the M of S^T)
constexpr int kNR = kTcRowsPerItem; // query rows per item at most
constexpr int kThreads = 896;
constexpr int kSoftmaxWarps = 16;
constexpr int kQWarps = 3;
constexpr uint32_t kTmemCols = 512; // S^T[4] at columns 0, 64, 128, 192, O^T[2] (hi and lo rows) at 256 / 384
constexpr long long kWaitCycles = 4000000000LL;  // about two seconds: a wait that long is a failure
constexpr uint32_t kAhead = 3;      // the item loader takes the next item when the K producer is this many tiles from
                                    // the end of what is published
constexpr float kHead = 6.0f;       // log2 of P at a row's reference
constexpr float kUp = 2.6f;         // a tile's maximum may be this far above the reference (with its rounding: P <= 431, e4m3
                                    // holds 448)
constexpr float kDown = 4.0f;       // ... and this far below
constexpr float kFar = 30.0f;       // what is this far below the largest reference so far weighs nothing
constexpr float kLazy = 64.0f;      // the correction's running references follow a row's when it is this far above (log2)
constexpr float kLeastScaleLog2 = -100.0f;  // a V scale of 0 weighs as 2^-100, so that its keys still count in the sums
static_assert(kNR == 64, "TMEM and shared-memory layout assume 64 rows per item");

template <int D>
struct Cfg {
  static constexpr int KV_TILE = kBT * D;       // bytes of K (or V) of one tile
  static constexpr int Q_BYTES = 2 * kNR * D;   // hi rows, then lo rows
  static constexpr int P_BYTES = kBT * 2 * kNR; // [128 tokens][hi rows, lo rows]
  static constexpr int NSK = D == 128 ? 3 : 6;  // K ring stages
  static constexpr int NSV = D == 128 ? 3 : 6;  // V ring stages
  static constexpr int SC = 16;                 // slots of the scales' ring: tile n in n % SC
  static constexpr int RF = 8;                  // slots of the row factors' ring: item li in li % RF
  static constexpr int RING = 4;                // slots of the item ring
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + 2 * Q_BYTES;
  static constexpr int OFF_V = OFF_K + NSK * KV_TILE;
  static constexpr int OFF_P = OFF_V + NSV * KV_TILE;
  static constexpr int OFF_BAR = OFF_P + 4 * P_BYTES;
  static constexpr int N_BAR = 2 * NSK + 2 * NSV + 28 + 2 * RING + 7;
  static constexpr int OFF_SC = (OFF_BAR + N_BAR * 8 + 15) / 16 * 16;  // float2 [SC][8]: a page's K and V scale
  static constexpr int OFF_RF = OFF_SC + SC * 64;                      // float [RF][64]
  static constexpr int OFF_RED = OFF_RF + RF * kNR * 4;                // [4 groups][2][4][8] row maxima per quadrant, bf16 pairs
  static constexpr int OFF_MW = OFF_RED + 4 * 2 * 4 * 8 * 4;           // float [16][16] per warp: kHead - reference
  static constexpr int OFF_M = OFF_MW + kSoftmaxWarps * 16 * 4;        // float [8][64] references of tile n in n % 8
  static constexpr int OFF_CW = OFF_M + 8 * kNR * 4;                   // float [4][64] per correction warp
  static constexpr int OFF_HL = OFF_CW + 4 * kNR * 4;                  // float [2][4 groups][4][16] row-sum shares
  static constexpr int OFF_LR = OFF_HL + 2 * 4 * 4 * 16 * 4;           // float [2][4 groups][16] their references
  static constexpr int OFF_NAN = OFF_LR + 2 * 4 * 16 * 4;              // int [2][D] first row that a NaN value reaches
  static constexpr int OFF_MISC = OFF_NAN + 2 * D * 4;
  static constexpr int OFF_RING = OFF_MISC + 32;
  static constexpr int SMEM = OFF_RING + RING * 64 + 1024;             // + slack to align the base to 1024
  static_assert(SMEM <= 227 * 1024, "shared memory of one CTA on sm_103a");
  static_assert(OFF_K % 1024 == 0 && OFF_V % 1024 == 0 && OFF_P % 1024 == 0 && OFF_RING % 16 == 0, "alignment");
  // a slot is written again once S^T of its tile (or item) and of the tiles NSK (items 2) after it has been read
  static_assert(SC >= NSK + 4 && RF >= 5, "rings");
};

// The CTA's mbarriers: shared-memory addresses at constant offsets from one base.
template <int D>
struct Bars {
  using C = Cfg<D>;
  uint32_t base;
  static constexpr int K_FULL = 0, K_EMPTY = C::NSK, V_FULL = 2 * C::NSK, V_EMPTY = V_FULL + C::NSV;
  static constexpr int Q_FULL = V_EMPTY + C::NSV, Q_EMPTY = Q_FULL + 2, S_FULL = Q_EMPTY + 2, S_EMPTY = S_FULL + 4;
  static constexpr int P_FULL = S_EMPTY + 4;   // [4] P of tile n in buffer n & 3
  static constexpr int P_EMPTY = P_FULL + 4;   // [4] PV of tile n is done
  static constexpr int O_FULL = P_EMPTY + 4;   // [2] ... and its O is complete
  static constexpr int O_EMPTY = O_FULL + 2;   // [2] the correction warps have read it
  static constexpr int EP_FULL = O_EMPTY + 2;  // [2] per item parity: the softmax warps handed their sums over
  static constexpr int EP_EMPTY = EP_FULL + 2; // [2] the correction warps have read them
  static constexpr int MMA_DONE = EP_EMPTY + 2;  // the two MMA issuers, at the end
  static constexpr int IT_FULL = MMA_DONE + 1, IT_EMPTY = IT_FULL + C::RING;
  static constexpr int EGRP = IT_EMPTY + C::RING;  // the correction warps
  static constexpr int RED = EGRP + 1;         // [4] per softmax group: its four warps, once per tile
  static constexpr int FIN = RED + 4;          // every warp, once: its last access to TMEM is done
  static_assert(FIN + 1 <= C::N_BAR, "barrier count");
  __device__ __forceinline__ uint32_t at(int i) const { return base + 8 * i; }
};

__device__ __forceinline__ bool wait_bar(uint32_t b, uint32_t parity, volatile int *abort) {
  if (ptx::mbar_try_wait(b, parity)) return true;
  const long long t0 = clock64();
  while (true) {
    if (ptx::mbar_try_wait(b, parity)) return true;
    if (*abort) return false;
    if (clock64() - t0 > kWaitCycles) {
      *abort = 1;
      return false;
    }
  }
}

__device__ __forceinline__ bool item_ok(const AttnParams &p, const WorkItem &w) {
  // (a refused request's items are empty)
  return w.r >= 0 && w.r < p.B && w.t1 > w.t0 && w.rows > 0 && w.rows <= kNR &&
         w.row0 >= 0 && w.nrg >= 1 && w.nrg <= p.row_groups && w.rg >= 0 && w.rg < w.nrg;
}

// Transposing sum over the 32 lanes of a warp (v is consumed): lanes i and 16 + i get the sum over all lanes of v[i].
__device__ __forceinline__ float warp_transpose_sum(float (&v)[16], int lane) {
#pragma unroll
  for (int w = 8; w >= 1; w >>= 1) {
    const bool up = (lane & w) != 0;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const float keep = up ? v[i + w] : v[i];
      const float send = up ? v[i] : v[i + w];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
    }
  }
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 16);
}

__device__ __forceinline__ uint32_t bmax2(uint32_t a, uint32_t b) {  // NaN never wins
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Transposing maximum of bf16 pairs over the 32 lanes of a warp (v is consumed): lane i gets that of v[i & 7].
__device__ __forceinline__ uint32_t warp_transpose_max(uint32_t (&v)[8], int lane) {
#pragma unroll
  for (int w = 4; w >= 1; w >>= 1) {
    const bool up = (lane & w) != 0;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const uint32_t keep = up ? v[i + w] : v[i];
      const uint32_t send = up ? v[i] : v[i + w];
      v[i] = bmax2(keep, __shfl_xor_sync(0xffffffffu, send, w));
    }
  }
  const uint32_t y = bmax2(v[0], __shfl_xor_sync(0xffffffffu, v[0], 8));
  return bmax2(y, __shfl_xor_sync(0xffffffffu, y, 16));
}

__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The parts of an item's rows (rounded up to 8), one, two or four of at most 16 rows, in whole units of 8: part i starts
// at row(i).
struct Parts {
  int n, units;
  __device__ __forceinline__ explicit Parts(int nrow) : n(nrow <= 16 ? 1 : nrow <= 32 ? 2 : 4), units(nrow / 8) {}
  __device__ __forceinline__ int row(int i) const { return i * units / n * 8; }
};
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// hi and lo codes (two of each) of two values of magnitude at most 448: x = hi + lo, or hi + lo / 16 (S16)
template <bool S16>
__device__ __forceinline__ void split2(float a, float b, uint32_t &hi, uint32_t &lo) {
  hi = e4m3x2(a, b);
  const uint32_t h = e4m3x2_to_h2(hi);
  __half2 r = __hsub2(__floats2half2_rn(a, b), *reinterpret_cast<const __half2 *>(&h));
  if (S16) r = __hmul2(r, __floats2half2_rn(16.0f, 16.0f));
  lo = e4m3x2_h(*reinterpret_cast<const uint32_t *>(&r));
}

// Byte offset of 16-byte chunk c of row `row` in a swizzled tile with rows of D bytes.
template <int D>
__device__ __forceinline__ uint32_t swz(int row, int c) {
  return row * D + ((c ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4);
}
template <int D>
__device__ __forceinline__ uint64_t sdesc(uint32_t addr) {  // eight rows of D bytes are D * 8 apart
  return D == 128 ? ptx::sdesc_sw128(addr, D == 128 ? 16 : 0, 1024) : ptx::sdesc_sw64(addr, 0, 512);
}

}  // namespace

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    attn_kv8_tc_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap tmk,
                       const __grid_constant__ CUtensorMap tmv, const __grid_constant__ CUtensorMap tmk8,
                       const __grid_constant__ CUtensorMap tmv8) {
  using C = Cfg<D>;
  using BR = Bars<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t *smem = smem_raw + ((1024u - (ptx::smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t sbase = ptx::smem_u32(smem);
  const BR B{sbase + C::OFF_BAR};
  float2 *s_sc = reinterpret_cast<float2 *>(smem + C::OFF_SC);
  float *s_rf = reinterpret_cast<float *>(smem + C::OFF_RF);
  float *s_m = reinterpret_cast<float *>(smem + C::OFF_M);
  float *s_hl = reinterpret_cast<float *>(smem + C::OFF_HL);
  float *s_lr = reinterpret_cast<float *>(smem + C::OFF_LR);
  int *s_nan = reinterpret_cast<int *>(smem + C::OFF_NAN);
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + C::OFF_MISC);
  volatile int *s_abort = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 4);
  volatile int *s_last = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 8);
  volatile uint32_t *s_issued = reinterpret_cast<volatile uint32_t *>(smem + C::OFF_MISC + 12);  // K tiles issued
  struct RingSlot {
    int it;
    int pad[3];
    WorkItem w;
  };
  static_assert(sizeof(RingSlot) <= 64, "item ring slot");
  RingSlot *s_ring = reinterpret_cast<RingSlot *>(smem + C::OFF_RING);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    auto init = [&](int first, int n, int count) {
      for (int i = 0; i < n; ++i) ptx::mbar_init(B.at(first + i), count);
    };
    init(BR::K_FULL, C::NSK, 2);  // the tile's bytes, its scales
    init(BR::K_EMPTY, C::NSK + 2 * C::NSV, 1);
    init(BR::Q_FULL, 2, kQWarps);
    init(BR::Q_EMPTY, 2, 1);
    init(BR::S_FULL, 4, 1);
    init(BR::S_EMPTY, 4, 16);  // the warps of the tile's softmax groups, four, two or one arrival each
    init(BR::P_FULL, 4, 16);
    init(BR::P_EMPTY, 4, 1);
    init(BR::O_FULL, 2, 1);
    init(BR::O_EMPTY, 2, 4);   // the correction warps
    init(BR::EP_FULL, 2, kSoftmaxWarps);
    init(BR::EP_EMPTY, 2, 4);
    init(BR::MMA_DONE, 1, 2);
    init(BR::IT_FULL, C::RING, 1);
    init(BR::IT_EMPTY, C::RING, 4 + kQWarps + kSoftmaxWarps + 4);  // KV producers, MMA issuers, Q, softmax, correction
    init(BR::EGRP, 1, 4);
    init(BR::RED, 4, 4);       // a group's warps
    init(BR::FIN, 1, kThreads / 32);
    *s_issued = 0;
    *s_abort = 0;
    ptx::fence_mbar_init();
  }
  for (int i = threadIdx.x; i < 2 * D; i += kThreads) s_nan[i] = INT32_MAX;
  if (warp == 0 && lane == 0) {
    ptx::prefetch_tmap(&tmk);
    ptx::prefetch_tmap(&tmv);
    ptx::prefetch_tmap(&tmk8);
    ptx::prefetch_tmap(&tmv8);
  }
  __syncwarp();
  if (warp == 1) {
    ptx::tmem_alloc(s_tmem, kTmemCols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *s_tmem;

  // everything above may overlap the planner (programmatic dependent launch); the plan is read
  // only once the planner's grid has completed and its writes are visible
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n_items = p.header->n_items;
  if ((int)blockIdx.x >= p.header->attn_ctas) {
    // the planner leaves this SM to the acceptance pass of the same step: nothing was issued yet
    if (warp == 1) ptx::tmem_dealloc(tmem, kTmemCols);
    return;
  }
  const int g = p.Hq / p.Hkv;
  // a query row's position and head: row / g for rows below 128 as a product (exact: 127 (g - 1) < 2^16)
  const unsigned gm = (65536u + g - 1) / g;
  auto div_g = [&](int row) -> int { return (int)(((unsigned)row * gm) >> 16); };
  bool ok = true;

  // ------------------------------------------------------------------ MMA issuers: S^T by warp 1, PV by warp 24
  auto issue = [&](auto which) {
    constexpr bool is_s = decltype(which)::value;
    uint32_t n = 0;
    int li = 0;
    for (uint32_t j = 0; ok; ++j, ++li) {
      const int slot = j % C::RING;
      if (!wait_bar(B.at(BR::IT_FULL + slot), (j / C::RING) & 1, s_abort)) { ok = false; break; }
      const int it = s_ring[slot].it;
      const int rows = s_ring[slot].w.rows, ntok = s_ring[slot].w.t1 - s_ring[slot].w.t0;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::IT_EMPTY + slot));
      if (it < 0) break;
      const int nt = (ntok + kBT - 1) / kBT;
      if constexpr (is_s) {
        // S^T(n): K(n) has landed, the item's Q is loaded, the TMEM tile has been read
        const uint32_t idesc = ptx::idesc_e4m3_f32(kBT, (rows + 15) / 16 * 16, false, false);
        const int qb = li & 1;
        if (!wait_bar(B.at(BR::Q_FULL + qb), (li >> 1) & 1, s_abort)) { ok = false; break; }
        const uint64_t qd = sdesc<D>(sbase + C::OFF_Q + qb * C::Q_BYTES);
        for (int t = 0; t < nt; ++t, ++n) {
          const int st = (int)(n % C::NSK), sb = n & 3;
          if (!wait_bar(B.at(BR::K_FULL + st), (n / C::NSK) & 1, s_abort) ||
              !wait_bar(B.at(BR::S_EMPTY + sb), ((n >> 2) & 1) ^ 1, s_abort)) {
            ok = false;
            break;
          }
          if (lane == 0) {
            ptx::tc_fence_after();
            const uint64_t kd = sdesc<D>(sbase + C::OFF_K + st * C::KV_TILE);
#pragma unroll
            for (int ks = 0; ks < D / 32; ++ks) {  // descriptor addresses are in units of 16 bytes
              ptx::umma_f8(tmem + sb * kNR, kd + 2 * ks, qd + 2 * ks, idesc, ks > 0);
              ptx::umma_f8(tmem + sb * kNR, kd + 2 * ks, qd + ((kNR * D) >> 4) + 2 * ks, idesc, 1);
            }
            ptx::umma_commit(B.at(BR::S_FULL + sb));
            ptx::umma_commit(B.at(BR::K_EMPTY + st));
            if (t == nt - 1) ptx::umma_commit(B.at(BR::Q_EMPTY + qb));
          }
          __syncwarp();
        }
      } else {
        // PV(n): P(n) is published, V(n) has landed, the accumulator has been read.  A = V^T, MN-major (for D = 64
        // both halves of M read the same 64 columns: lanes 64..127 repeat lanes 0..63 and are not used)
        const uint32_t idesc = ptx::idesc_e4m3_f32(128, (rows + 7) / 8 * 16, true, true);  // N: hi and lo of the rows
        for (int t = 0; t < nt; ++t, ++n) {
          const int st = (int)(n % C::NSV), b = n & 1, pb = n & 3;
          if (!wait_bar(B.at(BR::O_EMPTY + b), ((n >> 1) & 1) ^ 1, s_abort) ||
              !wait_bar(B.at(BR::V_FULL + st), (n / C::NSV) & 1, s_abort) ||
              !wait_bar(B.at(BR::P_FULL + pb), (n >> 2) & 1, s_abort)) {
            ok = false;
            break;
          }
          if (lane == 0) {
            ptx::tc_fence_after();
            const uint64_t vd = sdesc<D>(sbase + C::OFF_V + st * C::KV_TILE);
            const uint64_t pd = ptx::sdesc_sw128(sbase + C::OFF_P + pb * C::P_BYTES, C::P_BYTES, 1024);
#pragma unroll
            for (int ks = 0; ks < kBT / 32; ++ks)
              ptx::umma_f8(tmem + 256 + b * 128, vd + ((ks * 32 * D) >> 4), pd + ((ks * 32 * 128) >> 4), idesc, ks > 0);
            ptx::umma_commit(B.at(BR::O_FULL + b));
            ptx::umma_commit(B.at(BR::P_EMPTY + pb));
            ptx::umma_commit(B.at(BR::V_EMPTY + st));
          }
          __syncwarp();
        }
      }
    }
    if (lane == 0) {
      // every MMA the issuers issued must finish before the TMEM is released
      ptx::umma_commit(B.at(BR::MMA_DONE));
      const long long c0 = clock64();
      while (!ptx::mbar_try_wait(B.at(BR::MMA_DONE), 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  };

  // registers: 28 warps launch with 72 each, 2016 a lane in all = 16 x 72 + 4 x 120 + 8 x 48.  (Each split stands at the
  // head of its own branch: after a join the compiler counts with the least.)
  const int wg = warp >> 2;
  if (wg >= 1 && wg <= 4) {
    // ------------------------------------------------------------------ softmax warps
    // Four groups of four warps, a group at most 16 rows of a tile: up to 16 rows the groups take turns by tile, up to 32
    // two pairs of groups do, a half of the rows each, and above that each group takes a quarter of the rows of every
    // tile.  A thread holds one key's scores for the group's rows and its share of their sums.  A group's four warps
    // agree on the rows' maxima over the tile, and from them on P's references: a row's reference follows its maximum when that
    // leaves [-4, 2.6] around it.
    const int qd = warp & 3;                // TMEM lane quadrant: keys 32*qd .. 32*qd + 31 of a tile
    const int grp = wg - 1;
    const uint32_t lane_addr = (uint32_t)(qd * 32) << 16;
    const int l8 = lane & 7;
    float *mw = reinterpret_cast<float *>(smem + C::OFF_MW) + (grp * 4 + qd) * 16;  // kHead - reference per row, this warp's copy
    uint32_t *red = reinterpret_cast<uint32_t *>(smem + C::OFF_RED) + grp * 2 * 4 * 8;
    uint32_t n0 = 0;                        // tiles before the item
    uint32_t mine = 0;                      // tiles of this group so far
    int li = 0;
    for (uint32_t j = 0; ok; ++j, ++li) {
      const int slot = j % C::RING;
      if (!wait_bar(B.at(BR::IT_FULL + slot), (j / C::RING) & 1, s_abort)) { ok = false; break; }
      const int it = s_ring[slot].it;
      const int t0 = s_ring[slot].w.t0, t1 = s_ring[slot].w.t1, rows = s_ring[slot].w.rows;
      const int ctx = s_ring[slot].w.ctx, row0 = s_ring[slot].w.row0;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::IT_EMPTY + slot));
      if (it < 0) break;
      const int ob = li & 1;
      const int ntiles = (t1 - t0 + kBT - 1) / kBT;
      const int nfull = (max(t0, min(t1, ctx + 1)) - t0) / kBT;  // tiles whose keys every row sees
      const int nrow = (rows + 7) / 8 * 8;
      const Parts pt(nrow);
      // A group's tiles are those of its number modulo the turns, whatever the number of parts: so it has at least one of
      // any four tiles, and the phase of a barrier that it waits for is never two ahead of what it has seen.
      const int turns = 4 / pt.n, part = grp / turns;
      const int r0 = pt.row(part);                   // the group's rows: r0 .. r0 + 8 nu - 1
      const int nu = (pt.row(part + 1) - r0) / 8;
      const uint32_t share = turns;                  // a warp's arrivals per tile (sixteen in all)
      const float *rf = s_rf + (li % C::RF) * kNR + r0;
      float2 lp[8];  // this thread's (key's) share of every row sum
#pragma unroll
      for (int i = 0; i < 8; ++i) lp[i] = make_float2(0.0f, 0.0f);
      float m[2] = {-INFINITY, -INFINITY};    // the references, rows r0 + 2 l8 and the next
      float most[2] = {-INFINITY, -INFINITY}; // the largest so far
      float lsv0 = 0.0f;                      // log2 of V's scale at the group's first key: the sums count in its inverse
      if (lane < 16) mw[lane] = 0.0f;         // (a row without a reference: its weights are 2^-inf)
      __syncwarp();
      bool fresh = true;
      for (int t = (grp - (int)n0) & (turns - 1); t < ntiles; t += turns, ++mine) {
        const uint32_t n = n0 + t;
        const int buf = n & 3;
        if (!wait_bar(B.at(BR::S_FULL + buf), (n >> 2) & 1, s_abort)) { ok = false; break; }
        ptx::tc_fence_after();
        uint32_t v[16];
        ptx::tmem_ld16(tmem + lane_addr + buf * kNR + r0, v);
        const float2 sc = s_sc[(n % C::SC) * 8 + qd * 2 + (lane >> 4)];
        const float lsv = fmaxf(lg2(sc.y), kLeastScaleLog2);
        if (fresh) {
          lsv0 = fmaxf(lg2(s_sc[(n % C::SC) * 8].y), kLeastScaleLog2);
          fresh = false;
        }
        ptx::tmem_wait_ld();
        // the scores are in registers: the tile may be overwritten
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_n(B.at(BR::S_EMPTY + buf), share);
        float x[16];  // in log2 units, plus log2 of V's scale
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 r4 = *reinterpret_cast<const float4 *>(rf + i);
#pragma unroll
          for (int q = 0; q < 4; q += 2) {
            const float2 u = __fmul2_rn(q == 0 ? make_float2(r4.x, r4.y) : make_float2(r4.z, r4.w), both(sc.x));
            const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[i + q]), __uint_as_float(v[i + q + 1])), u, both(lsv));
            x[i + q] = y.x;
            x[i + q + 1] = y.y;
          }
        }
        // Causal mask: key tok is visible to row jr iff row0 + jr >= g * (tok - ctx); keys past the item are masked too.
        // Only an item's last tiles (from nfull on) have such keys.
        if (__builtin_expect(t >= nfull, 0)) {
          const int tok = t0 + t * kBT + qd * 32 + lane;
          const int jmin = tok >= t1 ? 16 : max(0, min(16, g * max(tok - ctx, 0) - row0 - r0));
#pragma unroll
          for (int i = 0; i < 16; ++i)
            if (i < jmin) x[i] = -INFINITY;
        }
        // the rows' maxima over this warp's keys as bf16 pairs (lane i & 7 gets rows 2 i and 2 i + 1), then the group's
        uint32_t wd[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) wd[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
        uint32_t top = warp_transpose_max(wd, lane);
        uint32_t *rd = red + (mine & 1) * 4 * 8;
        if (lane < 8) rd[qd * 8 + lane] = top;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::RED + grp));
        if (!wait_bar(B.at(BR::RED + grp), mine & 1, s_abort)) { ok = false; break; }
        top = bmax2(bmax2(rd[l8], rd[8 + l8]), bmax2(rd[16 + l8], rd[24 + l8]));
        {
          // (rounded up: 2^-8 of their magnitude covers the rounding to bf16)
          float now[2] = {__uint_as_float(top << 16), __uint_as_float(top & 0xffff0000u)};
          bool move[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            if (now[y] != -INFINITY) now[y] = fmaf(fabsf(now[y]), 0x1p-8f, now[y]);
            move[y] = !(now[y] <= m[y] + kUp) || (now[y] < m[y] - kDown && now[y] > most[y] - kFar);  // (a NaN too)
          }
          if (__any_sync(0xffffffffu, move[0] || move[1])) {
            float al[2];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              al[y] = 1.0f;
              if (move[y]) {
                if (m[y] != -INFINITY) al[y] = ptx::ex2(m[y] - now[y]);
                m[y] = now[y];
                most[y] = !(now[y] <= most[y]) ? now[y] : most[y];
              }
            }
            if (lane < 8)
              reinterpret_cast<float2 *>(mw)[lane] = make_float2(m[0] == -INFINITY ? 0.0f : kHead - m[0], m[1] == -INFINITY ? 0.0f : kHead - m[1]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float a0 = __shfl_sync(0xffffffffu, al[0], i), a1 = __shfl_sync(0xffffffffu, al[1], i);
              lp[i] = __fmul2_rn(lp[i], make_float2(a0, a1));
            }
            __syncwarp();
          }
        }
        // P buffer n & 3 is free again once PV(n - 4) is done (and the references of tile n - 8 have been read by then)
        if (!wait_bar(B.at(BR::P_EMPTY + buf), ((n >> 2) & 1) ^ 1, s_abort)) { ok = false; break; }
        if (qd == 0 && lane < 4 * nu) reinterpret_cast<float2 *>(s_m + (n & 7) * kNR + r0)[lane] = make_float2(m[0], m[1]);
        // P = 2^(s - m + kHead), its shares of the sums, its two parts
        const float2 inv2 = both(ptx::ex2(lsv0 - lsv));
        uint8_t *prow = smem + C::OFF_P + buf * C::P_BYTES + (qd * 32 + lane) * 128;
        const int sw = lane & 7;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (u < nu) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float4 m4 = reinterpret_cast<const float4 *>(mw + 8 * u)[h];
#pragma unroll
              for (int q = 0; q < 2; ++q) {
                const int i = 8 * u + 4 * h + 2 * q;
                const float2 a = __fadd2_rn(make_float2(x[i], x[i + 1]), q == 0 ? make_float2(m4.x, m4.y) : make_float2(m4.z, m4.w));
                const float2 e = make_float2(ptx::ex2(a.x), ptx::ex2(a.y));
                lp[i >> 1] = __ffma2_rn(e, inv2, lp[i >> 1]);
                split2<true>(e.x, e.y, hi[2 * h + q], lo[2 * h + q]);
              }
            }
            const int oh = r0 + 8 * u, ol = nrow + oh;
            *reinterpret_cast<uint2 *>(prow + (((oh >> 4) ^ sw) << 4) + (oh & 8)) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
            *reinterpret_cast<uint2 *>(prow + (((ol >> 4) ^ sw) << 4) + (ol & 8)) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
          }
        }
        if (__builtin_expect(t >= nfull && part == 0, 0)) {
          // slots past the request's tokens hold anything, and a NaN times a weight of zero is NaN: zeros in their
          // place.  A value of the new tokens that is NaN is taken out, too, and put back at the end for the rows
          // that see it.
          const int st = (int)(n % C::NSV), tok = t0 + t * kBT + qd * 32 + lane;
          // (first the stage's tile before, PV(n - NSV), then V(n): in one step the wait could pass on the phase before)
          if (!wait_bar(B.at(BR::V_EMPTY + st), ((n / C::NSV) & 1) ^ 1, s_abort) ||
              !wait_bar(B.at(BR::V_FULL + st), (n / C::NSV) & 1, s_abort)) {
            ok = false;
            break;
          }
          uint8_t *vt = smem + C::OFF_V + st * C::KV_TILE;
          const int row = qd * 32 + lane;
          uint32_t bad = 0;
          if (tok > ctx) {
#pragma unroll 1
            for (int c = 0; c < D / 16; ++c) {
              uint4 *v = reinterpret_cast<uint4 *>(vt + swz<D>(row, c));
              if (tok >= t1) {
                *v = make_uint4(0, 0, 0, 0);
              } else {
                const uint4 y = *v;
                const uint32_t k7 = 0x7f7f7f7fu;
                const uint32_t any = __vcmpeq4(y.x & k7, k7) | __vcmpeq4(y.y & k7, k7) | __vcmpeq4(y.z & k7, k7) | __vcmpeq4(y.w & k7, k7);
                bad |= any ? 1u << c : 0u;
              }
            }
          }
          if (__any_sync(0xffffffffu, bad != 0)) {
            if (!wait_bar(B.at(BR::EP_EMPTY + ob), ((li >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
#pragma unroll 1
            for (int i = 0; i < D; ++i) {
              if (bad & (1u << (i >> 4))) {
                uint8_t *v = vt + swz<D>(row, i >> 4) + (i & 15);
                if ((*v & 0x7f) == 0x7f) {
                  *v = 0;
                  atomicMin(s_nan + ob * D + i, g * (tok - ctx) - row0);
                }
              }
            }
            __syncwarp();
          }
        }
        // P(n) is published
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_n(B.at(BR::P_FULL + buf), share);
      }
      if (!ok) break;
      n0 += ntiles;
      // ---- hand the sums over to the correction warps, which must be done with those of item li - 2
      float ls[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) ls[i] = i & 1 ? lp[i >> 1].y : lp[i >> 1].x;
      const float sum = warp_transpose_sum(ls, lane);
      if (!wait_bar(B.at(BR::EP_EMPTY + ob), ((li >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
      if (lane < 16) s_hl[((ob * 4 + grp) * 4 + qd) * 16 + lane] = sum;
      if (qd == 0 && lane < 8)
        reinterpret_cast<float2 *>(s_lr + (ob * 4 + grp) * 16)[lane] = make_float2(m[0] - lsv0 - kHead, m[1] - lsv0 - kHead);
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::EP_FULL + ob));
    }
  } else if (wg == 5) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 120;");
    // ------------------------------------------------------------------ correction warps
    // Thread d (lane d of O^T) keeps head-dim index d of every row: acc += (hi + lo / 16) 2^(m - M - 8) per tile, M a
    // row's reference, which follows its maximum when that is 2^64 above.
    const int qd = warp & 3;
    const int d = qd * 32 + lane;
    const bool dval = d < D;  // for D = 64 the upper two quadrants hold copies
    const uint32_t lane_addr = (uint32_t)(qd * 32) << 16;
    float *cw = reinterpret_cast<float *>(smem + C::OFF_CW) + qd * kNR;
    uint32_t gph = 0, n = 0;
    int li = 0;
    // barrier of the four correction warps (an mbarrier, so that the wait is bounded)
    auto group_sync = [&]() -> bool {
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::EGRP));
      return wait_bar(B.at(BR::EGRP), (gph++) & 1, s_abort);
    };
    for (uint32_t j = 0; ok; ++j, ++li) {
      const int slot = j % C::RING;
      if (!wait_bar(B.at(BR::IT_FULL + slot), (j / C::RING) & 1, s_abort)) { ok = false; break; }
      const int it = s_ring[slot].it;
      const WorkItem w = s_ring[slot].w;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::IT_EMPTY + slot));
      if (it < 0) break;
      const int ob = li & 1, nrow = (w.rows + 7) / 8 * 8;
      const int ntiles = (w.t1 - w.t0 + kBT - 1) / kBT;
      float2 acc[kNR / 2];
#pragma unroll
      for (int i = 0; i < kNR / 2; ++i) acc[i] = make_float2(0.0f, 0.0f);
      float M[2] = {-INFINITY, -INFINITY};  // rows 2 lane and 2 lane + 1
      for (int t = 0; t < ntiles; ++t, ++n) {
        const int b = n & 1;
        if (!wait_bar(B.at(BR::O_FULL + b), (n >> 1) & 1, s_abort)) { ok = false; break; }
        ptx::tc_fence_after();
        bool move = false;
        const float2 m2 = reinterpret_cast<const float2 *>(s_m + (n & 7) * kNR)[lane];
        const float m[2] = {m2.x, m2.y};
        float al[2], f[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          al[x] = 1.0f;
          if (!(m[x] <= M[x] + kLazy)) {  // (a NaN too)
            if (M[x] != -INFINITY) {
              al[x] = ptx::ex2(M[x] - m[x]);
              move = true;
            }
            M[x] = m[x];
          }
          f[x] = m[x] == -INFINITY ? 0.0f : ptx::ex2(m[x] - M[x] - kHead);
        }
        reinterpret_cast<float2 *>(cw)[lane] = make_float2(f[0], f[1]);
        if (__builtin_expect(__any_sync(0xffffffffu, move), 0)) {
#pragma unroll
          for (int i = 0; i < kNR / 2; ++i) {
            const float a0 = __shfl_sync(0xffffffffu, al[0], i), a1 = __shfl_sync(0xffffffffu, al[1], i);
            acc[i] = __fmul2_rn(acc[i], make_float2(a0, a1));
          }
        }
        __syncwarp();
        const uint32_t at = tmem + lane_addr + 256 + b * 128;
#pragma unroll
        for (int c = 0; c < kNR / 8; ++c) {
          if (8 * c < nrow) {
            uint32_t hi[8], lo[8];
            ptx::tmem_ld8(at + 8 * c, hi);
            ptx::tmem_ld8(at + nrow + 8 * c, lo);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
              const float4 f4 = *reinterpret_cast<const float4 *>(cw + 8 * c + i);
#pragma unroll
              for (int q = 0; q < 4; q += 2) {
                const float2 o = __ffma2_rn(make_float2(__uint_as_float(lo[i + q]), __uint_as_float(lo[i + q + 1])), both(0.0625f),
                                            make_float2(__uint_as_float(hi[i + q]), __uint_as_float(hi[i + q + 1])));
                acc[4 * c + (i + q) / 2] = __ffma2_rn(o, q == 0 ? make_float2(f4.x, f4.y) : make_float2(f4.z, f4.w), acc[4 * c + (i + q) / 2]);
              }
            }
          }
        }
        ptx::tc_fence_before();
        __syncwarp();  // (cw has been read, too)
        if (lane == 0) ptx::mbar_arrive(B.at(BR::O_EMPTY + b));
      }
      if (!ok || !wait_bar(B.at(BR::EP_FULL + ob), (li >> 1) & 1, s_abort)) { ok = false; break; }
      // the row sums: four shares of each group that had the row, against its references.  The group that had the
      // item's first tile comes first, so that results repeat to the bit whatever the CTA did before.
      const int nan0 = dval ? s_nan[ob * D + d] : INT32_MAX;
      if (dval) s_nan[ob * D + d] = INT32_MAX;
      float l[2] = {0.0f, 0.0f};
      {
        const Parts pt(nrow);
        int part = 0;  // of rows 2 lane and 2 lane + 1
        for (int i = 1; i < pt.n; ++i) part += 2 * lane >= pt.row(i);
        const int at = (2 * lane - pt.row(part)) / 2 & 7, turns = 4 / pt.n, first = (int)(n - ntiles);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= turns) break;
          const int gr = part * turns + ((first + i) & (turns - 1));
          const float2 *hl = reinterpret_cast<const float2 *>(s_hl + (ob * 4 + gr) * 4 * 16) + at;
          const float2 lr = reinterpret_cast<const float2 *>(s_lr + (ob * 4 + gr) * 16)[at];
          const float2 h0 = hl[0], h1 = hl[8], h2 = hl[16], h3 = hl[24];
          if (lr.x != -INFINITY) l[0] = fmaf((h0.x + h1.x) + (h2.x + h3.x), ptx::ex2(lr.x - M[0]), l[0]);
          if (lr.y != -INFINITY) l[1] = fmaf((h0.y + h1.y) + (h2.y + h3.y), ptx::ex2(lr.y - M[1]), l[1]);
        }
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::EP_EMPTY + ob));
      if (nan0 != INT32_MAX) {  // a value that is NaN: rows from nan0 on see it
#pragma unroll
        for (int i = 0; i < kNR / 2; ++i) {
          if (2 * i >= nan0) acc[i].x = NAN;
          if (2 * i + 1 >= nan0) acc[i].y = NAN;
        }
      }
      if (w.poff < 0) {
        reinterpret_cast<float2 *>(cw)[lane] = make_float2(1.0f / l[0], 1.0f / l[1]);
        __syncwarp();
        // (row pointers stepped from row to row)
        int hh = w.row0 - div_g(w.row0) * g;
        uint16_t *og = static_cast<uint16_t *>(p.out) + ((int64_t)(w.q0 + div_g(w.row0)) * p.Hq + w.h * g + hh) * D + d;
        const int wrap = (p.Hq - g + 1) * D;  // from a position's last head to the next one's first
#pragma unroll
        for (int i = 0; i < kNR; i += 2) {
          if (i < w.rows) {
            const float2 f = *reinterpret_cast<const float2 *>(cw + i);
            if (dval) *og = __bfloat16_as_ushort(__float2bfloat16_rn(acc[i / 2].x * f.x));
            og += hh == g - 1 ? wrap : D;
            hh = hh == g - 1 ? 0 : hh + 1;
            if (dval && i + 1 < w.rows) *og = __bfloat16_as_ushort(__float2bfloat16_rn(acc[i / 2].y * f.y));
            og += hh == g - 1 ? wrap : D;
            hh = hh == g - 1 ? 0 : hh + 1;
          }
        }
        __syncwarp();  // cw is written again by the next item
      } else {
        float *part = p.partials + w.poff;
#pragma unroll
        for (int i = 0; i < kNR; i += 2) {
          if (dval && i < w.rows) __stcg(part + (int64_t)i * D + d, acc[i / 2].x);
          if (dval && i + 1 < w.rows) __stcg(part + (int64_t)(i + 1) * D + d, acc[i / 2].y);
        }
        if (qd == 0) {
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (2 * lane + x < w.rows) {
              __stcg(part + w.rows * D + 2 * lane + x, M[x]);
              __stcg(part + w.rows * D + w.rows + 2 * lane + x, l[x]);
            }
          }
        }
        // ---- the last chunk of this (request, head, row group) to finish merges all ----
        __threadfence();
        if (!group_sync()) { ok = false; break; }
        if (qd == 0 && lane == 0) {
          const int chunks = p.req_chunks[w.r];
          const int done = atomicAdd(p.pair_done + ((int64_t)w.r * p.Hkv + w.h) * p.row_groups + w.rg, 1);
          *s_last = done == chunks - 1 ? chunks : 0;
          __threadfence();
        }
        if (!group_sync()) { ok = false; break; }
        const int chunks = *s_last;
        if (chunks > 0) merge_chunks<D, uint16_t>(p, w, g, chunks, qd, 4);
      }
    }
  } else if (wg == 0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 0 || warp == 3) {
      // ------------------------------------------------------------------ K / V producers
      const bool is_k = warp == 0;
      constexpr uint32_t ns = C::NSK;
      static_assert(C::NSK == C::NSV, "one ring length");
      const CUtensorMap *tm1 = is_k ? &tmk : &tmv;
      const CUtensorMap *tm8 = is_k ? &tmk8 : &tmv8;
      const uint32_t off_t = sbase + (is_k ? C::OFF_K : C::OFF_V);
      const uint32_t full = B.at(is_k ? BR::K_FULL : BR::V_FULL), empty = B.at(is_k ? BR::K_EMPTY : BR::V_EMPTY);
      uint32_t tile_n = 0;
      for (uint32_t j = 0; ok; ++j) {
        const int slot = j % C::RING;
        if (!wait_bar(B.at(BR::IT_FULL + slot), (j / C::RING) & 1, s_abort)) { ok = false; break; }
        const int it = s_ring[slot].it;
        const int t0 = s_ring[slot].w.t0, t1 = s_ring[slot].w.t1, r = s_ring[slot].w.r, h = s_ring[slot].w.h;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::IT_EMPTY + slot));
        if (it < 0) break;
        const int32_t *bt = p.block_tables + (int64_t)r * p.max_blocks_per_seq + t0 / 16;
        const int nblk = (t1 - t0 + 15) / 16;
        auto fetch = [&](int base) -> int {
          const int i = base + lane;
          return i < nblk ? __ldg(bt + i) : -1;
        };
        // the scales of a lane's block (K's producer brings both; blocks that do not exist: any)
        auto scales = [&](int bid) -> float2 {
          if (!is_k || bid < 0 || bid >= p.num_blocks) return make_float2(1.0f, 1.0f);
          const int64_t at = (int64_t)bid * p.Hkv + h;
          return make_float2(__ldg(p.k_scale + at), __ldg(p.v_scale + at));
        };
        int cur = fetch(0), nxt = fetch(32);  // block ids of tiles t..t+3 and t+4..t+7
        float2 sc_cur = scales(cur), sc_nxt = scales(nxt);
        const int ntiles = (t1 - t0 + kBT - 1) / kBT;
        for (int t = 0; t < ntiles; ++t, ++tile_n) {
          if (is_k && lane == 0) *s_issued = tile_n;
          if (t > 0 && (t & 3) == 0) {
            cur = nxt;
            sc_cur = sc_nxt;
            nxt = fetch(32 * ((t >> 2) + 1));
            sc_nxt = scales(nxt);
          }
          const int s = (int)(tile_n % ns);
          const uint32_t round = tile_n / ns;
          if (!wait_bar(empty + 8 * s, (round & 1) ^ 1, s_abort)) { ok = false; break; }
          if (lane == 0) ptx::mbar_arrive_expect_tx(full + 8 * s, C::KV_TILE);
          __syncwarp();
          const int bi = lane & 7;  // block of the tile this lane looks after
          int bid = __shfl_sync(0xffffffffu, cur, (8 * t + bi) & 31);
          const int rel = 8 * t + bi;
          const bool valid = rel < nblk && bid >= 0 && bid < p.num_blocks;
          if (is_k && lane < 8 && rel < nblk && !valid) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, r);
          const int b0 = __shfl_sync(0xffffffffu, bid, 0);
          // eight consecutive valid blocks: one box with the 8-block maps
          const unsigned contig = __ballot_sync(0xffffffffu, lane < 8 && valid && bid == b0 + lane);
          if (contig == 0xFFu) {
            if (lane == 0) ptx::tma_load_4d(off_t + s * C::KV_TILE, tm8, full + 8 * s, 0, 0, h, b0);
          } else if (lane < 8) {
            if (!valid) bid = p.num_blocks;  // past the item (or invalid): out-of-range box, reads zeros
            ptx::tma_load_4d(off_t + s * C::KV_TILE + lane * 16 * D, tm1, full + 8 * s, 0, 0, h, bid);
          }
          if (is_k) {  // the scales, which may arrive later than the block ids
            const float sk = __shfl_sync(0xffffffffu, sc_cur.x, (8 * t + bi) & 31);
            const float sv = __shfl_sync(0xffffffffu, sc_cur.y, (8 * t + bi) & 31);
            if (lane < 8) s_sc[(tile_n % C::SC) * 8 + bi] = make_float2(sk, sv);
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(full + 8 * s);
          }
        }
      }
      // drain: every stage issued must land before the CTA's shared memory goes away
      if (lane == 0) {
        for (uint32_t k = 0; k < ns && k < tile_n; ++k) {
          const uint32_t n = tile_n - 1 - k;
          const long long c0 = clock64();
          while (!ptx::mbar_try_wait(full + 8 * (n % ns), (n / ns) & 1) && clock64() - c0 < kWaitCycles) {
          }
        }
      }
    } else if (warp == 2) {
      // ------------------------------------------------------------------ item loader
      uint32_t published = 0;  // K tiles of the items published so far
      for (uint32_t j = 0; ok; ++j) {
        // items are taken just in time, so that the work counter balances the CTAs to the end, but early enough to
        // hide the way from the claim to the first load
        const int slot = j % C::RING;
        for (const long long c0 = clock64(); published > *s_issued + kAhead;) {
          if (*s_abort || clock64() - c0 > kWaitCycles) {
            *s_abort = 1;
            ok = false;
            break;
          }
          __nanosleep(100);
        }
        if (!ok) break;
        if (!wait_bar(B.at(BR::IT_EMPTY + slot), ((j / C::RING) & 1) ^ 1, s_abort)) { ok = false; break; }
        int tiles = 0;
        if (lane == 0) {
          int it;
          WorkItem w;
          do {
            it = atomicAdd(&p.header_mut->next_item, 1);
            if (it >= n_items) { it = -1; break; }
            w = p.items[it];
          } while (!item_ok(p, w));
          s_ring[slot].it = it;
          if (it >= 0) {
            s_ring[slot].w = w;
            tiles = (w.t1 - w.t0 + kBT - 1) / kBT;
          }
          ptx::mbar_arrive(B.at(BR::IT_FULL + slot));
        }
        tiles = __shfl_sync(0xffffffffu, tiles, 0);
        if (tiles == 0) {
          // no item left for this CTA: a kernel launched after this one as a programmatic
          // dependent may be scheduled; it still waits for this grid to finish
          asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
          break;
        }
        published += tiles;
      }
    } else {
      issue(std::true_type());
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 48;");
    if (warp == 24) {
      issue(std::false_type());
    } else {
      // ------------------------------------------------------------------ Q loaders
      // Query row row0 + rho = j * g + hh at MMA row rho (hi) and 64 + rho (lo), rows past the item up to the MMA's N zero.  A row's
      // factor 2^e / sqrt(D) in log2 units goes to s_rf.
      const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
      constexpr int CPR = D / 8;     // 16-byte chunks per row, a lane each
      constexpr int RPP = 32 / CPR;  // rows per warp pass
      constexpr int QB = 2;          // passes in flight
      const int cc = lane % CPR;
      int li = 0;
      for (uint32_t j = 0; ok; ++j, ++li) {
        const int slot = j % C::RING;
        if (!wait_bar(B.at(BR::IT_FULL + slot), (j / C::RING) & 1, s_abort)) { ok = false; break; }
        const int it = s_ring[slot].it;
        const int rows = s_ring[slot].w.rows, row0 = s_ring[slot].w.row0, q0 = s_ring[slot].w.q0, h = s_ring[slot].w.h;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::IT_EMPTY + slot));
        if (it < 0) break;
        const int qb = li & 1, nrow = (rows + 15) / 16 * 16;
        if (!wait_bar(B.at(BR::Q_EMPTY + qb), ((li >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
        const uint16_t *qi = static_cast<const uint16_t *>(p.q) + ((int64_t)q0 * p.Hq + h * g) * D + cc * 8;
        uint8_t *qs = smem + C::OFF_Q + qb * C::Q_BYTES;
        float *rf = s_rf + (li % C::RF) * kNR;
        for (int base = (warp - 25) * RPP; base < nrow; base += kQWarps * RPP * QB) {
          uint4 v[QB];
#pragma unroll
          for (int u = 0; u < QB; ++u) {
            const int row = base + u * kQWarps * RPP + lane / CPR;
            v[u] = make_uint4(0, 0, 0, 0);
            if (row < rows) {
              const int rj = row0 + row, jj = div_g(rj), hh = rj - jj * g;
              v[u] = __ldg(reinterpret_cast<const uint4 *>(qi + (int64_t)(jj * p.Hq + hh) * D));
            }
          }
#pragma unroll
          for (int u = 0; u < QB; ++u) {
            const int row = base + u * kQWarps * RPP + lane / CPR;
            if (base + u * kQWarps * RPP < nrow) {  // (nrow is a multiple of RPP: the same for the whole warp)
              const uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
              uint32_t big = 0;  // largest magnitude, as bf16 bits
#pragma unroll
              for (int i = 0; i < 4; ++i) big = max(big, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
#pragma unroll
              for (int x = 1; x < CPR; x <<= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, x));
              const bool finite = big < 0x7f80u;
              const int e = finite ? scale_exp(__uint_as_float(big << 16)) : 0;
              const float inv = exp2i(-e);
              uint32_t hi[4], lo[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                split2<false>(__uint_as_float(w[i] << 16) * inv, __uint_as_float(w[i] & 0xffff0000u) * inv, hi[i], lo[i]);
              const uint32_t half = (cc & 1) * 8;
              *reinterpret_cast<uint2 *>(qs + swz<D>(row, cc >> 1) + half) = make_uint2(hi[0] | hi[1] << 16, hi[2] | hi[3] << 16);
              *reinterpret_cast<uint2 *>(qs + swz<D>(kNR + row, cc >> 1) + half) = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
              if (cc == 0) rf[row] = finite ? exp2i(e) * scale_log2 : NAN;
            }
          }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::Q_FULL + qb));
      }
    }
  }
  if (!ok && lane == 0) report(p.status, WISP_DEV_TIMEOUT, p.request_ids, -1);

  // Teardown: every warp reports on an mbarrier that it is done with TMEM, and warp 1 frees the
  // TMEM once all have (a bounded wait; the warps' shared memory stays until the last one exits).
  __syncwarp();
  ptx::tc_fence_before();
  if (lane == 0) ptx::mbar_arrive(B.at(BR::FIN));
  if (warp == 1) {
    const long long c0 = clock64();
    while (!ptx::mbar_try_wait(B.at(BR::FIN), 0) && clock64() - c0 < kWaitCycles) {
    }
    __syncwarp();
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, kTmemCols);
  }
}

// ---------------------------------------------------------------------------- host side
namespace {

PFN_cuTensorMapEncodeTiled_v12000 g_encode = nullptr;

// The paged pool [num_blocks, Hkv, 16, D] of codes as a 4-D tensor (d, slot, head, block); one box = a head's page in
// `box_blocks` consecutive blocks (1, or 8 for a whole tile), rows of D bytes swizzled.
cudaError_t encode_pool(CUtensorMap *map, const void *base, int D, int Hkv, int num_blocks, int box_blocks) {
  const cuuint64_t dims[4] = {(cuuint64_t)D, 16, (cuuint64_t)Hkv, (cuuint64_t)num_blocks};
  const cuuint64_t strides[3] = {(cuuint64_t)D, (cuuint64_t)16 * D, (cuuint64_t)Hkv * 16 * D};
  const cuuint32_t box[4] = {(cuuint32_t)D, 16, 1, (cuuint32_t)box_blocks};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  const CUresult r = g_encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void *>(base), dims, strides, box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// The four tensor maps of a (K pool, V pool, D, Hkv, num_blocks) are the same from step to step:
// the last few sets are kept, so that a launch does not encode them again.
struct PoolMaps {
  const void *k = nullptr, *v = nullptr;
  int D = 0, Hkv = 0, num_blocks = 0;
  CUtensorMap tk, tv, tk8, tv8;
};
constexpr int kMapCache = 8;
PoolMaps g_maps[kMapCache];
int g_maps_next = 0;
std::mutex g_maps_mu;

cudaError_t pool_maps(const AttnParams &p, PoolMaps *out) {
  std::lock_guard<std::mutex> lk(g_maps_mu);
  for (const PoolMaps &m : g_maps) {
    if (m.k == p.k_cache && m.v == p.v_cache && m.D == p.D && m.Hkv == p.Hkv && m.num_blocks == p.num_blocks) {
      *out = m;
      return cudaSuccess;
    }
  }
  PoolMaps m;
  m.k = p.k_cache;
  m.v = p.v_cache;
  m.D = p.D;
  m.Hkv = p.Hkv;
  m.num_blocks = p.num_blocks;
  cudaError_t e = encode_pool(&m.tk, p.k_cache, p.D, p.Hkv, p.num_blocks, 1);
  if (e == cudaSuccess) e = encode_pool(&m.tv, p.v_cache, p.D, p.Hkv, p.num_blocks, 1);
  if (e == cudaSuccess) e = encode_pool(&m.tk8, p.k_cache, p.D, p.Hkv, p.num_blocks, 8);
  if (e == cudaSuccess) e = encode_pool(&m.tv8, p.v_cache, p.D, p.Hkv, p.num_blocks, 8);
  if (e != cudaSuccess) return e;
  g_maps[g_maps_next] = m;
  g_maps_next = (g_maps_next + 1) % kMapCache;
  *out = m;
  return cudaSuccess;
}

}  // namespace

cudaError_t attn_kv8_tc_setup() {
  if (!g_encode) {
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult q;
    const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q);
    if (e != cudaSuccess || q != cudaDriverEntryPointSuccess || !fn) return cudaErrorNotSupported;
    g_encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
  }
  auto set = [](const void *k, int smem) {
    const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  };
  const cudaError_t e = set((const void *)attn_kv8_tc_kernel<128>, Cfg<128>::SMEM);
  return e != cudaSuccess ? e : set((const void *)attn_kv8_tc_kernel<64>, Cfg<64>::SMEM);
}

cudaError_t attn_kv8_tc_launch(const AttnParams &p, int grid, cudaStream_t s) {
  PoolMaps m;
  const cudaError_t e = pool_maps(p, &m);
  if (e != cudaSuccess) return e;
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
  cfg.dynamicSmemBytes = p.D == 128 ? Cfg<128>::SMEM : Cfg<64>::SMEM;
  return p.D == 128 ? cudaLaunchKernelEx(&cfg, attn_kv8_tc_kernel<128>, p, m.tk, m.tv, m.tk8, m.tv8)
                    : cudaLaunchKernelEx(&cfg, attn_kv8_tc_kernel<64>, p, m.tk, m.tv, m.tk8, m.tv8);
}

}  // namespace wisp
