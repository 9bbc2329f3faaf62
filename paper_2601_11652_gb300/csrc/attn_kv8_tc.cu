// attn_kv8_tc.cu -- tensor-core paged GQA attention of the verification forward over an e4m3 cache, bf16 queries.
//
// Same contract as attn_tc.cu (request r's k+1 new queries over its L_total paged keys, query j seeing keys
// 0..c_r + j), with K and V of a page of one head worth code * scale (include/wisp_kv8.h).  K and V go from HBM to the
// tensor core as they are:
//   S^T = K Q^T       (M = 128 keys of a tile, N = the item's rows, K = D),     kind::f8f6f4
//   O^T += V^T P^T    (M = D, N = 2 * rows, K = 128 keys)
// The other operand of each product is split into two e4m3 parts, with 4 + 4 significant bits, what a bf16 value has:
//   * Q = (hi + lo) 2^e: e is one power of two per item, its largest magnitude to at most 448.  Both parts' products add to one
//     accumulator.  An element counts in steps of 2^-9 2^e at least, e4m3's smallest.  A page's K scale enters as a factor of its keys' scores.
//   * P = 2^(s + log2(V's scale) - ref + 5) = hi + lo / 16: V's scale rides on P, and the sums of a row, which must not have it, take P
//     times the inverse, in fp32.  hi and lo rows lie side by side along N and are added when O^T is read; until then each has
//     its own accumulator, so lo may have a factor: it puts P's smallest step at 2^-13.  (Without it, at 2^-9, a thousand
//     weights of 2^-10 of their tile's largest were lost, which can be a seventh of a row.)
//   * ref is a row's reference: the maximum of s + log2(scale) over the tile, taken anew only where the row's maximum
//     over a tile is 3.6 above it (P must stay below 448) or 4 below it (and not 30 below the largest so far, where it
//     weighs nothing).  So a tile's largest P is 2 or more, and a P is off by 2^-8 of itself or 2^-14, whichever is more: 128
//     keys by at most 2^-8 of their largest together.  O^T stays in TMEM for the whole item; only where a reference moves it is
//     read, multiplied and written back.
//
// Persistent CTAs (one per SM) take work items (request, KV head, key chunk, row group) from the plan's counter,
// longest first.  28 warps:
//   * warps 0 and 3 stream K and V tiles of 128 tokens with TMA, one 16 KB box where the tile's eight pages are
//     consecutive in the pool, else one box per page; warp 0 also brings the pages' scales;
//   * warps 1 and 24 issue the MMAs, S^T and PV;
//   * warp 2 takes items just in time and publishes them in a 4-slot ring; warps 25-27 split an item's query rows into
//     one of two Q buffers;
//   * warps 4-19, four groups of four: the softmax.  A thread has one key's scores for up to 32 rows.  Items of up to 32
//     rows: a group has every fourth tile; of more: half of the rows of every second one.  A group's warps agree on the
//     rows' maxima through shared memory; references go from tile to tile, in order, in a 4-slot ring;
//   * warps 20-23 write the outputs or the (O, m, l) partials of a split item, whose last chunk merges all; at their end they compute
//     the items with V scales that P cannot carry.
//
// What bounds it: up to 32 rows the cache's bytes, above that the softmax's instructions.  A tile of 32 KB (D = 128) takes an
// SM 735 ns at the measured copy rate (368 ns for D = 64).  Measured, ns per tile and SM, 38 requests of 8192 tokens, for
// 4 / 16 / 32 / 36 / 64 rows: 920 / 980 / 1045 / 1340 / 1575 (D = 128; 5.4 TB/s at 4 rows), 690 / 735 / 880 / 1255 / 1465
// (D = 64); pages in no order 975 / 1020 / 1085 / 1380 / 1595 and 775 / 805 / 920 / 1270 / 1475.  The bf16 cache's kernel, with
// twice the bytes: 1468 to 1516 and 823 to 880.  Lo's factor and the narrower window of the references cost 0 to 3% of that; the code
// for V scales that P cannot carry, which other items do not run, 0 to 4% up to 32 rows of D = 128 and nothing elsewhere.
// Short items are bound by their own start and end, most of it code that is fetched again for every item: one of a
// single tile takes 4.4 us (4 rows) to 5.4 us (20 rows), one of four tiles 6.1 to 7.3 us.  What the choices gave
// as they were made (before those two), at 4 / 32 / 64 rows of D = 128:
//   * two groups of warps with O in registers of four correction warps, PV products added there per tile: 990 / 1082 / 1681,
//     and 1557 at 36 rows;
//   * groups of at most 24 rows (three or four parts above 32 rows): 955 / 1273 / 2248 against 985 / 1200 / 1701; 16-row parts
//     pay the group's fixed part (waits, maxima, references: about 230 instructions a warp) twice;
//   * tensor and TMA instructions issued under elect.sync and not under `lane == 0`: 985 / 1200 / 1701 to 943 / 1129 / 1685;
//     an MMA took the issuing warp 100 clocks before, 25 after;
//   * the maxima's loop over a group's rows not unrolled, so that less code goes round: 947 / 1118 / 1658 to 924 / 1080 / 1687;
//   * a fourth stage for K: 919 / 1081 / 1691 to 893 / 1019 / 1694; for V instead: nothing;
//   * pages in no order, eight boxes a tile, from one elected lane and not from eight: 1018 / 1144 / 1702 to 970 / 1094 / 1701
//     (D = 64: 869 / 989 / 1579 to 761 / 946 / 1594); pages in order lose 1%;
//   * block ids brought in 12 tiles ahead and scales 8, checked and written four tiles at a time: 1047 to 955 at 4 rows;
//   * less code: masks once, in TMEM, and not wherever scores are read, four rows of O at a time at the end, factors through
//     shared memory, the queries' second look in a loop: one-tile items 5.3 to 4.4 us (4 rows), 5.9 to 5.4 (20 rows), four-tile
//     ones 8.1 to 7.3, 36 rows 1473 to 1345.  One copy of the producers for K and V: one-tile items 4.1 us, but 7% slower with
//     pages in no order.
//
// Every mbarrier wait is bounded in time; an expired wait records WISP_DEV_TIMEOUT and the CTA drains.
#include "attn_merge.cuh"
#include "fp8.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>
#include <cfloat>
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
constexpr uint32_t kNap = 20000;    // ns
constexpr uint32_t kAhead = 3;      // the item loader takes the next item when the K producer is this many tiles from
                                    // the end of what is published
constexpr int kPart = 32;           // rows of a softmax group at most
constexpr float kHead = 5.0f;       // log2 of P at a row's reference
constexpr float kUp = 3.6f;         // a tile's maximum may be this far above the reference (P <= 389, e4m3 holds 448)
constexpr float kDown = 4.0f;       // ... and this far below (P >= 2)
constexpr int kLoFactor = 16;       // of P's lo part (at most 256 of e4m3's 448)
constexpr float kFar = 30.0f;       // what is this far below the largest reference so far weighs nothing
// log2 of V's scales that P can carry: whatever the pages' order, a key that ex2 flushes to 0 for its page's scale then weighs less than
// 2^-30 of another, and the sums stay below 2^120 for 2^20 keys.  A page with a scale of 0 counts with the least (its keys still have
// weight), and V's producer brings zeros for it.  Items with other scales are computed in fp32 (item_in_fp32).
constexpr float kScaleMin = -60.0f, kScaleMax = 40.0f;
static_assert(kNR == 64, "TMEM and shared-memory layout assume 64 rows per item");

template <int D>
struct Cfg {
  static constexpr int KV_TILE = kBT * D;       // bytes of K (or V) of one tile
  static constexpr int Q_BYTES = 2 * kNR * D;   // hi rows, then lo rows
  static constexpr int P_BYTES = kBT * 2 * kNR; // [128 tokens][hi rows, lo rows]
  static constexpr int NSK = D == 128 ? 4 : 8;  // K ring stages
  static constexpr int NSV = D == 128 ? 3 : 6;  // V ring stages
  static constexpr int SC = 16;                 // slots of the scales' ring: tile n in n % SC
  static constexpr int RF = 8;                  // slots of the queries' factors: item li in li % RF
  static constexpr int RING = 4;                // slots of the item ring
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = OFF_Q + 2 * Q_BYTES;
  static constexpr int OFF_V = OFF_K + NSK * KV_TILE;
  static constexpr int OFF_P = OFF_V + NSV * KV_TILE;
  static constexpr int OFF_BAR = OFF_P + 4 * P_BYTES;
  static constexpr int N_BAR = 2 * NSK + 2 * NSV + 28 + 2 * RING + 12;
  static constexpr int OFF_SC = (OFF_BAR + N_BAR * 8 + 15) / 16 * 16;  // float2 [SC][8]: a page's K scale, log2 of its V scale
  static constexpr int OFF_RF = OFF_SC + SC * 64;                      // float [RF]
  static constexpr int OFF_FAR = OFF_RF + RF * 4;                      // int [RF] item li has V scales that P cannot carry
  static constexpr int OFF_RED = OFF_RF + RF * 16;                     // float [4 groups][2][4][32] row maxima per quadrant
  static constexpr int OFF_MW = OFF_RED + 4 * 2 * 4 * 32 * 4;          // float [16][32] per warp: kHead - reference
  static constexpr int OFF_REF = OFF_MW + kSoftmaxWarps * 32 * 4;      // float4 [4][32] two rows' references, the largest so far
  static constexpr int OFF_CW = OFF_REF + 4 * kNR * 8;                 // float [4][64] per epilogue warp
  static constexpr int OFF_HL = OFF_CW + 4 * kNR * 4;                  // float [2][4 groups][4][32] row-sum shares
  static constexpr int OFF_LR = OFF_HL + 2 * 4 * 4 * 32 * 4;           // float [2][4 groups][32] their references
  static constexpr int OFF_FIN = OFF_LR + 2 * 4 * 32 * 4;              // float [2][64] O^T's references
  static constexpr int OFF_NAN = OFF_FIN + 2 * kNR * 4;                // int [2][D] first row that a NaN value reaches
  static constexpr int OFF_MISC = OFF_NAN + 2 * D * 4;
  static constexpr int OFF_RING = OFF_MISC + 64;
  static constexpr int SMEM = OFF_RING + RING * 64 + 1024;             // + slack to align the base to 1024
  static_assert(SMEM <= 227 * 1024, "shared memory of one CTA on sm_103a");
  static_assert(OFF_K % 1024 == 0 && OFF_V % 1024 == 0 && OFF_P % 1024 == 0 && OFF_RING % 16 == 0, "alignment");
  // A tile's scales are written up to three tiles ahead of its K: then S^T of the tile NSK before that K's is done and the
  // scores of the tile NSK + 4 before have been read.  An item's factor is written two items ahead, and its mark for V scales while
  // the epilogue warps have begun the item RING before it at the least.
  static_assert(SC >= NSK + 4 + 3 && RF >= 5, "rings");
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
  static constexpr int O_FULL = P_EMPTY + 4;   // [2] per item parity: its last PV is done
  static constexpr int O_EMPTY = O_FULL + 2;   // [2] the epilogue warps have read O^T
  static constexpr int EP_FULL = O_EMPTY + 2;  // [2] per item parity: the softmax warps handed their sums over
  static constexpr int EP_EMPTY = EP_FULL + 2; // [2] the epilogue warps have read them
  static constexpr int MMA_DONE = EP_EMPTY + 2;  // the two MMA issuers, at the end
  static constexpr int IT_FULL = MMA_DONE + 1, IT_EMPTY = IT_FULL + C::RING;
  static constexpr int EGRP = IT_EMPTY + C::RING;  // the epilogue warps
  static constexpr int RED = EGRP + 1;         // [4] per softmax group: its four warps, once per tile
  static constexpr int DEC = RED + 4;          // [4] the references after tile n stand in slot n & 3
  static constexpr int QX = DEC + 4;           // the Q loaders have an item's largest magnitude
  static constexpr int FIN = QX + 1;          // every warp, once: its last access to TMEM is done
  static_assert(FIN + 1 <= C::N_BAR, "barrier count");
  __device__ __forceinline__ uint32_t at(int i) const { return base + 8 * i; }
};

// (The hint lets a thread sleep while it waits; without it the kernel issues as many instructions.  The second copy of the try
// keeps the first, which mostly passes, short: with a loop in its place items of 36 rows were 10% slower.)
__device__ __forceinline__ bool wait_bar(uint32_t b, uint32_t parity, volatile int *abort) {
  if (ptx::mbar_try_wait_sleep(b, parity, kNap)) return true;
  const long long t0 = clock64();
  while (true) {
    if (ptx::mbar_try_wait_sleep(b, parity, kNap)) return true;
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

// Transposing sum over the 32 lanes of a warp (v is consumed): on return lane i holds the sum over all
// lanes of v[i].
__device__ __forceinline__ float warp_transpose_sum(float (&v)[32], int lane) {
#pragma unroll
  for (int w = 16; w >= 1; w >>= 1) {
    const bool up = (lane & w) != 0;
#pragma unroll
    for (int i = 0; i < w; ++i) {
      const float keep = up ? v[i + w] : v[i];
      const float send = up ? v[i] : v[i + w];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, w);
    }
  }
  return v[0];
}

// The largest of the lanes' values (a NaN never is).
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The parts of an item's rows (rounded up to 8), one or two of at most kPart rows, in whole units of 8: part i starts at
// row(i).
struct Parts {
  int n, units;
  __device__ __forceinline__ explicit Parts(int nrow) : n(nrow <= kPart ? 1 : 2), units(nrow / 8) {}
  __device__ __forceinline__ int row(int i) const { return i * units / n * 8; }
};
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// Four values of magnitude at most 448 as hi + lo / F, four e4m3 codes each: lo is F (1 or 16) times what hi's rounding left
// (exact in fp16, and at most 16 F), rounded.
template <int F>
__device__ __forceinline__ void split4(float a, float b, float c, float d, uint32_t &hi, uint32_t &lo) {
  static_assert(F == 1 || F == 16, "factor of lo");
  uint32_t r0, r1;
  asm("{\n\t.reg .b16 h0, h1;\n\t.reg .b32 p0, p1, q0, q1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h0, %4, %3;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h1, %6, %5;\n\t"
      "cvt.rn.f16x2.f32 p0, %4, %3;\n\t"
      "cvt.rn.f16x2.f32 p1, %6, %5;\n\t"
      "cvt.rn.f16x2.e4m3x2 q0, h0;\n\t"
      "cvt.rn.f16x2.e4m3x2 q1, h1;\n\t"
      "sub.rn.f16x2 %1, p0, q0;\n\t"
      "sub.rn.f16x2 %2, p1, q1;\n\t"
      "mov.b32 %0, {h0, h1};\n\t}"
      : "=r"(hi), "=r"(r0), "=r"(r1)
      : "f"(a), "f"(b), "f"(c), "f"(d));
  if (F == 16) {
    asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(r0) : "r"(0x4c004c00u));
    asm("mul.rn.f16x2 %0, %0, %1;" : "+r"(r1) : "r"(0x4c004c00u));
  }
  asm("{\n\t.reg .b16 l0, l1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 l0, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f16x2 l1, %2;\n\t"
      "mov.b32 %0, {l0, l1};\n\t}"
      : "=r"(lo)
      : "r"(r0), "r"(r1));
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

// A work item on the CUDA cores in fp32, by warp wq of nw: for V scales that P cannot carry.  A warp takes R rows; a lane has one of 32
// keys for their scores, then D / 32 columns of the keys' values.  From the first V scale above 2^64 on sums are taken times 2^-20, so
// that up to 2^20 of the largest values stay finite.  38 requests of 8192 keys, 8 KV heads, D = 128, 4 / 20 / 64 rows: 4.7 / 9.3 / 18 ms.
template <int D>
__device__ __forceinline__ void item_in_fp32(const AttnParams &p, const WorkItem &w, int wq, int nw) {
  constexpr int R = 4, CPL = D / 32;
  const int lane = threadIdx.x & 31, g = p.Hq / p.Hkv;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  const int32_t *bt = p.block_tables + (int64_t)w.r * p.max_blocks_per_seq;
#pragma unroll 1
  for (int rho = wq * R; rho < w.rows; rho += nw * R) {
    int last[R], off[R];  // the last key that a row sees, its elements' offset from the item's first query position
    float m[R], l[R], acc[R][CPL], down = 1.0f;
    const int64_t q0 = ((int64_t)w.q0 * p.Hq + w.h * g) * D;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int rj = w.row0 + min(rho + i, w.rows - 1), j = rj / g;  // (rows past the item: its last one once more)
      last[i] = min(w.t1 - 1, w.ctx + j);
      off[i] = (j * p.Hq + rj - j * g) * D;
      m[i] = -INFINITY;
      l[i] = 0.0f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) acc[i][c] = 0.0f;
    }
#pragma unroll 1
    for (int base = w.t0; base <= last[R - 1]; base += 32) {
      const int tok = base + lane, bid = tok <= last[R - 1] ? __ldg(bt + tok / 16) : -1;
      const bool in = bid >= 0 && bid < p.num_blocks;
      const int64_t page = in ? (int64_t)bid * p.Hkv + w.h : -1;
      float e[R], vs = 0.0f, ks = 0.0f;
#pragma unroll
      for (int i = 0; i < R; ++i) e[i] = 0.0f;
      if (in) {
        ks = __ldg(p.k_scale + page) * scale_log2;
        vs = __ldg(p.v_scale + page);
        const uint4 *k = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.k_cache) + (page * 16 + tok % 16) * D);
        const uint16_t *q = static_cast<const uint16_t *>(p.q) + q0;
#pragma unroll 1
        for (int c = 0; c < D / 16; ++c) {
          const uint4 kv = __ldg(k + c);
          const uint32_t kw[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
          for (int i = 0; i < R; ++i) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint4 qv = __ldg(reinterpret_cast<const uint4 *>(q + off[i] + 16 * c + 8 * h));
              const uint32_t qw[4] = {qv.x, qv.y, qv.z, qv.w};
#pragma unroll
              for (int u = 0; u < 4; ++u) {
                const float2 x = h2_to_f2(e4m3x2_to_h2(kw[2 * h + u / 2] >> (16 * (u & 1)) & 0xffffu));
                e[i] = fmaf(x.x, __uint_as_float(qw[u] << 16), e[i]);
                e[i] = fmaf(x.y, __uint_as_float(qw[u] & 0xffff0000u), e[i]);
              }
            }
          }
        }
      }
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const float s = in && tok <= last[i] ? e[i] * ks : -INFINITY;
        const float mn = fmaxf(m[i], warp_max(s));
        const float alpha = mn == m[i] ? 1.0f : exp2f(m[i] - mn);
        e[i] = s == -INFINITY ? 0.0f : exp2f(s - mn);
        m[i] = mn;
        l[i] = fmaf(l[i], alpha, e[i]);
#pragma unroll
        for (int c = 0; c < CPL; ++c) acc[i][c] *= alpha;
      }
      if (down == 1.0f && __any_sync(0xffffffffu, vs > kLargeScale)) {
        down = kSumDown;
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
          for (int c = 0; c < CPL; ++c) acc[i][c] *= down;
      }
      vs *= down;
#pragma unroll 1
      for (int k0 = 0; k0 < 32; k0 += 8) {
        const int64_t pg = __shfl_sync(0xffffffffu, page, k0 & 16);
        const float y = __shfl_sync(0xffffffffu, vs, k0 & 16);
        if (pg < 0) continue;
        const uint8_t *v = static_cast<const uint8_t *>(p.v_cache) + (pg * 16 + k0 % 16) * D + lane * CPL;
        uint32_t codes[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
          codes[k] = CPL == 4 ? __ldg(reinterpret_cast<const uint32_t *>(v + k * D)) : __ldg(reinterpret_cast<const uint16_t *>(v + k * D));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          float z[CPL];
#pragma unroll
          for (int c = 0; c < CPL; c += 2) {
            const float2 x = h2_to_f2(e4m3x2_to_h2(codes[k] >> (8 * c) & 0xffffu));
            z[c] = y * x.x;
            z[c + 1] = y * x.y;
          }
#pragma unroll
          for (int i = 0; i < R; ++i) {
            const float x = __shfl_sync(0xffffffffu, e[i], k0 + k);
            if (base + k0 + k <= last[i]) {  // (a key that the row does not see adds nothing, whatever it holds)
#pragma unroll
              for (int c = 0; c < CPL; ++c) acc[i][c] = fmaf(x, z[c], acc[i][c]);
            }
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
      if (rho + i >= w.rows) continue;
      l[i] *= down;
      if (w.poff < 0) {
        st_cols<CPL>(static_cast<uint16_t *>(p.out) + q0 + off[i] + lane * CPL, acc[i], 1.0f / l[i]);
      } else {  // as the other chunks have them: O and l times 2^(m - kHead) are the sums
        float *part = p.partials + w.poff;
#pragma unroll
        for (int c = 0; c < CPL; ++c) __stcg(part + (int64_t)(rho + i) * D + lane * CPL + c, acc[i][c]);
        if (lane == 0) {
          __stcg(part + w.rows * D + rho + i, m[i] + (down == 1.0f ? kHead : kHead + kSumDownLog2));
          __stcg(part + w.rows * D + w.rows + rho + i, l[i]);
        }
      }
    }
    __syncwarp();
  }
}

// The items that this CTA's four epilogue warps marked, by the same warps at their end (not a call within the loop over items, whose
// registers and code it would take).  `bar`: the warps' own barrier, at phase `ph`.  False: a wait ran out.
template <int D>
__device__ __noinline__ bool far_items(const AttnParams &p, int n_items, uint32_t bar, uint32_t ph, volatile int *s_last,
                                       volatile int *s_abort) {
  const int lane = threadIdx.x & 31, qd = (threadIdx.x >> 5) & 3;
  auto group_sync = [&]() -> bool {
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(bar);
    return wait_bar(bar, (ph++) & 1, s_abort);
  };
  __threadfence();
  if (!group_sync()) return false;  // (the marks are written)
  for (int base = 0; base < n_items; base += 32) {
    const bool mine = base + lane < n_items && __ldcg(&p.items[base + lane].nrg) == -1 - (int)blockIdx.x;
    for (unsigned left = __ballot_sync(0xffffffffu, mine); left; left &= left - 1) {
      const WorkItem w = p.items[base + __ffs(left) - 1];
      item_in_fp32<D>(p, w, qd, 4);
      if (w.poff < 0) continue;
      // the last chunk of the (request, head, row group) to finish merges all
      __threadfence();
      if (!group_sync()) return false;
      if (qd == 0 && lane == 0) {
        const int chunks = p.req_chunks[w.r];
        const int done = atomicAdd(p.pair_done + ((int64_t)w.r * p.Hkv + w.h) * p.row_groups + w.rg, 1);
        *s_last = done == chunks - 1 ? chunks : 0;
        __threadfence();
      }
      if (!group_sync()) return false;
      const int chunks = *s_last;
      if (chunks > 0) merge_chunks<D, uint16_t>(p, w, p.Hq / p.Hkv, chunks, qd, 4);
    }
  }
  return true;
}

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
  float *s_qf = reinterpret_cast<float *>(smem + C::OFF_RF);
  volatile int *s_far = reinterpret_cast<volatile int *>(smem + C::OFF_FAR);
  volatile uint32_t *s_qmax = reinterpret_cast<volatile uint32_t *>(smem + C::OFF_MISC + 32);
  float4 *s_ref = reinterpret_cast<float4 *>(smem + C::OFF_REF);
  float *s_fin = reinterpret_cast<float *>(smem + C::OFF_FIN);
  float *s_hl = reinterpret_cast<float *>(smem + C::OFF_HL);
  float *s_lr = reinterpret_cast<float *>(smem + C::OFF_LR);
  int *s_nan = reinterpret_cast<int *>(smem + C::OFF_NAN);
  uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + C::OFF_MISC);
  volatile int *s_abort = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 4);
  volatile int *s_last = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 8);
  volatile int *s_marked = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 16);  // the epilogue warps marked an item
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
    init(BR::S_EMPTY, 4, 16);  // the warps of the tile's softmax groups, four or two arrivals each
    init(BR::P_FULL, 4, 16);
    init(BR::P_EMPTY, 4, 1);
    init(BR::O_FULL, 2, 1);
    init(BR::O_EMPTY, 2, 4);   // the epilogue warps
    init(BR::EP_FULL, 2, kSoftmaxWarps);
    init(BR::EP_EMPTY, 2, 4);
    init(BR::MMA_DONE, 1, 2);
    init(BR::IT_FULL, C::RING, 1);
    init(BR::IT_EMPTY, C::RING, 4 + kQWarps + kSoftmaxWarps + 4);  // KV producers, MMA issuers, Q, softmax, correction
    init(BR::EGRP, 1, 4);
    init(BR::QX, 1, kQWarps);
    init(BR::RED, 4, 4);       // a group's warps
    init(BR::DEC, 4, 16);      // the warps of the tile's softmax groups, as for S_EMPTY
    init(BR::FIN, 1, kThreads / 32);
    *s_issued = 0;
    *s_marked = 0;
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
          __syncwarp();
          if (ptx::elect_one()) {
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
        // PV(n): P(n) is published, V(n) has landed and, for an item's first tile, the accumulator has been read.  A = V^T,
        // MN-major (for D = 64 both halves of M read the same 64 columns: lanes 64..127 repeat lanes 0..63 and are not used)
        const uint32_t idesc = ptx::idesc_e4m3_f32(128, (rows + 7) / 8 * 16, true, true);  // N: hi and lo of the rows
        const int ob = li & 1;
        for (int t = 0; t < nt; ++t, ++n) {
          const int st = (int)(n % C::NSV), pb = n & 3;
          if ((t == 0 && !wait_bar(B.at(BR::O_EMPTY + ob), ((li >> 1) & 1) ^ 1, s_abort)) ||
              !wait_bar(B.at(BR::V_FULL + st), (n / C::NSV) & 1, s_abort) ||
              !wait_bar(B.at(BR::P_FULL + pb), (n >> 2) & 1, s_abort)) {
            ok = false;
            break;
          }
          __syncwarp();
          if (ptx::elect_one()) {
            ptx::tc_fence_after();
            const uint64_t vd = sdesc<D>(sbase + C::OFF_V + st * C::KV_TILE);
            const uint64_t pd = ptx::sdesc_sw128(sbase + C::OFF_P + pb * C::P_BYTES, C::P_BYTES, 1024);
#pragma unroll
            for (int ks = 0; ks < kBT / 32; ++ks)
              ptx::umma_f8(tmem + 256 + ob * 128, vd + ((ks * 32 * D) >> 4), pd + ((ks * 32 * 128) >> 4), idesc, t > 0 || ks > 0);
            ptx::umma_commit(B.at(BR::P_EMPTY + pb));
            ptx::umma_commit(B.at(BR::V_EMPTY + st));
            if (t == nt - 1) ptx::umma_commit(B.at(BR::O_FULL + ob));
          }
          __syncwarp();
        }
      }
    }
    __syncwarp();
    if (ptx::elect_one()) {
      // every MMA the issuers issued must finish before the TMEM is released
      ptx::umma_commit(B.at(BR::MMA_DONE));
      const long long c0 = clock64();
      while (!ptx::mbar_try_wait(B.at(BR::MMA_DONE), 0) && clock64() - c0 < kWaitCycles) {
      }
    }
  };

  // registers: 28 warps launch with 72 each, 2016 a lane in all = 16 x 88 + 4 x 72 + 8 x 40.  (Each split stands at the
  // head of its own branch: after a join the compiler counts with the least.)
  const int wg = warp >> 2;
  if (wg >= 1 && wg <= 4) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
    // ------------------------------------------------------------------ softmax warps
    // A group's four warps, one per TMEM lane quadrant, have at most 32 rows of a tile: of up to 32 rows the groups take
    // turns by tile, of more two pairs of groups do, a half of the rows each.  A thread holds one key's scores for the
    // group's rows and its share of their sums.  The warps agree on the rows' maxima over the tile, and from them and the
    // references after the tile before on P's references.
    const int qd = warp & 3;                // TMEM lane quadrant: keys 32*qd .. 32*qd + 31 of a tile
    const int grp = wg - 1;
    const uint32_t lane_addr = (uint32_t)(qd * 32) << 16;
    const int lw = min(lane & 15, kPart / 2 - 1);
    float *mw = reinterpret_cast<float *>(smem + C::OFF_MW) + (grp * 4 + qd) * 32;  // kHead - reference per row, this warp's copy
    float4 *red = reinterpret_cast<float4 *>(smem + C::OFF_RED) + grp * 2 * 4 * 8;
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
      const int ta = (grp - (int)n0) & (turns - 1);  // the group's first tile
      if (ta >= ntiles) {  // none of the item's
        n0 += ntiles;
        if (!wait_bar(B.at(BR::EP_EMPTY + ob), ((li >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
        if (qd == 0) s_lr[(ob * 4 + grp) * 32 + lane] = -INFINITY;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::EP_FULL + ob));
        continue;
      }
      float2 lp[kPart / 2];  // this thread's (key's) share of every row sum
#pragma unroll
      for (int i = 0; i < kPart / 2; ++i) lp[i] = make_float2(0.0f, 0.0f);
      float m[2] = {-INFINITY, -INFINITY};    // the references that lp counts in, rows r0 + 2 lw and the next
      if (lane < kPart) mw[lane] = 0.0f;      // (a row without a reference: its weights are 2^-inf)
      __syncwarp();
      float qf = 0.0f;                        // the queries' factor
      bool fresh = true;
      for (int t = ta; t < ntiles; t += turns, ++mine) {
        const uint32_t n = n0 + t;
        const int buf = n & 3;
        if (!wait_bar(B.at(BR::S_FULL + buf), (n >> 2) & 1, s_abort)) { ok = false; break; }
        ptx::tc_fence_after();
        const float2 sc = s_sc[(n % C::SC) * 8 + qd * 2 + (lane >> 4)];
        const float lsv = sc.y;
        if (fresh) {
          qf = s_qf[li % C::RF];
          fresh = false;
        }
        // (not 0, so that -inf stays: a score is wrong by 2^-100; not infinite, so that a score of 0 stays)
        const float fk = fminf(fmaxf(sc.x * qf, FLT_MIN), FLT_MAX);
        // Causal mask: key tok is visible to row jr iff row0 + jr >= g * (tok - ctx); keys past the item are masked too.
        // Only an item's last tiles (from nfull on) have such keys: -inf in their scores' place.
        if (__builtin_expect(t >= nfull, 0)) {
          const int tok = t0 + t * kBT + qd * 32 + lane;
          const int jmin = tok >= t1 ? kNR : max(0, min(kNR, g * max(tok - ctx, 0) - row0 - r0));
#pragma unroll 1
          for (int u = 0; u < nu; ++u) {
            uint32_t v[8];
            ptx::tmem_ld8(tmem + lane_addr + buf * kNR + r0 + 8 * u, v);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (8 * u + i < jmin) v[i] = 0xff800000u;
            ptx::tmem_st8(tmem + lane_addr + buf * kNR + r0 + 8 * u, v);
          }
          ptx::tmem_wait_st();
        }
        // the scores of unit u (log2 units, plus log2 of V's scale)
        auto scores = [&](int u, float (&x)[8]) {
          uint32_t v[8];
          ptx::tmem_ld8(tmem + lane_addr + buf * kNR + r0 + 8 * u, v);
          ptx::tmem_wait_ld();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 y = __ffma2_rn(make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), both(fk), both(lsv));
            x[2 * i] = y.x;
            x[2 * i + 1] = y.y;
          }
        };
        float4 *rd = red + (mine & 1) * 4 * 8;
#pragma unroll 1
        for (int u = 0; u < kPart / 8; ++u) {
          if (u < nu) {
            float x[8];
            scores(u, x);
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = warp_max(x[i]);
            if (lane == 0) {
              rd[qd * 8 + 2 * u] = make_float4(y[0], y[1], y[2], y[3]);
              rd[qd * 8 + 2 * u + 1] = make_float4(y[4], y[5], y[6], y[7]);
            }
          }
        }
        // ... then the group's, and the references after the tile before
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::RED + grp));
        if (!wait_bar(B.at(BR::RED + grp), mine & 1, s_abort) ||
            (n > 0 && !wait_bar(B.at(BR::DEC + ((n - 1) & 3)), ((n - 1) >> 2) & 1, s_abort))) {
          ok = false;
          break;
        }
        float2 top = reinterpret_cast<const float2 *>(rd)[lw];  // (of rows that the group has)
#pragma unroll
        for (int i = 1; i < 4; ++i) {
          const float2 y = reinterpret_cast<const float2 *>(rd + 8 * i)[lw];
          top = make_float2(fmaxf(top.x, y.x), fmaxf(top.y, y.y));
        }
        if (lw >= 4 * nu) top = both(-INFINITY);
        float4 ref = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);  // two rows' references, the largest so far
        if (t > 0) ref = s_ref[((n - 1) & 3) * (kNR / 2) + r0 / 2 + lw];
        const float old[2] = {ref.x, ref.y};
        // (a NaN moves a reference, too)
        if (!(top.x <= ref.x + kUp) || (top.x < ref.x - kDown && top.x > ref.z - kFar)) {
          ref.x = top.x;
          ref.z = !(top.x <= ref.z) ? top.x : ref.z;
        }
        if (!(top.y <= ref.y + kUp) || (top.y < ref.y - kDown && top.y > ref.w - kFar)) {
          ref.y = top.y;
          ref.w = !(top.y <= ref.w) ? top.y : ref.w;
        }
        if (qd == 0 && lane < 4 * nu) s_ref[(n & 3) * (kNR / 2) + r0 / 2 + lane] = ref;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_n(B.at(BR::DEC + buf), turns);
        // (a NaN differs from itself: its sums become NaN, whatever the factor)
        if (__builtin_expect(__any_sync(0xffffffffu, ref.x != m[0] || ref.y != m[1]), 0)) {
          const float a0 = m[0] == -INFINITY || ref.x == m[0] ? 1.0f : ptx::ex2(m[0] - ref.x);
          const float a1 = m[1] == -INFINITY || ref.y == m[1] ? 1.0f : ptx::ex2(m[1] - ref.y);
          if (lane < kPart / 2) reinterpret_cast<float2 *>(mw)[lane] = make_float2(a0, a1);
          __syncwarp();
#pragma unroll
          for (int i = 0; i < kPart / 4; ++i) {
            const float4 f = reinterpret_cast<const float4 *>(mw)[i];
            lp[2 * i] = __fmul2_rn(lp[2 * i], make_float2(f.x, f.y));
            lp[2 * i + 1] = __fmul2_rn(lp[2 * i + 1], make_float2(f.z, f.w));
          }
          __syncwarp();
          m[0] = ref.x;
          m[1] = ref.y;
          if (lane < kPart / 2)
            reinterpret_cast<float2 *>(mw)[lane] = make_float2(m[0] == -INFINITY ? 0.0f : kHead - m[0], m[1] == -INFINITY ? 0.0f : kHead - m[1]);
          __syncwarp();
        }
        // P buffer n & 3 is free again once PV(n - 4) is done
        if (!wait_bar(B.at(BR::P_EMPTY + buf), ((n >> 2) & 1) ^ 1, s_abort)) { ok = false; break; }
        if (__builtin_expect(t > 0 && __any_sync(0xffffffffu, ref.x != old[0] || ref.y != old[1]), 0)) {
          // O^T so far counts in the references before: PV(n - 1) is the last product on it
          if (!wait_bar(B.at(BR::P_EMPTY + ((n - 1) & 3)), ((n - 1) >> 2) & 1, s_abort)) { ok = false; break; }
          ptx::tc_fence_after();
          const float f0 = old[0] == -INFINITY || ref.x == old[0] ? 1.0f : ptx::ex2(old[0] - ref.x);
          const float f1 = old[1] == -INFINITY || ref.y == old[1] ? 1.0f : ptx::ex2(old[1] - ref.y);
#pragma unroll 1
          for (int u = 0; u < 2 * nu; ++u) {  // hi, then lo
            const uint32_t at = tmem + lane_addr + 256 + ob * 128 + (u < nu ? r0 + 8 * u : nrow + r0 + 8 * (u - nu));
            const int from = 4 * (u < nu ? u : u - nu);  // the lane of the rows' factors
            uint32_t y[8];
            ptx::tmem_ld8(at, y);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 8; ++i)
              y[i] = __float_as_uint(__uint_as_float(y[i]) * __shfl_sync(0xffffffffu, i & 1 ? f1 : f0, from + i / 2));
            ptx::tmem_st8(at, y);
          }
          ptx::tmem_wait_st();
          ptx::tc_fence_before();
          __syncwarp();
        }
        // P = 2^(s - reference + kHead), its shares of the sums, its two parts
        const float2 inv2 = both(ptx::ex2(-lsv));
        uint8_t *prow = smem + C::OFF_P + buf * C::P_BYTES + (qd * 32 + lane) * 128;
        const int sw = lane & 7;
#pragma unroll
        for (int u = 0; u < kPart / 8; ++u) {
          if (u < nu) {
            float x[8];
            scores(u, x);
            uint32_t hi[2], lo[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float4 m4 = reinterpret_cast<const float4 *>(mw + 8 * u)[h];
              const int i = 4 * h;
              const float2 a = __fadd2_rn(make_float2(x[i], x[i + 1]), make_float2(m4.x, m4.y));
              const float2 c = __fadd2_rn(make_float2(x[i + 2], x[i + 3]), make_float2(m4.z, m4.w));
              const float2 e = make_float2(ptx::ex2(a.x), ptx::ex2(a.y)), f = make_float2(ptx::ex2(c.x), ptx::ex2(c.y));
              lp[4 * u + 2 * h] = __ffma2_rn(e, inv2, lp[4 * u + 2 * h]);
              lp[4 * u + 2 * h + 1] = __ffma2_rn(f, inv2, lp[4 * u + 2 * h + 1]);
              split4<kLoFactor>(e.x, e.y, f.x, f.y, hi[h], lo[h]);
            }
            const int oh = r0 + 8 * u, ol = nrow + oh;
            *reinterpret_cast<uint2 *>(prow + (((oh >> 4) ^ sw) << 4) + (oh & 8)) = make_uint2(hi[0], hi[1]);
            *reinterpret_cast<uint2 *>(prow + (((ol >> 4) ^ sw) << 4) + (ol & 8)) = make_uint2(lo[0], lo[1]);
          }
        }
        // the scores have been read: the tile may be overwritten
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_n(B.at(BR::S_EMPTY + buf), turns);
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
        if (lane == 0) ptx::mbar_arrive_n(B.at(BR::P_FULL + buf), turns);  // (sixteen in all)
      }
      if (!ok) break;
      n0 += ntiles;
      // ---- hand the sums over to the epilogue warps, which must be done with those of item li - 2
      float ls[32];
#pragma unroll
      for (int i = 0; i < 32; ++i) ls[i] = i >= kPart ? 0.0f : i & 1 ? lp[i >> 1].y : lp[i >> 1].x;
      const float sum = warp_transpose_sum(ls, lane);
      if (!wait_bar(B.at(BR::EP_EMPTY + ob), ((li >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
      s_hl[((ob * 4 + grp) * 4 + qd) * 32 + lane] = sum;
      if (qd == 0 && lane < kPart / 2) {
        reinterpret_cast<float2 *>(s_lr + (ob * 4 + grp) * 32)[lane] = make_float2(m[0] - kHead, m[1] - kHead);
        // (the group of the last tile has the references of O^T)
        if (((n0 - 1 - grp) & (turns - 1)) == 0 && lane < 4 * nu) reinterpret_cast<float2 *>(s_fin + ob * kNR + r0)[lane] = make_float2(m[0], m[1]);
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::EP_FULL + ob));
    }
  } else if (wg == 5) {
    // ------------------------------------------------------------------ epilogue warps
    // Thread d (lane d of O^T) writes head-dim index d of every row once the item's last product is done.
    const int qd = warp & 3;
    const int d = qd * 32 + lane;
    const bool dval = d < D;  // for D = 64 the upper two quadrants hold copies
    const uint32_t lane_addr = (uint32_t)(qd * 32) << 16;
    float *cw = reinterpret_cast<float *>(smem + C::OFF_CW) + qd * kNR;
    uint32_t gph = 0, n0 = 0;
    int li = 0;
    // barrier of the four epilogue warps (an mbarrier, so that the wait is bounded)
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
      if (!wait_bar(B.at(BR::EP_FULL + ob), (li >> 1) & 1, s_abort)) { ok = false; break; }
      if (__builtin_expect(s_far[li % C::RF] != 0, 0)) {  // V scales that P cannot carry: marked, and computed after the others
        *s_marked = 1;
        if (qd == 0 && lane == 0) const_cast<WorkItem *>(p.items)[it].nrg = -1 - (int)blockIdx.x;
        if (dval) s_nan[ob * D + d] = INT32_MAX;
        n0 += (w.t1 - w.t0 + kBT - 1) / kBT;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::EP_EMPTY + ob));
        if (!wait_bar(B.at(BR::O_FULL + ob), (li >> 1) & 1, s_abort)) { ok = false; break; }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(B.at(BR::O_EMPTY + ob));
        continue;
      }
      // The row sums: four shares of each group that had the row, against its references.  The group that had the
      // item's first tile comes first, so that results repeat to the bit whatever the CTA did before.
      const int nan0 = dval ? s_nan[ob * D + d] : INT32_MAX;
      if (dval) s_nan[ob * D + d] = INT32_MAX;
      const float2 fin = reinterpret_cast<const float2 *>(s_fin + ob * kNR)[lane];  // rows 2 lane and 2 lane + 1
      float l[2] = {0.0f, 0.0f};
      {
        const Parts pt(nrow);
        int part = 0;  // of the two rows
        if (pt.n == 2) part = 2 * lane >= pt.row(1);
        const int at = min((2 * lane - pt.row(part)) / 2, 15), turns = 4 / pt.n, first = (int)n0;
#pragma unroll 1
        for (int i = 0; i < turns; ++i) {
          const int gr = part * turns + ((first + i) & (turns - 1));
          const float2 *hl = reinterpret_cast<const float2 *>(s_hl + (ob * 4 + gr) * 4 * 32) + at;
          const float2 lr = reinterpret_cast<const float2 *>(s_lr + (ob * 4 + gr) * 32)[at];
          const float2 h0 = hl[0], h1 = hl[16], h2 = hl[32], h3 = hl[48];
          if (lr.x != -INFINITY) l[0] = fmaf((h0.x + h1.x) + (h2.x + h3.x), ptx::ex2(lr.x + kHead - fin.x), l[0]);
          if (lr.y != -INFINITY) l[1] = fmaf((h0.y + h1.y) + (h2.y + h3.y), ptx::ex2(lr.y + kHead - fin.y), l[1]);
        }
      }
      n0 += (w.t1 - w.t0 + kBT - 1) / kBT;
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(B.at(BR::EP_EMPTY + ob));
      const bool whole = w.poff < 0;
      float *part = p.partials + w.poff;
      reinterpret_cast<float2 *>(cw)[lane] = whole ? make_float2(rcp(l[0]), rcp(l[1])) : both(1.0f);
      if (!whole && qd == 0) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          if (2 * lane + x < w.rows) {
            __stcg(part + w.rows * D + 2 * lane + x, x ? fin.y : fin.x);
            __stcg(part + w.rows * D + w.rows + 2 * lane + x, l[x]);
          }
        }
      }
      __syncwarp();
      if (!wait_bar(B.at(BR::O_FULL + ob), (li >> 1) & 1, s_abort)) { ok = false; break; }
      ptx::tc_fence_after();
      // (row pointers stepped from row to row)
      int hh = w.row0 - div_g(w.row0) * g;
      uint16_t *og = static_cast<uint16_t *>(p.out) + ((int64_t)(w.q0 + div_g(w.row0)) * p.Hq + w.h * g + hh) * D + d;
      const int wrap = (p.Hq - g + 1) * D;  // from a position's last head to the next one's first
      const uint32_t at = tmem + lane_addr + 256 + ob * 128;
#pragma unroll 1
      for (int r = 0; r < w.rows; r += 4) {
        uint32_t hi[4], lo[4];
        ptx::tmem_ld4(at + r, hi);
        ptx::tmem_ld4(at + nrow + r, lo);
        ptx::tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float o = fmaf(__uint_as_float(lo[i]), 1.0f / kLoFactor, __uint_as_float(hi[i])) * cw[r + i];
          if (r + i >= nan0) o = NAN;  // a value that is NaN: rows from nan0 on see it
          if (dval && r + i < w.rows) {
            if (whole)
              *og = __bfloat16_as_ushort(__float2bfloat16_rn(o));
            else
              __stcg(part + (int64_t)(r + i) * D + d, o);
          }
          og += hh == g - 1 ? wrap : D;
          hh = hh == g - 1 ? 0 : hh + 1;
        }
      }
      ptx::tc_fence_before();
      __syncwarp();  // (cw has been read, too)
      if (lane == 0) ptx::mbar_arrive(B.at(BR::O_EMPTY + ob));
      if (!whole) {
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
    if (__builtin_expect(ok && *s_marked, 0)) ok = far_items<D>(p, n_items, B.at(BR::EGRP), gph, s_last, s_abort);
  } else if (wg == 0) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    // ------------------------------------------------------------------ K / V producers
    auto produce = [&](auto which) {
      constexpr bool is_k = decltype(which)::value;
      constexpr uint32_t ns = is_k ? C::NSK : C::NSV;
      const CUtensorMap *tm1 = is_k ? &tmk : &tmv;
      const CUtensorMap *tm8 = is_k ? &tmk8 : &tmv8;
      const uint32_t off_t = sbase + (is_k ? C::OFF_K : C::OFF_V);
      const uint32_t full = B.at(is_k ? BR::K_FULL : BR::V_FULL), empty = B.at(is_k ? BR::K_EMPTY : BR::V_EMPTY);
      uint32_t tile_n = 0, s = 0, phase = 1;  // the ring's stage and its barrier's parity
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
        auto valid = [&](int bid) -> bool { return bid >= 0 && bid < p.num_blocks; };
        // the scales of a lane's block (K's producer brings both; blocks that do not exist: any)
        auto scales = [&](int bid) -> float2 {
          if (!valid(bid)) return make_float2(1.0f, 1.0f);
          const int64_t at = (int64_t)bid * p.Hkv + h;
          return make_float2(is_k ? __ldg(p.k_scale + at) : 1.0f, __ldg(p.v_scale + at));
        };
        // block ids of tiles t..t+3, t+4..t+7 and t+8..t+11, the scales of the first two
        int cur = fetch(0), nxt = fetch(32), far = fetch(64);
        float2 sc_cur = scales(cur), sc_nxt = scales(nxt);
        bool v_far = false;               // one of the item's V scales so far is one that P cannot carry
        unsigned runs = 0;                // bit 8 i + 7 of tiles t..t+3: i's blocks are consecutive and valid
        const int ntiles = (t1 - t0 + kBT - 1) / kBT;
        for (int t = 0; t < ntiles; ++t, ++tile_n) {
          if ((t & 3) == 0) {
            if (t > 0) {
              cur = nxt;
              nxt = far;
              far = fetch(8 * t + 64);
              sc_cur = sc_nxt;
              sc_nxt = scales(nxt);
            }
            bool good = valid(cur);
            if (is_k && !good && 8 * t + lane < nblk) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, r);
            if (!is_k) good = good && sc_cur.y != 0.0f;
            if (!good) cur = p.num_blocks;  // past the item (or invalid, or V scaled by 0): out-of-range box, reads zeros
            __syncwarp();
            const int lead = __shfl_sync(0xffffffffu, cur, lane & 24);
            runs = __ballot_sync(0xffffffffu, good & (cur == lead + (lane & 7)));
          }
          const int i = t & 3;
          if (!wait_bar(empty + 8 * s, phase, s_abort)) { ok = false; break; }
          const int bid = __shfl_sync(0xffffffffu, cur, 8 * i + (lane & 7));
          if (lane == 0) {
            if (is_k) *s_issued = tile_n;
            ptx::mbar_arrive_expect_tx(full + 8 * s, C::KV_TILE);
          }
          __syncwarp();
          if (((runs >> (8 * i)) & 0xffu) == 0xffu) {  // one box with the 8-block maps
            if (ptx::elect_one()) ptx::tma_load_4d(off_t + s * C::KV_TILE, tm8, full + 8 * s, 0, 0, h, bid);
          } else {
            int bids[8];
#pragma unroll
            for (int b = 0; b < 8; ++b) bids[b] = __shfl_sync(0xffffffffu, bid, b);
            if (ptx::elect_one()) {
#pragma unroll
              for (int b = 0; b < 8; ++b)
                ptx::tma_load_4d(off_t + s * C::KV_TILE + b * 16 * D, tm1, full + 8 * s, 0, 0, h, bids[b]);
            }
          }
          __syncwarp();
          if (is_k) {  // the scales, which may arrive later than the block ids, of four tiles at a time
            if (i == 0) {
              const float lv = sc_cur.y == 0.0f ? kScaleMin : lg2(sc_cur.y);
              v_far |= __any_sync(0xffffffffu, !(lv >= kScaleMin && lv <= kScaleMax));
              if (lane == 0) s_far[j % C::RF] = v_far;
              s_sc[((tile_n + (lane >> 3)) % C::SC) * 8 + (lane & 7)] = make_float2(sc_cur.x, lv);
              __syncwarp();
            }
            if (lane == 0) ptx::mbar_arrive(full + 8 * s);
          }
          if (++s == ns) {
            s = 0;
            phase ^= 1;
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
    };
    if (warp == 0) {
      produce(std::true_type());
    } else if (warp == 3) {
      produce(std::false_type());
    } else if (warp == 2) {
      // ------------------------------------------------------------------ item loader
      uint32_t published = 0;  // K tiles of the items published so far
      bool first = true;
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
            // (the first one is the CTA's own: a way to memory and back less before its first load)
            it = first ? (int)blockIdx.x : p.header->attn_ctas + atomicAdd(&p.header_mut->next_item, 1);
            first = false;
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
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 24) {
      issue(std::false_type());
    } else {
      // ------------------------------------------------------------------ Q loaders
      // Query row row0 + rho = j * g + hh at MMA row rho (hi) and 64 + rho (lo), rows past the item up to the MMA's N zero.
      // The rows are read twice, for the item's exponent e (their largest finite magnitude is at most 448 * 2^e) and for their
      // parts; the queries' factor 2^e / sqrt(D) in log2 units goes to s_qf.  What is not finite becomes NaN in both parts, and
      // the scores of its own row with it.
      const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
      constexpr int CPR = D / 8;     // 16-byte chunks per row, a lane each
      constexpr int RPP = 32 / CPR;  // rows per warp pass
      constexpr int STEP = kQWarps * RPP;
      const int cc = lane % CPR, wq = warp - 25;
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
        const uint16_t *qi = static_cast<const uint16_t *>(p.q) + ((int64_t)q0 * p.Hq + h * g) * D + cc * 8;
        auto load = [&](int row) -> uint4 {
          if (row >= rows) return make_uint4(0, 0, 0, 0);
          const int rj = row0 + row, jj = div_g(rj), hh = rj - jj * g;
          return __ldg(reinterpret_cast<const uint4 *>(qi + (int64_t)(jj * p.Hq + hh) * D));
        };
        uint32_t big = 0;  // largest magnitude, as bf16 bits
        auto look = [&](const uint4 &v) {
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a = w[i] & 0x7fffu, b = (w[i] >> 16) & 0x7fffu;
            big = max(big, max(a < 0x7f80u ? a : 0u, b < 0x7f80u ? b : 0u));
          }
        };
        const int first = wq * RPP + lane / CPR;
#pragma unroll 4
        for (int row = first; row < rows; row += STEP) look(load(row));
        __syncwarp();
        big = __reduce_max_sync(0xffffffffu, big);
        // the three warps' maxima (slot li & 1: its readers of item li - 2 have all arrived at item li - 1 since)
        if (lane == 0) {
          s_qmax[(li & 1) * 4 + wq] = big;
          ptx::mbar_arrive(B.at(BR::QX));
        }
        uint4 v = load(first);
        if (!wait_bar(B.at(BR::QX), li & 1, s_abort) || !wait_bar(B.at(BR::Q_EMPTY + qb), ((li >> 1) & 1) ^ 1, s_abort)) {
          ok = false;
          break;
        }
        big = max(s_qmax[(li & 1) * 4], max(s_qmax[(li & 1) * 4 + 1], s_qmax[(li & 1) * 4 + 2]));
        const int e = scale_exp(__uint_as_float(big << 16));
        const float inv = exp2i(-e);
        if (wq == 0 && lane == 0) s_qf[li % C::RF] = exp2i(e) * scale_log2;
        uint8_t *qs = smem + C::OFF_Q + qb * C::Q_BYTES;
        auto put = [&](int row, const uint4 &v) {
          // (x * 0: an infinity becomes NaN)
          auto low = [&](uint32_t w) { const float x = __uint_as_float(w << 16); return fmaf(x, 0.0f, x * inv); };
          auto high = [&](uint32_t w) { const float x = __uint_as_float(w & 0xffff0000u); return fmaf(x, 0.0f, x * inv); };
          uint32_t hi[2], lo[2];
          split4<1>(low(v.x), high(v.x), low(v.y), high(v.y), hi[0], lo[0]);
          split4<1>(low(v.z), high(v.z), low(v.w), high(v.w), hi[1], lo[1]);
          const uint32_t half = (cc & 1) * 8;
          *reinterpret_cast<uint2 *>(qs + swz<D>(row, cc >> 1) + half) = make_uint2(hi[0], hi[1]);
          *reinterpret_cast<uint2 *>(qs + swz<D>(kNR + row, cc >> 1) + half) = make_uint2(lo[0], lo[1]);
        };
#pragma unroll 1
        for (int row = first; row < nrow; row += STEP) {
          const uint4 now = v;
          v = load(row + STEP);
          put(row, now);
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
