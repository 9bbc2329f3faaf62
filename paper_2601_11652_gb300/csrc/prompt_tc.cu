// prompt_tc.cu -- tensor-core attention with many query rows: prompts, and the rows of requests that share a prefix
// (bf16 queries, paged cache, include/wisp_prompt.h).
//
// An item (prompt.cuh) is up to two tiles of 128 query rows of one KV head, row = position * g + head of the group, over a chunk of
// keys.  Per key tile of 128 and stream (a stream: 128 rows in the MMA's M):
//   S = Q K^T         M = 128 rows, N = 128 keys, K = D; fp32 in TMEM, a row per lane
//   P = 2^(S - m)     by 128 threads, one row each: no exchange between threads; bf16, back to TMEM over S
//   O += P V          M = 128 rows, N = D, K = 128 keys; A from TMEM, fp32 in TMEM
// m follows the row's maximum loosely: it moves (and O, l are rescaled) only where a tile's maximum has come 2^7 nearer to it, so rescales are rare after
// a row's first tiles; see kRoom.  A weight is rounded to bf16 (2^-9) for the second product, the row sum adds it before that.
//
// An item of more than one tile of rows runs its tiles as two streams over the same key tiles; one of a single tile runs
// the even and the odd key tiles as two streams of the same rows, joined at the end.  So there are always two chains
// (S, softmax, P V) that fill each other's gaps.
//
// Persistent CTAs take items from a global counter, longest first.  Warps:
//   * 0-3, 4-7: softmax and epilogue of stream 0 and 1, a thread per row;
//   * 8, 11: issue tcgen05.mma of stream 0 and 1.  With D = 128 a stream's next S follows its P V directly, so that an S that has
//     arrived says that the O before it is complete, and S may overwrite P; with D = 64 it comes before, as soon as S has been read;
//   * 9: takes items, and brings Q (boxes of whole positions), K and V (boxes of one page or of eight consecutive ones) by TMA;
//   * 10: looks at V where a tile has keys that some row does not see: 0 * NaN would reach every row.  Values that are not finite
//     are set to zero there and remembered with the first position that sees them; the epilogue writes what they make of its rows.
//   * 12-15, over an 8-bit cache: a tile's codes arrive in the upper half of its stage, or of each warp's part of it, and these warps
//     write it in bf16, times the page's scale, in place: a lane's row of codes in registers first.
// Every wait is bounded: an expired one records WISP_DEV_TIMEOUT and the CTA drains.
//
// Bound, D = 128: the tensor core; a tile of both streams takes 2530 cycles, 2048 of them at its nominal rate (S reads Q and K from shared
// memory).  16384 tokens, 32 heads over 8: 1.17 ms alone, the 1.88 PFLOP/s that a library product reaches, 1.32 ms in a row under the
// power limit; 4096 tokens 96 us; over e4m3 128 us.  D = 64: the softmax warps' chain, two warps a scheduler, 2400 cycles a tile; 48 prompts
// of up to 1500 tokens 245 us, 0.66 PFLOP/s.  Few rows and keys: latency, most of it code that is fetched for the first time (about ten
// cycles an instruction), so that less code is faster: 64 tokens, whole call 15 us.
// Measured and not kept: a part of the exponentials as polynomials (one in eight: 4096 tokens 99 to 109 us, heads of 64 85 to 92); m taken from
// the tile before (102 to 112); S read a second time instead of held in registers (102 to 121); items of one row tile (2000 tokens 46 to
// 52); two groups of softmax warps per stream (heads of 64, 84.5 to 101); warps without rows of the item skip its softmax (64 requests
// with a prefix 81.8 to 82.2, 4096 tokens 98.8 to 101.3); maxima only where weights come out large (96 to 107, heads of 64 83.7 to 83.2, 48 prompts
// 250 to 256); the streams' exponentials one after the other (heads of 64 84 to 93).
#include "attn_merge.cuh"
#include "fp8.cuh"
#include "prompt.cuh"
#include "sm100_ptx.cuh"

#include <cudaTypedefs.h>
#include <cstring>

namespace wisp {

namespace {

constexpr int kBT = 128;      // keys per tile
constexpr int kM = 128;       // rows per stream
constexpr int threads_of(bool kv8) { return kv8 ? 512 : 384; }
constexpr uint32_t kTmemCols = 512;  // S of the streams at 0 and 128, O at 256 and 256 + D, P: Cfg::P_COL
constexpr long long kWaitCycles = 4000000000LL;  // about two seconds: a wait that long is a failure
// Sums of weights stay below 1, so that sums of weights times values never leave the values' range: a tile adds 1/2 at most, as its largest score
// lies kRoom or more below the reference (log2), and with 1/2 in it the reference moves up by kRoom.  A new one lies kAbove above the largest score, whose
// weight then is a power of two, exact in bf16 (on whole numbers outputs were off by 0.0022 of their norm instead of 0.0018 to 0.0020): 8 more than it
// has to, as a tile that moves one waits for O (kAbove = 12: 4096 tokens 98 to 107 us).  What is below 2^-126 then counts as zero, 2^-110 of the
// row's sum.
constexpr float kRoom = 8.0f, kAbove = 16.0f;
constexpr int kItemRing = 2;

template <int D>
struct Cfg {
  static constexpr int HALVES = D / 64;
  static constexpr int HALF = kBT * 128;          // a 64-wide half of a tile: [128][128 B], swizzled
  static constexpr int TILE = HALVES * HALF;
  static constexpr int NS = D == 128 ? 2 : 4;     // stages of K, and of V
  // P: over S with D = 128, where S and O fill the TMEM; with D = 64 in columns of its own, and S of the next tile may be computed as soon
  // as S has been read, beside the softmax (P over S there: 280 us for 48 prompts of up to 1500 tokens)
  static constexpr bool P_APART = D == 64;
  static constexpr int P_COL = P_APART ? 384 : 0, P_STEP = P_APART ? 64 : kBT;
  static constexpr int NQ = D == 128 ? 1 : 2;     // buffers of an item's two tiles of Q
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = NQ * 2 * TILE;
  static constexpr int OFF_V = OFF_K + NS * TILE;
  static constexpr int OFF_ST = OFF_V + NS * TILE;  // the epilogue's rows on their way out: 2 KB a warp
  static constexpr int OFF_BAR = OFF_ST + 8 * 2048;
  static constexpr int N_BAR = 56;
  static constexpr int OFF_RING = OFF_BAR + N_BAR * 8;             // kItemRing x 64 bytes
  static constexpr int OFF_MISC = OFF_RING + kItemRing * 64;       // tmem base, abort flag, odd-value flags
  static constexpr int OFF_ML = OFF_MISC + 64;                     // float [2][128]: m, l of stream 1 for the join
  static constexpr int OFF_ODD = OFF_ML + 2 * kM * 4;              // int [2][3][D] first positions that see NaN, +inf, -inf
  static constexpr int OFF_FAR = OFF_ODD + 2 * 3 * D * 4;          // uint8 [2][128]: the row has had a reference far from zero
  static constexpr int SMEM = OFF_FAR + 2 * kM + 1024;             // + slack to align the base to 1024
  static_assert(SMEM <= 227 * 1024, "shared memory of one CTA on sm_103a");
};

template <int D>
struct Bars {
  using C = Cfg<D>;
  static constexpr int K_FULL = 0, K_EMPTY = C::NS, V_FULL = 2 * C::NS, V_EMPTY = 3 * C::NS;
  static constexpr int Q_FULL = 4 * C::NS, Q_EMPTY = Q_FULL + 2;  // [NQ]
  static constexpr int S_FULL = Q_EMPTY + 2, P_FULL = S_FULL + 2, O_FULL = P_FULL + 4;  // [2] per stream; P_APART: O_FULL after each P V
  static constexpr int IT_FULL = O_FULL + 2, IT_EMPTY = IT_FULL + kItemRing;
  static constexpr int V_CLEAN = IT_EMPTY + kItemRing;   // [NS] the tile's V has been looked at
  static constexpr int ODD_FREE = V_CLEAN + C::NS;           // [2] per buffer of odd values: its item's epilogues are done
  static constexpr int ML_FULL = ODD_FREE + 2, ML_EMPTY = ML_FULL + 1;  // stream 1's m and l (and O): published, read
  static constexpr int S_EMPTY = ML_EMPTY + 1;   // [2] S has been read (P_APART)
  static constexpr int TURN = S_EMPTY + 2;       // [2] the stream's issuer may go (P over S)
  static constexpr int MMA_DONE = TURN + 2, FIN = MMA_DONE + 1;
  static constexpr int KC_FULL = FIN + 1, VC_FULL = KC_FULL + C::NS;  // [NS] codes have arrived (8-bit cache)
  static_assert(VC_FULL + C::NS <= C::N_BAR, "barrier count");
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

// What the roles need to know of an item.
struct Shape {
  int nt;        // key tiles
  bool split;    // one tile of rows: its streams take the key tiles in turn
  int plain;     // key tiles from the first on that every row of the item sees entirely
};
__device__ __forceinline__ Shape shape_of(const WorkItem &w, int tile_rows, int tile_pos) {
  Shape s;
  s.nt = (w.t1 - w.t0 + kBT - 1) / kBT;
  s.split = w.rows <= tile_rows;
  const int all = min(w.t1, w.ctx + 2 * w.rg * tile_pos + 1);  // keys that the first row sees
  s.plain = max(all - w.t0, 0) / kBT;
  return s;
}

}  // namespace

template <int D, bool KV8>
__global__ void __launch_bounds__(threads_of(KV8), 1)
    prompt_tc_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ CUtensorMap tmq,
                     const __grid_constant__ CUtensorMap tmk, const __grid_constant__ CUtensorMap tmv,
                     const __grid_constant__ CUtensorMap tmk8, const __grid_constant__ CUtensorMap tmv8) {
  using C = Cfg<D>;
  using B = Bars<D>;
  constexpr int kThreads = threads_of(KV8);
  // registers: 12 warps launch with 168 each, 16 with 128; per scheduler 3 x 168 = 2 softmax warps + 1, or 4 x 128 = 2 + 1 that decodes + 1.
  // (Each split stands at the head of its own branch: after a join the compiler counts with the least.)
  constexpr int kSoftRegs = KV8 ? (D == 128 ? 168 : 184) : 200, kCodeRegs = D == 128 ? 96 : 72, kRestRegs = KV8 ? (D == 128 ? 80 : 72) : 104;
  static_assert(2 * kSoftRegs + kRestRegs + (KV8 ? kCodeRegs : 0) == (KV8 ? 4 * 128 : 3 * 168), "registers");
  // P is handed over in two halves of a tile's keys, so that the product with the first overlaps the softmax of the second: with D = 128 16384 tokens
  // 1239 -> 1187 us, 4096 101.5 -> 96.5; elsewhere the softmax warps' issue slots bound the tile, and it costs 2 to 3%.
  constexpr int kWhole = D == 128 && !KV8 ? 0 : 1;
  // With P in columns of its own the weights are computed beside the P V before and stored behind it: 48 prompts of up to 1500 tokens 250 ->
  // 247 us (over an 8-bit cache, with fewer registers, 196 -> 200).
  constexpr bool kBeside = C::P_APART && !KV8;
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
  volatile int *s_isodd = reinterpret_cast<volatile int *>(smem + C::OFF_MISC + 8);  // [2] an item's V held odd values
  float *s_ml = reinterpret_cast<float *>(smem + C::OFF_ML);
  int *s_odd = reinterpret_cast<int *>(smem + C::OFF_ODD);
  uint8_t *s_far = smem + C::OFF_FAR;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < C::NS; ++i) {
      ptx::mbar_init(bar(B::K_FULL + i), KV8 ? 4 : 1);
      ptx::mbar_init(bar(B::K_EMPTY + i), 2);  // both streams' issuers
      ptx::mbar_init(bar(B::V_FULL + i), KV8 ? 4 : 1);
      ptx::mbar_init(bar(B::KC_FULL + i), 1);
      ptx::mbar_init(bar(B::VC_FULL + i), 1);
      ptx::mbar_init(bar(B::V_EMPTY + i), 2);
      ptx::mbar_init(bar(B::V_CLEAN + i), 1);
    }
    for (int i = 0; i < C::NQ; ++i) {
      ptx::mbar_init(bar(B::Q_FULL + i), 1);
      ptx::mbar_init(bar(B::Q_EMPTY + i), 2);
    }
    for (int s = 0; s < 2; ++s) {
      ptx::mbar_init(bar(B::S_FULL + s), 1);
      ptx::mbar_init(bar(B::P_FULL + s), 4);      // the first half of a tile's keys
      ptx::mbar_init(bar(B::P_FULL + 2 + s), 4);  // the second
      ptx::mbar_init(bar(B::O_FULL + s), 1);
      ptx::mbar_init(bar(B::S_EMPTY + s), 4);
      ptx::mbar_init(bar(B::TURN + s), 1);
      ptx::mbar_init(bar(B::ODD_FREE + s), 8);
    }
    for (int i = 0; i < kItemRing; ++i) {
      ptx::mbar_init(bar(B::IT_FULL + i), 1);
      ptx::mbar_init(bar(B::IT_EMPTY + i), 8 + 2 + 1 + (KV8 ? 4 : 0));  // softmax warps, MMA issuers, the one that looks at V, decoders
    }
    ptx::mbar_init(bar(B::ML_FULL), 4);
    ptx::mbar_init(bar(B::ML_EMPTY), 4);
    ptx::mbar_init(bar(B::MMA_DONE), 2);
    ptx::mbar_init(bar(B::FIN), kThreads / 32);
    *s_abort = 0;
    s_isodd[0] = s_isodd[1] = 0;
    ptx::fence_mbar_init();
  }
  for (int i = threadIdx.x; i < 2 * 3 * D; i += kThreads) s_odd[i] = INT32_MAX;
  if (threadIdx.x < 2 * kM) s_far[threadIdx.x] = 0;
  if (warp == 9 && lane == 0) {
    ptx::prefetch_tmap(&tmq);
    ptx::prefetch_tmap(&tmk);
    ptx::prefetch_tmap(&tmv);
    ptx::prefetch_tmap(&tmk8);
    ptx::prefetch_tmap(&tmv8);
  }
  __syncwarp();
  if (warp == 8) {
    ptx::tmem_alloc(s_tmem, kTmemCols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *s_tmem;
  // everything above may overlap the planner (programmatic dependent launch)
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n_items = p.header->n_items;
  const int g = p.Hq / p.Hkv;
  const int tile_pos = kM / g, tile_rows = tile_pos * g;  // positions and rows of a tile

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

  bool ok = true;
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ------------------------------------------------------------------ softmax and epilogue, stream s, a row per thread
    const int s = warp >> 2;
    const int row = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + lanes + s * kBT, t_o = tmem + lanes + 2 * kBT + s * D, t_p = tmem + lanes + C::P_COL + s * C::P_STEP;
    const int pos0 = row / g;  // of this row within its tile
    // the epilogue: this lane's rows of the warp (8 x + lane / 4), as offsets from the tile's first row of the output
    const int warp0 = (warp & 3) * 32;
    int row_at[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int r = warp0 + 8 * x + (lane >> 2);
      row_at[x] = (r / g * p.Hq + r % g) * D;
    }
    const float scale = 1.4426950408889634f / sqrtf((float)D);
    const float2 scale2 = make_float2(scale, scale);
    uint32_t ns = 0, nml = 0, nof = 0;  // this stream's S tiles, joins and finished O so far
    WorkItem w;
    for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
      const Shape sh = shape_of(w, tile_rows, tile_pos);
      const int tile = sh.split ? 0 : s;
      const bool mine = row < tile_rows && tile * tile_rows + row < w.rows;
      const int pos = (2 * w.rg + tile) * tile_pos + pos0;
      const int end = min(w.t1, w.ctx + pos + 1);            // keys that it sees
      float m = -INFINITY, l = 0.0f;
      const int first = sh.split ? s : 0, inc = sh.split ? 2 : 1;
      for (int t = first; t < sh.nt; t += inc) {
        if (!wait_bar(bar(B::S_FULL + s), ns & 1, s_abort)) { ok = false; break; }
        ++ns;
        ptx::tc_fence_after();
        if (t >= sh.plain) {  // (in TMEM: a tile's usual way, and the other roles beside it, have to stay in the instruction cache; with this
                              // in registers 64 requests with a prefix took 80.8 us, 79.6 so, and e4m3 prompts 322 and 317)
          const int seen = end - (w.t0 + t * kBT);
#pragma unroll 1
          for (int c = 0; c < kBT; c += 32) {
            uint32_t y[32];
            ptx::tmem_ld32(t_s + c, y);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (c + i >= seen) y[i] = 0xff800000u;
            ptx::tmem_st32(t_s + c, y);
          }
          ptx::tmem_wait_st();
        }
        uint32_t x[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) ptx::tmem_ld32(t_s + 32 * c, x[c]);
        ptx::tmem_wait_ld();
        if (C::P_APART) {
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(B::S_EMPTY + s));
        }
        float mx[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          mx[c] = fmaxf(__uint_as_float(x[c][0]), __uint_as_float(x[c][1]));
#pragma unroll
          for (int i = 2; i < 32; i += 2) mx[c] = ptx::max3(mx[c], __uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1]));
        }
        const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
        bool done = !kBeside || t == first;
        auto finish = [&]() -> bool {  // the P V before: its P is written over, its O may be rescaled
          if (!wait_bar(bar(B::O_FULL + s), nof & 1, s_abort)) return false;
          ++nof;
          ptx::tc_fence_after();
          return true;
        };
        if (t == first) {
          m = top + kAbove;
        } else {
          if (C::P_APART && !kBeside && !finish()) { ok = false; break; }
          const bool move = mine && (top > m - kRoom || l > 0.5f);
          if (__any_sync(0xffffffffu, move)) {
            // (P over S: the O before this S is complete)
            if (kBeside) {
              if (!finish()) { ok = false; break; }
              done = true;
            }
            const float to = top > m - kRoom ? top + kAbove : m + kRoom;
            const float a = move ? ptx::ex2(m - to) : 1.0f;
            if (move && is_far(m)) s_far[threadIdx.x] = 1;
            if (move) m = to;
            l *= a;
#pragma unroll 1
            for (int c = 0; c < D; c += 16) {
              uint32_t o[16];
              ptx::tmem_ld16(t_o + c, o);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
              ptx::tmem_st16(t_o + c, o);
            }
          }
        }
        const float mm = m == -INFINITY ? 0.0f : -m;  // (nothing seen so far: every weight is zero)
        const float2 m2 = make_float2(mm, mm);
        float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        uint32_t pk[4][16];
        auto weigh = [&](int c) {
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float2 a = __ffma2_rn(make_float2(__uint_as_float(x[c][i]), __uint_as_float(x[c][i + 1])), scale2, m2);
            const float2 e = make_float2(ptx::ex2(a.x), ptx::ex2(a.y));
            sum[(i >> 1) & 1] = __fadd2_rn(sum[(i >> 1) & 1], e);
            pk[c][i >> 1] = pack_bf16(e.x, e.y);
          }
        };
        if (kBeside) {
#pragma unroll
          for (int c = 0; c < 4; ++c) weigh(c);
        }
        if (kBeside && !done && !finish()) { ok = false; break; }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          if (!kBeside) weigh(c);
          ptx::tmem_st16(t_p + 16 * c, pk[c]);
          if (c == 3 || (c == 1 && !kWhole)) {  // half of the keys: the product may begin
            ptx::tmem_wait_st();
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(bar(B::P_FULL + (c - 1) + s));
          }
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      }
      if (!ok) break;
      // ---- epilogue: the row's O
      bool far = is_far(m) || s_far[threadIdx.x];
      s_far[threadIdx.x] = 0;
      const bool join = sh.split && sh.nt > 1;
      const bool any = first < sh.nt;
      if (any) {
        if (!wait_bar(bar(B::O_FULL + s), nof & 1, s_abort)) { ok = false; break; }
        ++nof;
        ptx::tc_fence_after();
      }
      float a0 = 1.0f, a1 = 0.0f;
      if (join) {
        if (s == 1) {
          s_ml[row] = m;
          s_ml[kM + row] = far ? marked(l) : l;
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(B::ML_FULL));
          // (stream 0's threads read this O, too)
          if (!wait_bar(bar(B::ML_EMPTY), nml & 1, s_abort)) { ok = false; break; }
        } else {
          if (!wait_bar(bar(B::ML_FULL), nml & 1, s_abort)) { ok = false; break; }
          ptx::tc_fence_after();
          const float m1 = s_ml[row], l1 = s_ml[kM + row];
          far = far || is_marked(l1);
          const float mj = fmaxf(m, m1) + 1.0f;  // (the two sums together stay below 1, too)
          a0 = m == -INFINITY ? 0.0f : ptx::ex2(m - mj);
          a1 = m1 == -INFINITY ? 0.0f : ptx::ex2(m1 - mj);
          // (a stream that saw nothing has l = 0, or NaN scores only and l = NaN)
          l = (m == -INFINITY ? l : l * a0) + (m1 == -INFINITY ? l1 : l1 * a1);
          m = mj;
        }
        ++nml;
      }
      if (!(sh.split && s == 1)) {
        const float inv = 1.0f / l;
        const bool odd = s_isodd[j & 1] != 0;
        const int *so = s_odd + (j & 1) * 3 * D;
        // a lane's own row goes through the warp's 2 KB in pieces of 64 bytes, so that four lanes store a row's piece together (a lane
        // storing its row alone touches 32 lines per instruction)
        const bool part = w.poff >= 0;
        uint8_t *stage = smem + C::OFF_ST + warp * 2048;
        const int rows = min(min(tile_rows, w.rows - tile * tile_rows) - warp0, 32);  // and how many it has
        auto put = [&](int c, const uint32_t (&v)[4]) {
          *reinterpret_cast<uint4 *>(stage + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        };
        // this lane's share of 8 rows at a time: row 8 x + lane / 4, chunk lane % 4
        auto get = [&](int x) -> uint4 {
          const int r = 8 * x + (lane >> 2);
          return *reinterpret_cast<const uint4 *>(stage + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4));
        };
        uint8_t *dst[4];  // of those rows
        uint16_t *out0 = static_cast<uint16_t *>(p.out) + ((int64_t)(w.q0 + (2 * w.rg + tile) * tile_pos) * p.Hq + w.h * g) * D;
        float *part0 = p.partials + w.poff + (int64_t)(tile * tile_rows + warp0 + (lane >> 2)) * D;
#pragma unroll
        for (int x = 0; x < 4; ++x)
          dst[x] = (part ? reinterpret_cast<uint8_t *>(part0 + 8 * x * D) : reinterpret_cast<uint8_t *>(out0 + row_at[x])) + (lane & 3) * 16;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          ptx::tmem_ld32(t_o + c, o);
          ptx::tmem_wait_ld();
          if (join) {
            uint32_t o1[32];
            ptx::tmem_ld32(t_o + D + c, o1);
            ptx::tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              const float u = a0 == 0.0f ? 0.0f : __uint_as_float(o[i]) * a0;
              o[i] = __float_as_uint(a1 == 0.0f ? u : fmaf(__uint_as_float(o1[i]), a1, u));
            }
          }
          auto flush = [&](int at) {  // the staged pieces, to byte `at` of their rows
            __syncwarp();
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (8 * x + (lane >> 2) < rows) {
                if (part) __stcg(reinterpret_cast<uint4 *>(dst[x] + at), get(x));
                else *reinterpret_cast<uint4 *>(dst[x] + at) = get(x);
              }
            __syncwarp();
          };
          if (part) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int i = 16 * hf + 4 * e;
                const uint32_t v[4] = {o[i], o[i + 1], o[i + 2], o[i + 3]};
                put(e, v);
              }
              flush((c + 16 * hf) * 4);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t v[4];
#pragma unroll
              for (int i = 0; i < 4; ++i)
                v[i] = pack_bf16(__uint_as_float(o[8 * e + 2 * i]) * inv, __uint_as_float(o[8 * e + 2 * i + 1]) * inv);
              put(e, v);
            }
            flush(c * 2);
          }
        }
        if (odd) {  // V held values that are not finite: what they make of the rows that see them
          __syncwarp();
          uint16_t *dst16 = out0 + (row / g * p.Hq + row % g) * D;
          float *dst32 = p.partials + w.poff + (int64_t)(tile * tile_rows + row) * D;
#pragma unroll 1
          for (int i = 0; i < D; ++i) {
            const bool nan = pos >= so[i], up = pos >= so[D + i], down = pos >= so[2 * D + i];
            if (!mine || !(nan || up || down)) continue;
            const float add = nan || (up && down) ? __uint_as_float(0x7fffffffu) : up ? INFINITY : -INFINITY;
            if (part) dst32[i] = __ldcg(dst32 + i) + add;
            else dst16[i] = (uint16_t)pack_bf16(__uint_as_float((uint32_t)dst16[i] << 16) + add, 0.0f);
          }
        }
        if (part && mine) {
          float *stat = p.partials + w.poff + (int64_t)w.rows * D + tile * tile_rows + row;
          __stcg(stat, m);
          __stcg(stat + w.rows, far ? marked(l) : l);
        }
        if (far && mine) {
          hand_on(p, w.q0 + pos, w.h * g + row % g);
        }
        ptx::tc_fence_before();
        __syncwarp();
        if (join && lane == 0) ptx::mbar_arrive(bar(B::ML_EMPTY));
      }
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar(B::ODD_FREE + (j & 1)));
    }
  } else if (KV8 && warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kCodeRegs));
    // ------------------------------------------------------------------ codes to bf16
    const int row = (warp - 12) * 32 + lane;
    constexpr int CH = D / 16;  // 16-byte chunks of a row of codes
    uint32_t k0 = 0;
    WorkItem w;
    for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
      const int nt = (w.t1 - w.t0 + kBT - 1) / kBT, nblk = (w.t1 - w.t0 + 15) / 16;
      const int32_t *bt = p.block_tables + (int64_t)w.r * p.max_blocks_per_seq + w.t0 / 16;
      auto page = [&](int t) -> int {
        const int rel = 8 * t + row / 16;
        return rel < nblk ? __ldg(bt + rel) : -1;
      };
      auto scale_of = [&](const float *sc, int b) { return b >= 0 && b < p.num_blocks ? __ldg(sc + (int64_t)b * p.Hkv + w.h) : 0.0f; };
      auto decode = [&](uint8_t *tile, float sc) {
        // its own warp's rows lie over its own codes only
        const uint8_t *src = tile + (D == 128 ? C::HALF + row * 128 : (warp - 12) * 4096 + 2048 + lane * 64);
        uint4 v[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = *reinterpret_cast<const uint4 *>(src + (((c + lane) % CH) << 4));
        __syncwarp();
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          const int at = (c + lane) % CH;
          const uint32_t u[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
          uint32_t o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 f = __fmul2_rn(h2_to_f2(e4m3x2_to_h2(e & 1 ? u[e >> 1] >> 16 : u[e >> 1])), make_float2(sc, sc));
            o[e] = bf16x2_sat(f.x, f.y);
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int chunk = 2 * at + e;
            *reinterpret_cast<uint4 *>(tile + (chunk >> 3) * C::HALF + row * 128 + (((chunk & 7) ^ (row & 7)) << 4)) =
                make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        ptx::fence_proxy_async_smem();
        __syncwarp();
      };
      // scales one tile ahead, their pages two
      int b1 = page(0), b2 = page(1);
      float ks = scale_of(p.k_scale, b1), vs = scale_of(p.v_scale, b1), vs0 = 0.0f;
      for (int t = 0; t <= nt; ++t) {
        float ks1 = 0.0f, vs1 = 0.0f;
        if (t < nt) {
          ks1 = scale_of(p.k_scale, b2);
          vs1 = scale_of(p.v_scale, b2);
          b2 = page(t + 2);
          const uint32_t n = k0 + t;
          const int st = n % C::NS;
          if (!wait_bar(bar(B::KC_FULL + st), (n / C::NS) & 1, s_abort)) { ok = false; break; }
          decode(smem + C::OFF_K + st * C::TILE, ks);
          if (lane == 0) ptx::mbar_arrive(bar(B::K_FULL + st));
        }
        if (t > 0) {
          const uint32_t n = k0 + t - 1;
          const int st = n % C::NS;
          if (!wait_bar(bar(B::VC_FULL + st), (n / C::NS) & 1, s_abort)) { ok = false; break; }
          decode(smem + C::OFF_V + st * C::TILE, vs0);
          if (lane == 0) ptx::mbar_arrive(bar(B::V_FULL + st));
        }
        vs0 = vs;
        ks = ks1;
        vs = vs1;
      }
      k0 += nt;
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRestRegs));
    if (warp == 9) {
      // ------------------------------------------------------------------ items, Q, K, V
      uint32_t nk = 0, nv = 0, nq = 0;  // tiles and items' Q so far
      const WorkItem first_item = item_at(p, blockIdx.x);  // (read beside the items' number: there are at least as many places as CTAs)
      int claimed = (int)blockIdx.x < n_items ? (int)blockIdx.x : -1;
      auto claim = [&]() {
        if (lane == 0 && claimed == -2) {
          claimed = atomicAdd(&p.header_mut->next_item, 1);
          if (claimed >= n_items) claimed = -1;
        }
      };
      uint32_t j = 0;
      for (;; ++j) {
        const int slot = j % kItemRing;
        if (!wait_bar(bar(B::IT_EMPTY + slot), ((j / kItemRing) & 1) ^ 1, s_abort)) { ok = false; break; }
        claim();
        WorkItem w;
        int it = 0;
        if (lane == 0) {
          it = claimed;
          claimed = -2;
          s_ring[slot].it = it;
          if (it >= 0) s_ring[slot].w = j == 0 ? first_item : item_at(p, it);
        }
        it = __shfl_sync(0xffffffffu, it, 0);
        __syncwarp();
        w = s_ring[slot].w;
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(bar(B::IT_FULL + slot));
        if (it < 0) break;
        // K and V: K one tile ahead
        const int32_t *bt = p.block_tables + (int64_t)w.r * p.max_blocks_per_seq + w.t0 / 16;
        const int nblk = (w.t1 - w.t0 + 15) / 16;
        const int nt = (w.t1 - w.t0 + kBT - 1) / kBT;
        auto fetch = [&](int tile4) -> int {  // block ids of four tiles, a lane each
          const int i = tile4 * 32 + lane;
          return i < nblk ? __ldg(bt + i) : -1;
        };
        int prev = -1, cur = -1, next = fetch(0);
        auto load = [&](bool is_k, int t, int ids) -> bool {
          const uint32_t n = is_k ? nk : nv;
          const int s = n % C::NS;
          const int full = (KV8 ? (is_k ? B::KC_FULL : B::VC_FULL) : (is_k ? B::K_FULL : B::V_FULL)) + s;
          const int empty = (is_k ? B::K_EMPTY : B::V_EMPTY) + s;
          const int rel = 8 * t + (lane & 7);
          int bid = __shfl_sync(0xffffffffu, ids, rel & 31);
          if (!wait_bar(bar(empty), ((n / C::NS) & 1) ^ 1, s_abort)) return false;
          const bool valid = bid >= 0 && bid < p.num_blocks;
          if (is_k && lane < 8 && rel < nblk && !valid) report(p.status, WISP_DEV_BAD_BLOCK, p.request_ids, w.r);
          ++(is_k ? nk : nv);
          const uint32_t dst = sbase + (is_k ? C::OFF_K : C::OFF_V) + s * C::TILE;
          const int b0 = __shfl_sync(0xffffffffu, bid, 0);
          const bool row8 = __ballot_sync(0xffffffffu, lane < 8 && valid && bid == b0 + lane) == 0xffu;
          if (!valid) bid = p.num_blocks;  // past the item (or invalid): out-of-range box, reads zeros
          int bids[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) bids[x] = __shfl_sync(0xffffffffu, bid, x);
          const CUtensorMap *one = is_k ? &tmk : &tmv, *more = is_k ? &tmk8 : &tmv8;
          if (ptx::elect_one()) {
            ptx::mbar_arrive_expect_tx(bar(full), KV8 ? C::TILE / 2 : C::TILE);
            if constexpr (KV8) {
              // codes: where a warp's rows go it finds its two pages (D = 128: in the upper half of the tile; 64: of its own rows)
              if (D == 128) {
                if (row8) {
                  ptx::tma_load_4d(dst + C::HALF, more, bar(full), 0, 0, w.h, b0);
                } else {
#pragma unroll
                  for (int x = 0; x < 8; ++x) ptx::tma_load_4d(dst + C::HALF + x * (16 * 128), one, bar(full), 0, 0, w.h, bids[x]);
                }
              } else if (row8) {
#pragma unroll
                for (int x = 0; x < 4; ++x) ptx::tma_load_4d(dst + x * 4096 + 2048, more, bar(full), 0, 0, w.h, b0 + 2 * x);
              } else {
#pragma unroll
                for (int x = 0; x < 8; ++x)
                  ptx::tma_load_4d(dst + (x >> 1) * 4096 + 2048 + (x & 1) * 1024, one, bar(full), 0, 0, w.h, bids[x]);
              }
            } else if (row8) {
#pragma unroll
              for (int hf = 0; hf < C::HALVES; ++hf) ptx::tma_load_4d(dst + hf * C::HALF, more, bar(full), hf * 64, 0, w.h, b0);
            } else {
#pragma unroll
              for (int x = 0; x < 8; ++x)
#pragma unroll
                for (int hf = 0; hf < C::HALVES; ++hf)
                  ptx::tma_load_4d(dst + hf * C::HALF + x * (16 * 128), one, bar(full), hf * 64, 0, w.h, bids[x]);
            }
          }
          __syncwarp();
          return true;
        };
        for (int t = 0; t <= nt && ok; ++t) {
          if ((t & 3) == 0 && t < nt) {
            prev = cur;
            cur = next;
            next = fetch((t >> 2) + 1);
          }
          if (t < nt) ok = load(true, t, cur);
          if (t == 0 && ok) {  // Q: whole positions of the item's tiles
            const int qb = j % C::NQ;
            if (!wait_bar(bar(B::Q_EMPTY + qb), ((j / C::NQ) & 1) ^ 1, s_abort)) { ok = false; break; }
            ++nq;
            const int tiles = w.rows > tile_rows ? 2 : 1;
            if (ptx::elect_one()) {
              ptx::mbar_arrive_expect_tx(bar(B::Q_FULL + qb), (uint32_t)(tiles * C::HALVES * tile_rows * 128));
              for (int s = 0; s < tiles; ++s)
#pragma unroll
                for (int hf = 0; hf < C::HALVES; ++hf)
                  ptx::tma_load_4d(sbase + C::OFF_Q + (qb * 2 + s) * C::TILE + hf * C::HALF, &tmq, bar(B::Q_FULL + qb), hf * 64, 0, w.h,
                                   w.q0 + (2 * w.rg + s) * tile_pos);
            }
            __syncwarp();
          }
          if (t == max(nt - 2, 0)) claim();  // the next item, early enough to hide the way to it
          if (t > 0 && ok) ok = load(false, t - 1, (t & 3) == 0 && t < nt ? prev : cur);
        }
        if (!ok) break;
      }
      asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
      // drain: what was issued must land before the CTA's shared memory goes away
      if (lane == 0) {
        auto drain = [&](int full, uint32_t n) {
          for (uint32_t k = 0; k < C::NS && k < n; ++k) {
            const long long t0 = clock64();
            while (!ptx::mbar_try_wait(bar(full + (n - 1 - k) % C::NS), ((n - 1 - k) / C::NS) & 1) && clock64() - t0 < kWaitCycles) {
            }
          }
        };
        drain(KV8 ? B::KC_FULL : B::K_FULL, nk);
        drain(KV8 ? B::VC_FULL : B::V_FULL, nv);
        for (uint32_t k = 0; k < C::NQ && k < nq; ++k) {
          const long long t0 = clock64();
          while (!ptx::mbar_try_wait(bar(B::Q_FULL + (nq - 1 - k) % C::NQ), ((nq - 1 - k) / C::NQ) & 1) && clock64() - t0 < kWaitCycles) {
          }
        }
      }
    } else if (warp != 10) {
      // ------------------------------------------------------------------ MMA issuers, one per stream
      // (An MMA takes its issuer about 50 cycles and a commit 100, whatever it computes: one thread for both streams bounded the tile.)
      const int s = warp == 8 ? 0 : 1;
      const uint32_t idesc_s = ptx::idesc_bf16_f32(kM, kBT, false, false);
      const uint32_t idesc_o = ptx::idesc_bf16_f32(kM, D, false, true);
      uint32_t k0 = 0;               // key tiles of the items before
      uint32_t np = 0, ne = 0;       // P tiles and S tiles read so far
      // With P over S the issuers take turns: a stream's P V and next S go out together, and the other stream's behind them.  Without
      // that the tensor core works on both at once, both S arrive together, and then it waits for both softmaxes (a seventh more cycles
      // a tile).  An item's turns are as many for both, empty ones of stream 1 included.
      uint32_t turn = 0;
      auto my_turn = [&]() -> bool {
        if (C::P_APART) return true;
        const bool got = wait_bar(bar(B::TURN + s), (turn & 1) ^ (s == 0 ? 1 : 0), s_abort);
        ++turn;
        return got;
      };
      auto pass = [&]() {  // by one thread
        if (!C::P_APART) ptx::mbar_arrive(bar(B::TURN + 1 - s));
      };
      WorkItem w;
      for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
        const Shape sh = shape_of(w, tile_rows, tile_pos);
        const int first = sh.split ? s : 0, inc = sh.split ? 2 : 1;
        const int qb = j % C::NQ;
        if (!wait_bar(bar(B::Q_FULL + qb), (j / C::NQ) & 1, s_abort)) { ok = false; break; }
        // tiles of the other stream's alone: let go
        int kt = 0, vt = 0;
        auto skip = [&](int full, int empty, int &t, int to) -> bool {
          for (; t < to; ++t) {
            const int st = (k0 + t) % C::NS;
            if (!wait_bar(bar(full + st), ((k0 + t) / C::NS) & 1, s_abort)) return false;
            if (lane == 0) ptx::mbar_arrive(bar(empty + st));
          }
          return true;
        };
        auto issue_s = [&](int t) -> bool {
          if (!skip(B::K_FULL, B::K_EMPTY, kt, t)) return false;
          kt = t + 1;
          const uint32_t n = k0 + t;
          const int st = n % C::NS;
          if (!wait_bar(bar(B::K_FULL + st), (n / C::NS) & 1, s_abort)) return false;
          if (ptx::elect_one()) {
            ptx::tc_fence_after();
            const uint64_t qd = ptx::sdesc_sw128(sbase + C::OFF_Q + (qb * 2 + (sh.split ? 0 : s)) * C::TILE, 16, 1024);
            const uint64_t kd = ptx::sdesc_sw128(sbase + C::OFF_K + st * C::TILE, 16, 1024);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
              const int off = ((ks >> 2) * C::HALF + (ks & 3) * 32) >> 4;
              ptx::umma_f16(tmem + s * kBT, qd + off, kd + off, idesc_s, ks > 0);
            }
            pass();
            ptx::umma_commit(bar(B::S_FULL + s));
            ptx::umma_commit(bar(B::K_EMPTY + st));
            if (t + inc >= sh.nt) ptx::umma_commit(bar(B::Q_EMPTY + qb));
          }
          __syncwarp();
          return true;
        };
        if (!my_turn()) { ok = false; break; }
        if (first < sh.nt) {
          ok = issue_s(first);
        } else if (lane == 0) {
          ptx::mbar_arrive(bar(B::Q_EMPTY + qb));
          pass();
        }
        for (int t = first; t < sh.nt && ok; t += inc) {
          if (C::P_APART && t + inc < sh.nt) {
            if (!wait_bar(bar(B::S_EMPTY + s), ne & 1, s_abort)) { ok = false; break; }
            ok = issue_s(t + inc);
            if (!ok) break;
          }
          ++ne;
          ok = skip(B::V_FULL, B::V_EMPTY, vt, t);
          if (!ok) break;
          vt = t + 1;
          const uint32_t n = k0 + t;
          const int st = n % C::NS;
          if (!wait_bar(bar(B::V_FULL + st), (n / C::NS) & 1, s_abort) ||
              !wait_bar(bar(B::V_CLEAN + st), (n / C::NS) & 1, s_abort)) {
            ok = false;
            break;
          }
          ok = my_turn();
          if (!ok) break;
#pragma unroll
          for (int half = kWhole; half < 2; ++half) {
            if (!wait_bar(bar(B::P_FULL + 2 * half + s), np & 1, s_abort)) { ok = false; break; }
            if (ptx::elect_one()) {
              ptx::tc_fence_after();
              const uint64_t vd = ptx::sdesc_sw128(sbase + C::OFF_V + st * C::TILE, C::HALF, 1024);
#pragma unroll
              for (int ks = kWhole ? 0 : 4 * half; ks < 4 * half + 4; ++ks)
                ptx::umma_f16_ts(tmem + 2 * kBT + s * D, tmem + C::P_COL + s * C::P_STEP + ks * 8, vd + ((ks * 16 * 128) >> 4), idesc_o,
                                 t != first || ks > 0);
              if (half == 1) {
                if (t + inc >= sh.nt) pass();
                if (C::P_APART || t + inc >= sh.nt) ptx::umma_commit(bar(B::O_FULL + s));
                ptx::umma_commit(bar(B::V_EMPTY + st));
              }
            }
            __syncwarp();
          }
          if (!ok) break;
          ++np;
          if (!C::P_APART && t + inc < sh.nt) ok = issue_s(t + inc);
        }
        if (ok && sh.split && s == 1 && (sh.nt & 1)) {  // stream 0 has a tile more
          ok = my_turn();
          if (ok && lane == 0) pass();
        }
        if (ok) ok = skip(B::K_FULL, B::K_EMPTY, kt, sh.nt) && skip(B::V_FULL, B::V_EMPTY, vt, sh.nt);
        k0 += sh.nt;
      }
      if (ptx::elect_one()) {
        // every MMA issued must finish before the TMEM is released
        ptx::umma_commit(bar(B::MMA_DONE));
        const long long t0 = clock64();
        while (!ptx::mbar_try_wait(bar(B::MMA_DONE), 0) && clock64() - t0 < kWaitCycles) {
        }
      }
    } else if (warp == 10) {
      // ------------------------------------------------------------------ V of tiles that some row does not see entirely
      uint32_t k0 = 0;
      WorkItem w;
      for (uint32_t j = 0; ok && next_item(j, w, ok); ++j) {
        const Shape sh = shape_of(w, tile_rows, tile_pos);
        const int ob = j & 1;
        // this item's buffer of odd values: free, and cleared where it was used
        if (!wait_bar(bar(B::ODD_FREE + ob), ((j >> 1) & 1) ^ 1, s_abort)) { ok = false; break; }
        if (s_isodd[ob]) {
          __syncwarp();
          for (int i = lane; i < 3 * D; i += 32) s_odd[ob * 3 * D + i] = INT32_MAX;
          s_isodd[ob] = 0;
          __syncwarp();
        }
        for (int t = 0; t < sh.nt; ++t) {
          const uint32_t n = k0 + t;
          const int st = n % C::NS;
          if (!wait_bar(bar(B::V_FULL + st), (n / C::NS) & 1, s_abort)) { ok = false; break; }
          if (t < sh.plain) {
            if (lane == 0) ptx::mbar_arrive(bar(B::V_CLEAN + st));
            continue;
          }
#pragma unroll 1
          for (int x = 0; x < kBT / 32; ++x) {
            const int row = x * 32 + lane;
            uint8_t *line = smem + C::OFF_V + st * C::TILE + row * 128;
            __nv_bfloat162 acc = __floats2bfloat162_rn(0.0f, 0.0f);
            const __nv_bfloat162 zero = acc;
#pragma unroll
            for (int c = 0; c < 8 * C::HALVES; ++c) {  // (no two of eight lanes read the same banks)
              const uint4 v = *reinterpret_cast<const uint4 *>(line + (c >> 3) * C::HALF + (((c + lane) & 7) << 4));
              const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) acc = __hfma2(*reinterpret_cast<const __nv_bfloat162 *>(&u[e]), zero, acc);
            }
            if (__low2float(acc) + __high2float(acc) == 0.0f) continue;  // every value is finite
            const int key = w.t0 + t * kBT + row;
            for (int c = 0; c < 8 * C::HALVES; ++c)
              for (int e = 0; e < 8; ++e) {
                uint16_t *at = reinterpret_cast<uint16_t *>(line + (c >> 3) * C::HALF + ((c & 7) << 4)) + e;
                const uint32_t bits = *at;
                if ((bits & 0x7f80u) != 0x7f80u) continue;
                *at = 0;
                if (key >= w.t1) continue;  // nobody's
                const int d = (c >> 3) * 64 + (((c & 7) ^ (row & 7)) << 3) + e;
                const int kind = (bits & 0x7fu) ? 0 : (bits & 0x8000u) ? 2 : 1;
                atomicMin(&s_odd[(ob * 3 + kind) * D + d], max(key - w.ctx, 0));  // the first position that sees it
                s_isodd[ob] = 1;
              }
          }
          __threadfence_block();
          ptx::fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(bar(B::V_CLEAN + st));
        }
        k0 += sh.nt;
      }
      }
  }

  if (!ok && lane == 0) report(p.status, WISP_DEV_TIMEOUT, p.request_ids, -1);
  // teardown: the TMEM is freed once every warp has said that it is done with it
  __syncwarp();
  ptx::tc_fence_before();
  if (lane == 0) ptx::mbar_arrive(bar(B::FIN));
  if (warp == 8) {
    const long long t0 = clock64();
    while (!ptx::mbar_try_wait(bar(B::FIN), 0) && clock64() - t0 < kWaitCycles) {
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

// A 4-D tensor with D innermost, in boxes of b0 elements x b1 x 1 x b3: bf16, 64 elements (128 bytes, swizzled), or codes.
cudaError_t encode(CUtensorMap *map, bool codes, const void *base, int D, int64_t n1, int64_t n2, int64_t n3, int b1, int b3) {
  const cuuint64_t es = codes ? 1 : 2;
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)n1, (cuuint64_t)n2, (cuuint64_t)n3};
  const cuuint64_t strides[3] = {D * es, n1 * D * es, n2 * n1 * D * es};
  const cuuint32_t box[4] = {(cuuint32_t)(codes ? D : 64), (cuuint32_t)b1, 1, (cuuint32_t)b3};
  const cuuint32_t ones[4] = {1, 1, 1, 1};
  const CUresult r = g_encode(map, codes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                              const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              codes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

template <int D, bool KV8>
cudaError_t launch(const AttnParams &p, int total_q_rows, int grid, cudaStream_t s) {
  const int g = p.Hq / p.Hkv, more = KV8 && D == 64 ? 2 : 8;  // pages in a box of several
  CUtensorMap tq, tk, tv, tk8, tv8;
  cudaError_t e = encode(&tq, false, p.q, D, g, p.Hkv, total_q_rows, g, kM / g);
  if (e == cudaSuccess) e = encode(&tk, KV8, p.k_cache, D, 16, p.Hkv, p.num_blocks, 16, 1);
  if (e == cudaSuccess) e = encode(&tv, KV8, p.v_cache, D, 16, p.Hkv, p.num_blocks, 16, 1);
  if (e == cudaSuccess) e = encode(&tk8, KV8, p.k_cache, D, 16, p.Hkv, p.num_blocks, 16, more);
  if (e == cudaSuccess) e = encode(&tv8, KV8, p.v_cache, D, 16, p.Hkv, p.num_blocks, 16, more);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg;
  std::memset(&cfg, 0, sizeof cfg);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(threads_of(KV8));
  cfg.dynamicSmemBytes = Cfg<D>::SMEM;
  cfg.stream = s;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, prompt_tc_kernel<D, KV8>, p, tq, tk, tv, tk8, tv8);
}

template <int D, bool KV8>
cudaError_t setup() {
  return cudaFuncSetAttribute(prompt_tc_kernel<D, KV8>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<D>::SMEM);
}

}  // namespace

cudaError_t prompt_tc_setup() {
  cudaError_t e = get_encode();
  if (e == cudaSuccess) e = setup<128, false>();
  if (e == cudaSuccess) e = setup<128, true>();
  if (e == cudaSuccess) e = setup<64, false>();
  return e == cudaSuccess ? setup<64, true>() : e;
}

cudaError_t prompt_tc_launch(const AttnParams &p, int total_q_rows, int grid, cudaStream_t s) {
  if (p.k_scale) return p.D == 128 ? launch<128, true>(p, total_q_rows, grid, s) : launch<64, true>(p, total_q_rows, grid, s);
  return p.D == 128 ? launch<128, false>(p, total_q_rows, grid, s) : launch<64, false>(p, total_q_rows, grid, s);
}

}  // namespace wisp
