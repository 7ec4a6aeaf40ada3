// sc_expert_linear.cu -- matrix products grouped by expert, ragged sizes known on
// the device alone.  Expert e has the slots offsets[e] .. offsets[e + 1]:
//   forward       out[s][n]    = act(sum_k x[row(s)][k] W_e[n][k] + b_e[n])
//   back (input)  out[s][k]    = (sum_n dy[s][n] W_e[n][k]) GELU'(pre[s][k])
//   back (weight) out[e][n][k] = sum_s dy[s][n] x[row(s)][k],  db_e[n] = sum_s dy[s][n]
//
// Pair kernel: tcgen05 products of two CTAs (cta_group::2), M = 256.  The weight's
// features are the M side, so it is always full; the ragged slots are the N side,
// whose width follows what an expert has (64 to 256, evenly split over its tiles)
// -- or, in the weight gradient, the contraction.  Persistent CTA pairs walk the
// tiles that exist; every role counts them out from the offsets.
//   warp 0      copies the operands, 64 of the contraction a stage, four to six stages
//   warp 1      (even CTA) issues the products into one of two 256-column accumulators
//   16 warps    (weight gradient: eight) read the other accumulator back, 32 features x
//               32 columns at a time, through a staging area of the warp's own and tiled
//               copies.  Each chunk is a chain of short waits, so the more warps the
//               better hidden: with eight, GELU cost 7 us of 41
//   four warps more (rows of x gathered) copy these rows, 16 bytes a thread: four-row
//               TMA gathers of 128-byte rows took 81 cycles each, 8 x 1024 rows x 2
//               experts 768 -> 1536 99 us against 34 without the gather
//   four warps more (weight gradient) sum dy over the slots for the bias, from the
//               stages in shared memory (by the gathering warps 63 us instead of 47)
// Operands as they lie in memory: K-major where the contraction is contiguous
// (forward; dy in back (input)), else MN-major (W in back (input), both sides of the
// weight gradient), 128-byte swizzle throughout.
// A long contraction is bound by the operands' way from the L2 into shared memory, which the
// outputs' way out shares: 59,000 slots 2048 -> 1024 164 us (1.5 PFLOP/s; without the copies
// 123; 180 to 188 on other boxes).  A short one is not: 16384 slots 768 -> 1536 35 us (1.1), with
// GELU and the value before it 43 (50 MB more to write).  There the tiles of eight uneven
// experts are 5.3 to 5.45 rounds of the pairs, run as six, and launch, first copies and last
// write-back cost 6 us a call (one expert of 16384 slots: 33 us, the library's product 25).
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>
#include <cstdint>

#include "sc_expert.cuh"
#include "sm103_primitives.cuh"

namespace sc {

PFN_cuTensorMapEncodeTiled_v12000 api_tensor_map_encoder();

constexpr int kPairM = 128;          // features per CTA, 256 per pair
constexpr int kPairN = 256;          // widest tile on the other side; half of it per CTA
constexpr int kPairStep = 64;        // contraction per stage: one 128-byte swizzle atom
constexpr int kPairMaxStages = 6;
constexpr int kPairChunk = 32;       // columns read back at a time
constexpr uint32_t kPairABytes = kPairM * kPairStep * 2;
constexpr uint32_t kPairBBytes = kPairN / 2 * kPairStep * 2;
constexpr uint32_t kPairStageBytes = kPairABytes + kPairBBytes;
constexpr uint32_t kPairBoxBytes = 64 * kPairStep * 2;   // 64 x 64 box of an MN-major operand
// The tensor cores add to an fp32 accumulator with truncation, half a unit in the last
// place per 16 of the contraction: 2048 slots, 3.7e-6, growing with their number.  For
// fp32 outputs an accumulator takes kSpan stages (512 of the contraction) only; eight
// write-back warps add it, rounded, to sums in their registers (128 a thread; weight
// gradient: 64, and as many in the write-back areas, for the registers of the other
// warps).  Any depth from 512: 4.7e-7, torch's fp32 product 1.3e-7 to 3.9e-7.  bf16 outputs
// do not show the truncation of the forward product and of the rows' gradient, 8192 deep at
// most.  The weight gradient's depth is the number of slots: past kLongSlots, where an expert
// might lose 1.2e-4, a sixteenth of bf16's half unit, bf16 weights take the spans too (and no
// wait is for more than eight stages).  65600 slots of 8 experts, 768 x 1536: 120 us without,
// 130 with them.
constexpr int kSpan = 8;
constexpr int kLongSlots = 65536;
// kF32: sums over spans; of fp32 outputs, and of bf16 weight gradients of many slots.
// kPre: with the value before GELU, written (forward) or read (back, input).
template <ExpertProduct kWhat, bool kGather_, bool kF32_, bool kPre_>
struct PairKind {
  static constexpr bool kFwd = kWhat == ExpertProduct::kForward;
  static constexpr bool kBackX = kWhat == ExpertProduct::kBackInput;
  static constexpr bool kBackW = kWhat == ExpertProduct::kBackWeight;
  static constexpr bool kGather = kGather_, kF32 = kF32_, kPre = kPre_;
  static constexpr int kSteps = kF32 ? kSpan : 1 << 30;   // stages an accumulator takes
  // Warps: four (copies, products), the write-back, four that gather, four that sum dy.
  static constexpr int kEpiWarps = kBackW || kF32 ? 8 : 16;
  static constexpr int kGatherWarp = 4 + kEpiWarps, kSumWarp = kGatherWarp + (kGather ? 4 : 0);
  static constexpr int kThreads = 32 * (kSumWarp + (kBackW ? 4 : 0));
  // Registers where fp32 sums need them, of the write-back warps, of the first four and of
  // the others: what 65536 (61440 with 640 threads) leave.
  static constexpr bool kSplit = kF32 && (!kBackW || kGather);
  static constexpr int kEpiRegs = kBackW ? 128 : kThreads <= 384 ? 208 : 192;
  static constexpr int kFirstRegs = kBackW ? 72 : kThreads <= 384 ? 88 : 56;
  static constexpr int kAuxRegs = 72;
  // Write-back areas per warp.  Forward: a chunk of the output (bf16 2 KB, fp32 4) and one
  // of the value before GELU.  Back (weight): two chunks of 4 KB, the copy of one on its
  // way while the other is filled.  Back (input): a chunk of the output and a ring of two
  // chunks of the value before GELU, copied ahead across tiles: behind the copies of the
  // operands a load waits 3000 cycles.  Where there is none, its room is a stage's (59,000
  // slots, 2048 -> 1024: four stages 180 us, five 167, six 164).
  static constexpr uint32_t kChunkBytes = kF32 || kBackW ? 4096 : 2048;
  static constexpr uint32_t kPreBytes = 2048;
  static constexpr uint32_t kOutBytes =
      kBackW || kF32 ? 8192 : kChunkBytes + (!kPre ? 0 : kBackX ? 2 * kPreBytes : kPreBytes);
  static constexpr int kStages = kBackW || kF32 ? 5 : !kPre ? 6 : kBackX ? 4 : 5;
  static_assert(kStages <= kPairMaxStages, "barriers");
  static constexpr uint32_t kDyn = kStages * kPairStageBytes + kEpiWarps * kOutBytes + 1024;
};

// Weight gradient: most tiles beside the pairs' first ones that are dealt out.
constexpr int kMaxDealt = 160;

struct PairParams {
  ExpertLinearParams p;
  CUtensorMap map_a;     // forward: W, 128 x 64; back (input): W, 64 x 64; back (weight): dy, 64 x 64
  CUtensorMap map_b;     // other side, not gathered: 128 x 64, back (weight) 64 x 64
  CUtensorMap map_b32;   // ... 32 x 64 (tiles narrower than 256)
  CUtensorMap map_out;   // output, 32 x 32 boxes (128-byte swizzle in fp32, 64-byte in bf16)
  CUtensorMap map_pre;   // forward: the value before GELU, likewise
};

struct PairSmem {
  uint64_t full[kPairMaxStages], empty[kPairMaxStages];   // full: of the even CTA, both CTAs' copies
  uint64_t done[kPairMaxStages];                       // products done, the bias sums not yet
  uint64_t landed[kPairMaxStages];                     // this CTA's gathered rows
  uint64_t tfull[2], tempty[2];                     // tempty: of the even CTA
  uint64_t fin;                                     // every product issued is done
  uint64_t stall;                                   // test hook: never completed
  uint32_t tmem_base;
  int abort;
  // after a wait that ran out in either CTA: fills of the even CTA's `full` barriers, by the
  // two copying warps and the two threads that hand gathered rows over
  int gave_up, fills[2], handed[2];
  alignas(16) uint32_t mark[4];   // of the even CTA: written by the odd one's signals
  union {
    int tile0[kMaxExperts + 1];   // forward, back (input): tiles of slots of the experts before
    alignas(16) float sums[2][kPairM];   // weight gradient: bias sums of two warps each
  };
  uint8_t order[kMaxExperts];   // weight gradient: experts by decreasing number of slots
  // ... and the tiles this pair takes after its first, where they are dealt out
  int deal, dealt_n;
  uint64_t dealt_out;           // barrier: the list is there
  uint16_t dealt[kMaxDealt];
};

__device__ __forceinline__ float bf_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// GELU and its slope from the normal distribution's lower tail Phi(-|x|), in packed
// pairs: the read-back warps bound products with GELU.  Phi(-a) = exp(-a^2 / 2) t P(t),
// t = 1 / (1 + q a): with exp(a^2 / 2) taken out, what is left is smooth, and a polynomial P
// has it to a relative precision over 0 .. 14 (least-squares fits, weighted until the largest
// relative error was least: 1e-7 with eight terms).  An approximation of erf itself has no
// digits in the tail (x = -5 came 5 % off).  With eight terms GELU is within (16 + x^2) 2^-24
// of itself and its slope of Phi + |x| phi, x^2 for the rounded argument of the exponential.
// Six terms (kShort) are for what is rounded to bf16: 1.1e-6 up to 2, where most arguments
// lie, growing to 3.3e-5, a sixtieth of bf16's half unit, in the tail (5e-6 throughout moved four
// times as many values across a rounding boundary).  16384 slots, 768 -> 1536, with the value
// before GELU 45.9 us, GELU' 46.9; eight terms cost 0.6 and 0.8 more.
__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float relu_nan(float x) {
  float y;
  asm("max.NaN.f32 %0, %1, 0f00000000;" : "=f"(y) : "f"(x));
  return y;
}
// Phi(-a) = qt e, e = exp(-a^2 / 2), for na = -a, -16 <= na <= 0 (beyond it e is 0; clamped, so that a
// pair may share a reciprocal)
template <bool kShort>
__device__ __forceinline__ void normal_tail2(uint64_t na, uint64_t& qt, uint64_t& e) {
  float d0, d1, e0, e1;
  f2_unpack(f2_fma(na, f2_both(kShort ? -0.3f : -0.304f), f2_both(1.f)), d0, d1);
  f2_unpack(f2_mul(f2_mul(na, na), f2_both(-0.5f * 1.44269504088896341f)), e0, e1);
  // 1 / d0 and 1 / d1 from one reciprocal
  const uint64_t t = f2_mul(f2_pack(d1, d0), f2_both(rcp_approx(d0 * d1)));
  uint64_t q;
  if constexpr (kShort) {
    q = f2_fma(f2_both(-0.0807364211f), t, f2_both(0.226450577f));
    q = f2_fma(q, t, f2_both(-0.0280712485f));
    q = f2_fma(q, t, f2_both(0.149643015f));
    q = f2_fma(q, t, f2_both(0.11254811f));
    q = f2_fma(q, t, f2_both(0.120165424f));
  } else {
    q = f2_fma(f2_both(0.0366238666f), t, f2_both(-0.154347755f));
    q = f2_fma(q, t, f2_both(0.190593448f));
    q = f2_fma(q, t, f2_both(-0.0416993671f));
    q = f2_fma(q, t, f2_both(0.122815459f));
    q = f2_fma(q, t, f2_both(0.102640969f));
    q = f2_fma(q, t, f2_both(0.122136511f));
    q = f2_fma(q, t, f2_both(0.121236869f));
  }
  qt = f2_mul(q, t);
  e = f2_pack(ex2(e0), ex2(e1));
}
// GELU(x) = max(x, 0) - |x| Phi(-|x|); 0 at -infinity
template <bool kShort>
__device__ __forceinline__ void gelu2(float& x0, float& x1) {
  const uint64_t na = f2_pack(fmaxf(-fabsf(x0), -16.f), fmaxf(-fabsf(x1), -16.f));
  uint64_t qt, e;
  normal_tail2<kShort>(na, qt, e);
  f2_unpack(f2_fma(na, f2_mul(qt, e), f2_pack(relu_nan(x0), relu_nan(x1))), x0, x1);
}
// y *= GELU'(x): with s = Phi(-|x|) - |x| phi(x), s for negative x and 1 - s for others
template <bool kShort>
__device__ __forceinline__ void gelu_slope2(float x0, float x1, float& y0, float& y1) {
  const uint64_t na = f2_pack(fmaxf(-fabsf(x0), -16.f), fmaxf(-fabsf(x1), -16.f));
  uint64_t qt, e;
  normal_tail2<kShort>(na, qt, e);
  const uint64_t s = f2_mul(f2_fma(na, f2_both(0.3989422804014327f), qt), e);
  const uint64_t way = f2_pack(-copysignf(1.f, x0), -copysignf(1.f, x1));   // way s + (1 - way) / 2
  // + 0 x: NaN where x is (or infinite, as x phi(x) is)
  const uint64_t base = f2_fma(f2_pack(x0, x1), f2_both(0.f), f2_fma(way, f2_both(-0.5f), f2_both(0.5f)));
  f2_unpack(f2_mul(f2_pack(y0, y1), f2_fma(way, s, base)), y0, y1);
}

// One output tile of the pair: features f0 .. f0 + 256 of expert e, and slots
// lo + i0 .. (n of them, `width` columns) or, in the weight gradient, the columns
// i0 .. of the other side with the slots lo .. hi as the contraction.
struct PairTile {
  int e, lo, hi, f0, i0, n, width;
};

// Slots of a tile of an expert with n slots: evenly split, multiples of 64.  As wide as
// they go: the L2's rate to the SMs bounds long products (32 KB a stage and SM at about
// 54 bytes a cycle, 600 cycles where the products take 512), so narrower tiles lose more
// by copying the weights again than they win by evener rounds (96 columns: 81 us, not 34).
__device__ __forceinline__ int tile_slots(int n) {
  const int tiles = (n + kPairN - 1) / kPairN;
  return tiles == 0 ? 64 : ((n + tiles - 1) / tiles + 63) & ~63;
}

template <ExpertProduct kWhat>
__device__ __forceinline__ int features(const ExpertLinearParams& p) {
  return kWhat == ExpertProduct::kBackInput ? p.K : p.N;
}

// Tile t (in increasing order per role: t.e is advanced).
template <ExpertProduct kWhat>
__device__ __forceinline__ void pair_tile(const ExpertLinearParams& p, const PairSmem& sm, int t,
                                          PairTile& g) {
  const int tiles_f = (features<kWhat>(p) + 255) / 256;
  const int rest = t / tiles_f;
  g.f0 = (t - rest * tiles_f) * 256;
  if constexpr (kWhat == ExpertProduct::kBackWeight) {
    const int tiles_k = (p.K + kPairN - 1) / kPairN, o = rest / tiles_k;
    g.e = sm.order[o];
    g.i0 = (rest - o * tiles_k) * kPairN;
    expert_range(p, g.e, g.lo, g.hi);
    g.n = min(kPairN, p.K - g.i0);
  } else {
    while (sm.tile0[g.e + 1] <= rest) ++g.e;
    expert_range(p, g.e, g.lo, g.hi);
    const int w = tile_slots(g.hi - g.lo);
    g.i0 = (rest - sm.tile0[g.e]) * w;
    g.n = min(w, g.hi - g.lo - g.i0);
  }
  g.width = (g.n + 63) & ~63;
}

template <ExpertProduct kWhat>
__device__ __forceinline__ int pair_steps(const ExpertLinearParams& p, const PairTile& g) {
  const int depth = kWhat == ExpertProduct::kForward ? p.K
                    : kWhat == ExpertProduct::kBackInput ? p.N : g.hi - g.lo;
  return (depth + kPairStep - 1) / kPairStep;
}

// The tiles of a pair, in order.  Forward, back (input): every pairs-th.  Weight gradient:
// the tiles come by decreasing contraction, and where each pair has a few, they are
// dealt out one by one to the pair with the least so far (8 experts of 1002 to 3884 slots,
// two tiles a pair: every pairs-th 98 stages for the longest, there and back 76, dealt 68,
// the mean 61); where they have more, there and back.
template <ExpertProduct kWhat>
struct TileWalk {
  int t, i, pair, pairs, tiles;
  __device__ __forceinline__ TileWalk(int pair_, int pairs_, int tiles_)
      : t(pair_), i(0), pair(pair_), pairs(pairs_), tiles(tiles_) {}
  __device__ __forceinline__ bool more() const { return t < tiles; }
  __device__ __forceinline__ void next(PairSmem& sm) {
    if constexpr (kWhat != ExpertProduct::kBackWeight) {
      t += pairs;
    } else if (sm.deal) {
      // the dealing warp waits for nothing; whatever gives up elsewhere, all see the list
      bool ok = false;
      for (int polls = 0; !ok && polls < 1 << 22; ++polls) ok = mbar_try_wait_poll(&sm.dealt_out, 0);
      t = ok && i < sm.dealt_n ? sm.dealt[i] : tiles;
    } else {
      t = (i + 1) * pairs + (i % 2 == 0 ? pairs - 1 - pair : pair);
    }
    ++i;
  }
};

// Deals out tiles pairs .. tiles of the weight gradient, the first ones being the pairs'
// own; one warp, while the first ones are at work.  A tile's cost: its stages, and six for
// what it costs beside them.
__device__ __forceinline__ void deal_tiles(const ExpertLinearParams& p, PairSmem& sm, int pair, int pairs,
                                           int tiles) {
  constexpr int kPer = 5;   // pairs a lane
  const int lane = threadIdx.x & 31;
  const int each = tiles / p.E;   // tiles of an expert
  const auto cost = [&](int o) {
    int lo, hi;
    expert_range(p, sm.order[o], lo, hi);
    return static_cast<uint32_t>(min((hi - lo + kPairStep - 1) / kPairStep, 1 << 20) + 6);
  };
  uint32_t load[kPer];
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int o = lane + 32 * q;
    load[q] = o < pairs && o < tiles ? cost(o / each) : 0xffffffu;
  }
  int n = 0;
  uint32_t now = 0;
  for (int t = pairs; t < tiles; ++t) {
    if (t == pairs || t % each == 0) now = cost(t / each);
    uint32_t best = 0xffffffffu;
#pragma unroll
    for (int q = 0; q < kPer; ++q) best = min(best, min(load[q], 0xffffffu) << 8 | (lane + 32 * q));
    const int to = static_cast<int>(__reduce_min_sync(0xffffffffu, best) & 255u);
#pragma unroll
    for (int q = 0; q < kPer; ++q)
      if (to == lane + 32 * q) load[q] += now;
    if (to == pair) {
      if (lane == 0) sm.dealt[n] = static_cast<uint16_t>(t);
      ++n;
    }
  }
  if (lane == 0) {
    sm.dealt_n = n;
    mbar_arrive(&sm.dealt_out);
  }
  __syncwarp();
}

__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort) {
  return __all_sync(0xffffffffu, mbar_wait_poll(bar, parity, abort));
}

// Bounded wait that ignores the abort flag (teardown: no copy or product may still use
// this CTA's memory when it exits).
__device__ __forceinline__ void drain_wait_pair(uint64_t* bar, uint32_t parity) {
  int dummy = 0;
  mbar_wait(bar, parity, &dummy, 1000000000ull);
}

// Hands a stage that threads of this CTA wrote (and ordered before the products by a proxy fence)
// to the even CTA, whose product reads it: an arrival on `full` there.  The odd CTA's comes
// with a copy of 16 bytes, issued after the fence: its completion is a release over the
// cluster, to the product's acquire, and nobody waits for it here.  (An arrival of the CTA's scope
// alone orders nothing across CTAs; one with a release over the cluster holds its thread
// for most of a stage: 69 us, not 37, for 16384 slots 768 -> 1536.  GELU and the value before it
// 45.9 to 46.3 us so, 44.8 with the bare arrival; the weight gradient 47.9 and 47.4.)
__device__ __forceinline__ void hand_over(PairSmem& sm, int rank, int s) {
  const uint32_t full = dsmem_addr(smem_u32(&sm.full[s]), 0);
  if (rank == 0) {
    mbar_arrive(&sm.full[s]);
  } else {
    mbar_arrive_expect_tx_cluster(full, 16);
    bulk_copy16_cluster(dsmem_addr(smem_u32(sm.mark), 0), smem_u32(sm.mark), full);
  }
}

// The copies of both CTAs that are on their way, awaited by one thread of the even CTA once
// no role starts another: all of them count on its `full` barriers.  A stage is filled again
// only after everyone's last fill of it, so the fills of a stage differ by one at most;
// whoever gave up before the last one is stood in for.  (Not inlined: its registers cost the
// fp32 weight gradient 100 bytes of spills.)
template <int kStages, bool kGather>
__device__ __noinline__ void drain_copies(PairSmem& sm) {
#pragma unroll 1
  for (int q = 0; q < kStages; ++q) {
    const auto of = [&](int n) { return n / kStages + (q < n % kStages ? 1 : 0); };
    int n[4] = {of(sm.fills[0]), of(sm.fills[1])};
    if constexpr (kGather) n[2] = of(sm.handed[0]), n[3] = of(sm.handed[1]);
    int most = 0;
#pragma unroll
    for (int i = 0; i < (kGather ? 4 : 2); ++i) most = max(most, n[i]);
    if (most == 0) continue;
#pragma unroll
    for (int i = 0; i < (kGather ? 4 : 2); ++i)
      if (n[i] < most) mbar_arrive(&sm.full[q]);
    drain_wait_pair(&sm.full[q], (most - 1) & 1);
  }
}

// The rows of a last, partial stage of the weight gradient: 64 slots x 128 columns of a
// matrix into two 64 x 64 boxes, zeros past the expert's slots and the matrix's columns
// (a product with what lies there would not be 0 for NaN), by the copying warp itself.
__device__ __forceinline__ void copy_partial(uint32_t dst, const uint16_t* src, long long ld, int col0,
                                             int cols, int s0, int hi) {
  const int lane = threadIdx.x & 31;
#pragma unroll 4
  for (int q = lane; q < 2 * 64 * 8; q += 32) {
    const int c = q & 15, r = q >> 4;              // 16-byte piece of row r
    const int s = s0 + r, col = col0 + 8 * c;
    const bool in = s < hi && col < cols;
    cp_async16(dst + (c >> 3) * kPairBoxBytes + sw128_offset(r, c & 7),
               src + (in ? static_cast<long long>(s) * ld + col : 0), in);
  }
}

// A warp's staged chunk, 32 features of up to 32 slots (`left` of them in the tile), to
// rows slot0 .. of a [.][width] output: one tiled copy, or, where the tile ends within
// the chunk, the lanes' own stores of the slots that are there (the rows after it are
// another expert's).
template <bool kF32>
__device__ __forceinline__ void put_chunk(const CUtensorMap& map, void* out, const uint8_t* from, int slot0,
                                          int left, int f, int width, bool ok) {
  const int lane = threadIdx.x & 31;
  if (!ok || f >= width) return;
  if (left >= kPairChunk) {
    if (lane == 0) tma_store_2d(&map, f, slot0, smem_u32(from));
    return;
  }
  constexpr int kPieces = kF32 ? 8 : 4, kPer = kF32 ? 4 : 8;   // 16-byte pieces a row, values a piece
  const int x = lane % kPieces;
#pragma unroll 1
  for (int r = lane / kPieces; r < left; r += 32 / kPieces) {
    if (f + kPer * x >= width) break;
    const size_t at = static_cast<size_t>(slot0 + r) * width + f + kPer * x;
    *reinterpret_cast<uint4*>(static_cast<uint8_t*>(out) + at * (kF32 ? 4 : 2)) =
        *reinterpret_cast<const uint4*>(from + stage_offset<kPieces>(r, x));
  }
}

template <ExpertProduct kWhat, bool kGather, bool kF32, bool kPre>
__global__ void __launch_bounds__(PairKind<kWhat, kGather, kF32, kPre>::kThreads, 1)
    sc_expert_pair_kernel(const __grid_constant__ PairParams P) {
  using Kind = PairKind<kWhat, kGather, kF32, kPre>;
  constexpr bool kFwd = Kind::kFwd, kBackX = Kind::kBackX, kBackW = Kind::kBackW;
  constexpr int kStages = Kind::kStages, kEpiWarps = Kind::kEpiWarps, kGroups = kEpiWarps / 4;
  constexpr int kGatherWarp = Kind::kGatherWarp, kSumWarp = Kind::kSumWarp;
  static_assert(sizeof(PairSmem) + Kind::kDyn <= 227 * 1024, "one CTA's shared memory");
  const ExpertLinearParams& p = P.p;
  extern __shared__ uint8_t dyn_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  __shared__ PairSmem sm;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = static_cast<int>(cluster_rank());
  const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const bool sums = kBackW && p.dbias != nullptr;

  if (tid == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&sm.full[s], kGather ? 4 : 2);     // per CTA: the copies' (with their bytes), gathered rows
      mbar_init(&sm.landed[s], 128);
      mbar_init(&sm.empty[s], sums ? 4 : 1);       // the products', or the summing warps'
      mbar_init(&sm.done[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      mbar_init(&sm.tfull[a], 1);
      mbar_init(&sm.tempty[a], 2 * kEpiWarps);
    }
    mbar_init(&sm.dealt_out, 1);
    mbar_init(&sm.fin, 1);
    mbar_init(&sm.stall, 1);
    sm.abort = sm.gave_up = 0;
    fence_mbar_init();
  }
  if (warp == 1) tmem_alloc_pair(&sm.tmem_base, 512);
  // what the launch before this one writes is read from here on
  pdl_wait();
  pdl_launch_dependents();
  if constexpr (!kBackW) {
    if (warp == 0) {
      int total = 0;
#pragma unroll 1
      for (int e0 = 0; e0 < p.E; e0 += 32) {
        const int e = e0 + lane;
        int x = 0;
        if (e < p.E) {
          int lo, hi;
          expert_range(p, e, lo, hi);
          const int w = tile_slots(hi - lo);
          x = (hi - lo + w - 1) / w;
        }
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {   // inclusive scan
          const int y = __shfl_up_sync(0xffffffffu, x, off);
          if (lane >= off) x += y;
        }
        if (e < p.E) sm.tile0[e + 1] = total + x;
        total += __shfl_sync(0xffffffffu, x, 31);
      }
      if (lane == 0) sm.tile0[0] = 0;
    }
  }
  if constexpr (kBackW) {
    // ranks by (slots, expert)
    for (int e = tid; e < p.E; e += blockDim.x) {
      int lo, hi, rank_e = 0;
      expert_range(p, e, lo, hi);
      const int n = hi - lo;
      for (int o = 0; o < p.E; ++o) {
        expert_range(p, o, lo, hi);
        rank_e += hi - lo > n || (hi - lo == n && o < e);
      }
      sm.order[rank_e] = static_cast<uint8_t>(e);
    }
  }
  if constexpr (kBackW) {
    const int n = p.E * ((p.N + 255) / 256) * ((p.K + kPairN - 1) / kPairN);
    if (tid == 0) sm.deal = pairs <= 160 && n > pairs && n - pairs <= kMaxDealt;
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();   // the other CTA's barriers are set up
  tc_fence_after();
  const uint32_t tm = sm.tmem_base;
  volatile int* abort_flag = &sm.abort;
  const uint32_t ring = smem_u32(base);
  const int tiles = ((features<kWhat>(p) + 255) / 256) *
                    (kBackW ? p.E * ((p.K + kPairN - 1) / kPairN) : sm.tile0[p.E]);
  PairTile g;
  g.e = 0;
  TileWalk<kWhat> walk(pair, pairs, tiles);

  if (warp >= 4 && warp < 4 + kEpiWarps) {
    if constexpr (Kind::kSplit) regs_alloc<Kind::kEpiRegs>();
    // ------------------------------------------------------------- write back
    const int q = warp & 3, grp = (warp - 4) >> 2;
    uint8_t* const stg = base + kStages * kPairStageBytes + (warp - 4) * Kind::kOutBytes;
    uint8_t* const stg_pre = stg + Kind::kChunkBytes;   // forward: of the value before GELU; back (input): ring
    const int pr = lane >> 2, px = lane & 3;   // this lane's 16-byte piece of columns pr + 8 k
    const int mi = lane >> 3;                  // fragment whose row address this lane gives
    const uint32_t tempty0 = dsmem_addr(smem_u32(&sm.tempty[0]), 0);
    bool ok = true;
    int j = 0, n_out = 0;
    // the next chunk's area: no earlier copy reads it any more
    const auto next_area = [&]() {
      if (lane == 0) bulk_wait_read<kBackW ? 1 : 0>();
      __syncwarp();
      return stg + (kBackW ? (n_out++ & 1) * 4096 : 0);
    };
    // back (input): chunks of `pre` on their way
    PairTile ahead;
    ahead.e = ahead.n = 0;
    int ht = pair - pairs, hc = 0, slot_in = 0, slot_out = 0;
    const auto copy_pre = [&]() {
      hc += kGroups * kPairChunk;
      while (ht < tiles && hc >= ahead.n) {
        ht += pairs;
        hc = kPairChunk * grp;
        if (ht < tiles) pair_tile<kWhat>(p, sm, ht, ahead);
      }
      if (ht < tiles) {
        const int x = ahead.f0 + rank * kPairM + 32 * q + 8 * px;
        const uint32_t to = smem_u32(stg_pre + slot_in * Kind::kPreBytes);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = 8 * k + pr;
          const bool in = hc + r < ahead.n && x < p.K;
          cp_async16(to + stage_offset<4>(r, px),
                     p.pre_in + (in ? (static_cast<size_t>(ahead.lo) + ahead.i0 + hc + r) * p.K + x : 0), in);
        }
      }
      cp_async_commit();
      slot_in ^= 1;
    };
    if (kBackX && kPre && p.pre_in != nullptr) {
      copy_pre();
      copy_pre();
    }
    // forward: a tile's bias is loaded during the tile before
    float bias[2][2] = {}, bias_next[2][2] = {};
    const auto load_bias = [&](const PairTile& g1) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int n = g1.f0 + rank * kPairM + 32 * q + 16 * h + 8 * u + lane / 4;
          if (n < p.N) bias_next[h][u] = __ldg(p.bias + static_cast<size_t>(g1.e) * p.N + n);
        }
    };
    if (kFwd && p.bias != nullptr && pair < tiles) {
      pair_tile<kWhat>(p, sm, pair, ahead);
      load_bias(ahead);
    }
    // weight gradient in bf16: 32 rows (features) of 32 columns, contiguous in memory, from
    // column c, a row a lane; from `to`, which no copy and no lane reads any more
    const auto put_pieces = [&](uint8_t* to, int f, int c, const uint4 (&v)[4]) {
#pragma unroll
      for (int k = 0; k < 4; ++k) stage_row_piece<4>(to, k, v[k]);
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) {
        tma_store_3d(&P.map_out, g.i0 + c, f, g.e, smem_u32(to));   // cut at N and K
        bulk_commit();
      }
    };
    const auto pack_row = [&](uint4 (&w)[4], const float (&v)[32]) {
#pragma unroll
      for (int k = 0; k < 32; k += 8)
        w[k / 8] = make_uint4(pack_bf16x2(v[k], v[k + 1]), pack_bf16x2(v[k + 2], v[k + 3]),
                              pack_bf16x2(v[k + 4], v[k + 5]), pack_bf16x2(v[k + 6], v[k + 7]));
    };
    // forward, back (input): 32 rows (features) of the 32 columns (slots) from c, in
    // fragments, transposed on the way out
    const auto put_columns = [&](int f, int c, float (&v)[2][16]) {
      const int width = features<kWhat>(p), slot0 = g.lo + g.i0 + c, left = g.n - c;
      // where this lane's row of fragment pair (h, b) is staged
      const auto at = [&](int h, int b) {
        return stage_offset<4>(8 * (b + (mi >> 1)) + (lane & 7), 2 * h + (mi & 1));
      };
      const auto pack = [&](uint32_t (&w)[2][8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 8; ++k) w[h][k] = pack_bf16x2(v[h][2 * k], v[h][2 * k + 1]);
      };
      const auto store = [&](uint8_t* area, const uint32_t (&w)[2][8]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < 4; b += 2)
            stmatrix4_trans(smem_u32(area + at(h, b)), w[h][2 * b], w[h][2 * b + 1], w[h][2 * b + 2],
                            w[h][2 * b + 3]);
      };
      if (kBackX && kPre && p.pre_in != nullptr) {
        // in the staging's layout, so that its fragments match the accumulator's
        uint32_t zf[2][2][4];
        cp_async_wait<1>();
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < 4; b += 2)
            ldmatrix4_trans(smem_u32(stg_pre + slot_out * Kind::kPreBytes + at(h, b)), zf[h][b / 2]);
        __syncwarp();
        slot_out ^= 1;
        copy_pre();
        if (!kF32) tmem_ld_wait();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint32_t x = zf[h][k >> 2][k & 3];
            gelu_slope2<!kF32>(bf_lo(x), bf_hi(x), v[h][2 * k], v[h][2 * k + 1]);
          }
      } else if (!kF32) {
        tmem_ld_wait();
      }
      if constexpr (kFwd) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 16; ++k) v[h][k] += bias[h][(k >> 1) & 1];
      }
      const auto gelu = [&]() {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 16; k += 2) gelu2<!kF32>(v[h][k], v[h][k + 1]);
      };
      uint8_t* to;
      uint32_t w[2][8];
      if constexpr (kF32) {
        // (its sums leave no registers for the value before GELU beside them)
        to = next_area();
        if (kFwd && kPre && p.pre != nullptr) {
          pack(w);
          store(stg_pre, w);
        }
        if (kFwd && p.gelu) gelu();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const int r = 8 * (k >> 2) + 2 * (lane & 3) + (k & 1);
            const int n = 16 * h + 8 * ((k >> 1) & 1) + lane / 4;
            *reinterpret_cast<float*>(to + stage_offset<8>(r, n >> 2) + 4 * (n & 3)) = v[h][k];
          }
      } else {
        // all arithmetic before the area is waited for (after it: 16384 slots,
        // 768 -> 1536 with GELU, 38.9 us instead of 37.7)
        uint32_t w_pre[2][8];
        if (kFwd && kPre && p.pre != nullptr) pack(w_pre);
        if (kFwd && p.gelu) gelu();
        pack(w);
        to = next_area();
        if (kFwd && kPre && p.pre != nullptr) store(stg_pre, w_pre);
        store(to, w);
      }
      fence_proxy_async_smem();
      __syncwarp();
      put_chunk<kF32>(P.map_out, p.out, to, slot0, left, f, width, ok);
      if (kFwd && kPre && p.pre != nullptr) put_chunk<false>(P.map_pre, p.pre, stg_pre, slot0, left, f, width, ok);
      if (lane == 0) bulk_commit();
    };
    for (; walk.more(); walk.next(sm)) {
      pair_tile<kWhat>(p, sm, walk.t, g);
      const int steps = pair_steps<kWhat>(p, g);
      const int f = g.f0 + rank * kPairM + 32 * q;   // this warp's features
      if (kFwd && p.bias != nullptr) {
#pragma unroll
        for (int u = 0; u < 4; ++u) bias[u >> 1][u & 1] = bias_next[u >> 1][u & 1];
        if (walk.t + pairs < tiles) {
          pair_tile<kWhat>(p, sm, walk.t + pairs, ahead);
          load_bias(ahead);
        }
      }
      const auto await_sum = [&]() {   // of the tile, or of its next stages
        ok = ok && warp_wait(&sm.tfull[j & 1], (j >> 1) & 1, abort_flag);
        tc_fence_after();
        return tm + (j & 1) * kPairN + (static_cast<uint32_t>(32 * q) << 16);
      };
      const auto release_sum = [&]() {   // the accumulator may be written again
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(tempty0 + 8 * (j & 1));
        ++j;
      };
      if constexpr (!kF32) {
        const uint32_t d = steps > 0 ? await_sum() : 0;
#pragma unroll 1
        for (int c = kPairChunk * grp; c < g.n; c += kGroups * kPairChunk) {
          if constexpr (kBackW) {
            if (!ok || f >= p.N) break;
            float v[32];
            if (steps > 0) {
              tmem_ld32(d + c, v);
              tmem_ld_wait();
            } else {
#pragma unroll
              for (int k = 0; k < 32; ++k) v[k] = 0.f;   // an expert without slots
            }
            uint4 w[4];
            pack_row(w, v);
            put_pieces(next_area(), f, c, w);
          } else {
            float v[2][16];
            tmem_ld_frag32(d + c, v[0]);
            tmem_ld_frag32(d + c + (16u << 16), v[1]);
            put_columns(f, c, v);
          }
        }
        if (steps > 0) release_sum();
      } else if constexpr (kBackW) {
        // columns 32 grp + 64 i: i = 0, 1 in registers, 2, 3 in the write-back areas, a
        // row a lane as they leave
        float sum[2][32];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int k = 0; k < 32; ++k) sum[i][k] = 0.f;
        if (lane == 0) bulk_wait_read<0>();
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          stage_row_piece<8>(stg, k, make_uint4(0, 0, 0, 0));
          stage_row_piece<8>(stg + 4096, k, make_uint4(0, 0, 0, 0));
        }
#pragma unroll 1
        for (int k0 = 0; k0 < steps; k0 += Kind::kSteps) {
          const uint32_t d = await_sum();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = kPairChunk * (grp + 2 * i);
            if (c >= g.n) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float v[16];
              tmem_ld16(d + c + 16 * h, v);
              tmem_ld_wait();
              if (i < 2) {
#pragma unroll
                for (int k = 0; k < 16; ++k) sum[i & 1][16 * h + k] += v[k];
              } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  float4* const at =
                      reinterpret_cast<float4*>(stg + (i - 2) * 4096 + stage_offset<8>(lane, 4 * h + k));
                  const float4 was = *at;
                  *at = make_float4(was.x + v[4 * k], was.y + v[4 * k + 1], was.z + v[4 * k + 2],
                                    was.w + v[4 * k + 3]);
                }
              }
            }
          }
          release_sum();
        }
        // the areas' columns leave, then the registers' through them
        if (!p.out_f32) {
#pragma unroll
          for (int o = 0; o < 4; ++o) {
            uint8_t* const area = stg + (o & 1) * 4096;
            const int c = kPairChunk * (grp + 2 * (o < 2 ? 2 + o : o - 2));
            uint4 w[4];
            if (o < 2) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const float4 a = *reinterpret_cast<const float4*>(area + stage_offset<8>(lane, 2 * k));
                const float4 b = *reinterpret_cast<const float4*>(area + stage_offset<8>(lane, 2 * k + 1));
                w[k] = make_uint4(pack_bf16x2(a.x, a.y), pack_bf16x2(a.z, a.w), pack_bf16x2(b.x, b.y),
                                  pack_bf16x2(b.z, b.w));
              }
            } else {
              pack_row(w, sum[o & 1]);
              if (o == 2 && lane == 0) bulk_wait_read<0>();
            }
            __syncwarp();
            if (ok && f < p.N && c < g.n) put_pieces(area, f, c, w);
          }
        } else {
#pragma unroll
          for (int i = 2; i >= 0; i -= 2) {
            if (i == 0) {
              if (lane == 0) bulk_wait_read<0>();
              __syncwarp();
#pragma unroll
              for (int k = 0; k < 32; k += 4)
#pragma unroll
                for (int o = 0; o < 2; ++o)
                  stage_row_piece<8>(stg + 4096 * o, k / 4,
                                     make_uint4(__float_as_uint(sum[o][k]), __float_as_uint(sum[o][k + 1]),
                                                __float_as_uint(sum[o][k + 2]), __float_as_uint(sum[o][k + 3])));
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0 && ok && f < p.N) {
#pragma unroll
              for (int o = 0; o < 2; ++o) {
                const int c = kPairChunk * (grp + 2 * (i + o));
                if (c < g.n) tma_store_3d(&P.map_out, g.i0 + c, f, g.e, smem_u32(stg + 4096 * o));   // cut at N and K
              }
              bulk_commit();
            }
          }
        }
      } else {
        // columns 32 grp + 64 i
        float sum[4][2][16];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int k = 0; k < 32; ++k) sum[i][k >> 4][k & 15] = 0.f;
#pragma unroll 1
        for (int k0 = 0; k0 < steps; k0 += Kind::kSteps) {
          const uint32_t d = await_sum();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int c = kPairChunk * (grp + 2 * i);
            if (c >= g.n) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float v[16];
              tmem_ld_frag32(d + c + (static_cast<uint32_t>(16 * h) << 16), v);
              tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < 16; ++k) sum[i][h][k] += v[k];
            }
          }
          release_sum();
        }
#pragma unroll 1
        for (int c = kPairChunk * grp; c < g.n; c += 2 * kPairChunk) {
          put_columns(f, c, sum[0]);
#pragma unroll
          for (int i = 0; i < 3; ++i)
#pragma unroll
            for (int k = 0; k < 32; ++k) sum[i][k >> 4][k & 15] = sum[i + 1][k >> 4][k & 15];
        }
      }
    }
    if (lane == 0) bulk_wait_all();
    if (kBackX) cp_async_wait_all();
  } else {
    if constexpr (Kind::kSplit) {
      if (warp < 4) regs_dealloc<Kind::kFirstRegs>();
      else regs_dealloc<Kind::kAuxRegs>();
    }
    if (warp == 0) {
      // ------------------------------------------------------------- copies
      bool ok = true;
      int s = 0, use = 0;
      for (; ok && walk.more(); walk.next(sm)) {
        pair_tile<kWhat>(p, sm, walk.t, g);
        const int steps = pair_steps<kWhat>(p, g);
        const int f = g.f0 + rank * kPairM;             // this CTA's features
        const int half = kBackW ? kPairN / 2 : g.width / 2;
        const int b0 = g.i0 + rank * half;              // ... and its columns of the tile
        const uint32_t bytes = kPairABytes + (kGather ? 0 : half * kPairStep * 2);
#pragma unroll 1
        for (int kt = 0; kt < steps; ++kt) {
          if (use > 0 && !(ok = warp_wait(&sm.empty[s], (use - 1) & 1, abort_flag))) break;
          const uint32_t a = ring + s * kPairStageBytes, b = a + kPairABytes;
          const uint32_t full = dsmem_addr(smem_u32(&sm.full[s]), 0);
          const int c0 = kt * kPairStep;
          if (kBackW && g.lo + c0 + kPairStep > g.hi) {
            copy_partial(a, p.dy, p.ldy, f, p.N, g.lo + c0, g.hi);
            if constexpr (!kGather) copy_partial(b, p.x, p.ldx, b0, p.K, g.lo + c0, g.hi);
            cp_async_wait_all();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) hand_over(sm, rank, s);
          } else if (lane == 0) {
            mbar_arrive_expect_tx_cluster(full, bytes);
            if constexpr (kFwd) {
              tma_load_3d_pair(a, &P.map_a, c0, f, g.e, full);
            } else if constexpr (kBackX) {
              tma_load_3d_pair(a, &P.map_a, f, c0, g.e, full);
              tma_load_3d_pair(a + kPairBoxBytes, &P.map_a, f + 64, c0, g.e, full);
            } else {
              tma_load_2d_pair(a, &P.map_a, f, g.lo + c0, full);
              tma_load_2d_pair(a + kPairBoxBytes, &P.map_a, f + 64, g.lo + c0, full);
            }
            if constexpr (!kGather) {
              if constexpr (kBackW) {
                tma_load_2d_pair(b, &P.map_b, b0, g.lo + c0, full);
                tma_load_2d_pair(b + kPairBoxBytes, &P.map_b, b0 + 64, g.lo + c0, full);
              } else if (half == kPairN / 2) {
                tma_load_2d_pair(b, &P.map_b, c0, g.lo + b0, full);
              } else {
                for (int q = 0; q < half; q += 32)
                  tma_load_2d_pair(b + q * 128, &P.map_b32, c0, g.lo + b0 + q, full);
              }
            }
          }
          __syncwarp();
          if (++s == kStages) {
            s = 0;
            ++use;
          }
        }
      }
      // every stage's products are done, and their arrivals have come, before this CTA ends
#pragma unroll 1
      for (int q = 0; q < kStages; ++q) {
        const int fills = use + (q < s ? 1 : 0);
        if (fills > 0) warp_wait(&sm.empty[q], (fills - 1) & 1, abort_flag);
      }
      // (the other CTA waits for this one's copies and products, and would for two seconds)
      if (lane == 0 && *abort_flag) st_cluster_u32(dsmem_addr(smem_u32(&sm.abort), rank ^ 1), 1u);
      if (lane == 0) st_cluster_u32(dsmem_addr(smem_u32(&sm.fills[rank]), 0), use * kStages + s);
    } else if (warp == 1) {
      // ------------------------------------------------------------- products
      if (rank == 0 && elect_one()) {
        bool ok = p.stall_ns == 0 || mbar_wait(&sm.stall, 0, abort_flag, p.stall_ns);
        int s = 0, use = 0, j = 0;
        for (; ok && walk.more(); walk.next(sm)) {
          pair_tile<kWhat>(p, sm, walk.t, g);
          const int steps = pair_steps<kWhat>(p, g);
          if (steps == 0) continue;
          const uint32_t idesc = idesc_bf16(256, kBackW ? kPairN : g.width, !kFwd, kBackW);
          // low descriptor words: K-major operands advance 32 bytes per 16 of the
          // contraction, MN-major ones two groups of eight 128-byte rows; their other
          // 64-feature boxes lie 8 KB apart
          constexpr uint32_t kFar = (kPairBoxBytes >> 4) << 16, kNear = 1u << 16;
          constexpr uint32_t kStepA = kFwd ? 2 : 128, kStepB = kBackW ? 128 : 2;
#pragma unroll 1
          for (int kt = 0; kt < steps; ++kt) {
            const int acc = j & 1, k0 = kt % Kind::kSteps;
            // the accumulator's previous sum has been read back
            if (k0 == 0 && j >= 2 &&
                !(ok = mbar_wait_poll(&sm.tempty[acc], ((j >> 1) - 1) & 1, abort_flag)))
              break;
            const uint32_t d = tm + acc * kPairN;
            if (kGather || (kBackW && g.lo + (kt + 1) * kPairStep > g.hi)) {   // written by threads
              if (!(ok = mbar_wait_cluster(&sm.full[s], use & 1, abort_flag))) break;
              fence_proxy_async_smem();
            } else if (!(ok = mbar_wait_poll(&sm.full[s], use & 1, abort_flag))) {
              break;
            }
            tc_fence_after();
            const uint32_t at = ring + s * kPairStageBytes;
            const uint32_t a = (at >> 4) | (kFwd ? kNear : kFar);
            const uint32_t b = ((at + kPairABytes) >> 4) | (kBackW ? kFar : kNear);
#pragma unroll
            for (int k = 0; k < kPairStep / 16; ++k)
              umma_bf16_pair_lo(d, a + kStepA * k, b + kStepB * k, idesc, (k0 | k) != 0);
            umma_commit_pair(sums ? &sm.done[s] : &sm.empty[s]);
            if (++s == kStages) {
              s = 0;
              ++use;
            }
            if (k0 == Kind::kSteps - 1 || kt == steps - 1) {
              umma_commit_pair(&sm.tfull[acc]);
              ++j;
            }
          }
        }
        umma_commit_pair(&sm.fin);
      }
      __syncwarp();
    } else if (kGather && warp == 2) {
      // ------------------------------------------------------------- gathered rows handed over
      // (what threads write to shared memory is ordered before the products by the proxy fence)
      if (elect_one()) {
        bool ok = true;
        int s = 0, use = 0;
        for (; ok && walk.more(); walk.next(sm)) {
          pair_tile<kWhat>(p, sm, walk.t, g);
          const int steps = pair_steps<kWhat>(p, g);
#pragma unroll 1
          for (int kt = 0; kt < steps; ++kt) {
            if (!(ok = mbar_wait_poll(&sm.landed[s], use & 1, abort_flag))) break;
            fence_proxy_async_smem();
            hand_over(sm, rank, s);
            if (++s == kStages) {
              s = 0;
              ++use;
            }
          }
        }
        st_cluster_u32(dsmem_addr(smem_u32(&sm.handed[rank]), 0), use * kStages + s);
      }
      __syncwarp();
    } else if (kGather && warp >= kGatherWarp && warp < kGatherWarp + 4) {
      // ------------------------------------------------------------- gathered rows
      const int l = tid - 32 * kGatherWarp;
      bool ok = true;
      int s = 0, use = 0;
      // forward: 8 pieces of each of up to 128 rows, the rows the same in every stage;
      // weight gradient: 16 pieces of each of 64 rows, other rows in every stage
      constexpr int kPieces = kFwd ? 8 : 16, kRowStep = 128 / kPieces;
      const int c = l % kPieces, r0 = l / kPieces;
      // this thread's piece of row r0 in a stage; rows r0 + kRowStep i lie 128 kRowStep i on
      static_assert(kRowStep % 8 == 0, "the same swizzle");
      const uint32_t to = kPairABytes + (c >> 3) * kPairBoxBytes + sw128_offset(r0, c & 7);
      for (; ok && walk.more(); walk.next(sm)) {
        pair_tile<kWhat>(p, sm, walk.t, g);
        const int steps = pair_steps<kWhat>(p, g);
        const int half = kBackW ? kPairN / 2 : g.width / 2;
        const int b0 = g.i0 + rank * half;
        const uint16_t* src[8];
        // weight gradient: the 16 rows that this warp copies of each of eight stages, two
        // stages a register; those of the eight after them are loaded meanwhile (a load
        // waits up to 3000 cycles behind the operands: four stages ahead 50 us, not 44)
        int row[4], row_next[4];
        const auto load_rows = [&](int kt) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = (r0 & ~1) + (lane & 1) + 8 * ((lane & 15) >> 1);
            row_next[i] = expert_row(p, min(g.lo + (kt + 2 * i + (lane >> 4)) * kPairStep + r, p.M - 1));
          }
        };
        // (few instructions a copy: the four warps have a stage's time for them)
        const int col = b0 + 8 * c;
        const char* const x_col = reinterpret_cast<const char*>(p.x + (col < p.K ? col : 0));
        const uint32_t row_bytes = static_cast<uint32_t>(p.ldx) * 2u;
        if constexpr (kFwd) {
          // columns past the tile repeat its last slot
#pragma unroll
          for (int i = 0; i < 8; ++i)
            src[i] = p.x + 8 * c +
                     p.ldx * expert_row(p, g.lo + min(b0 + r0 + kRowStep * i, g.i0 + g.n - 1));
        } else {
          load_rows(0);
        }
#pragma unroll 1
        for (int kt = 0; kt < steps; ++kt) {
          if (use > 0 && !(ok = warp_wait(&sm.empty[s], (use - 1) & 1, abort_flag))) break;
          const uint32_t dst = ring + s * kPairStageBytes + to;
          const int c0 = kt * kPairStep;
          if constexpr (kFwd) {
            const bool in = c0 + 8 * c < p.K;
#pragma unroll
            for (int i = 0; i < 8; ++i)
              if (r0 + kRowStep * i < half)
                cp_async16(dst + 128 * kRowStep * i, src[i] + (in ? c0 : 0), in);
          } else {
            if (kt % 8 == 0) {
#pragma unroll
              for (int i = 0; i < 4; ++i) row[i] = row_next[i];
              load_rows(kt + 8);
            }
            const int two = kt % 8 < 4 ? (kt % 8 < 2 ? row[0] : row[1]) : (kt % 8 < 6 ? row[2] : row[3]);
            const int left = col < p.K ? g.hi - g.lo - c0 - r0 : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const uint32_t at = __shfl_sync(0xffffffffu, two, 16 * (kt & 1) + 2 * i + (r0 & 1));
              cp_async16(dst + 128 * kRowStep * i, x_col + static_cast<uint64_t>(at) * row_bytes,
                         kRowStep * i < left);
            }
          }
          cp_async_arrive(&sm.landed[s]);   // once this thread's copies have landed
          if (++s == kStages) {
            s = 0;
            ++use;
          }
        }
      }
      cp_async_wait_all();
    } else if (kBackW && warp >= kSumWarp) {
      const int l = tid - 32 * kSumWarp;
      bool ok = true;   // no early exit: the four warps meet at every tile with a bias sum
      // ------------------------------------------------------------- bias sums
      // A lane has four features (8 bytes of a 256-byte row of the stage), a warp 16 of
      // the 64 slots.  A stage whose products are done is summed, in the first column
      // block of each expert and 256 features, and handed back to the copies.  The sums of
      // 64 stages (4096 slots) are added up apart: one chain of all slots loses what is
      // below a unit of the sum so far, each time.
      int s = 0, use = 0;
      for (; sums && walk.more(); walk.next(sm)) {
        pair_tile<kWhat>(p, sm, walk.t, g);
        const int steps = pair_steps<kWhat>(p, g);
        float part[4] = {}, block[4] = {};
#pragma unroll 1
        for (int kt = 0; kt < steps; ++kt) {
          if (!(ok = ok && warp_wait(&sm.done[s], use & 1, abort_flag))) break;
          float now[4] = {};
          if (g.i0 == 0) {
            const uint8_t* at = base + s * kPairStageBytes + (lane >> 4) * kPairBoxBytes + 8 * (lane & 1);
#pragma unroll 8
            for (int i = 0; i < 16; ++i) {
              const uint2 v =
                  *reinterpret_cast<const uint2*>(at + sw128_offset(16 * (l >> 5) + i, (lane & 15) >> 1));
              now[0] += bf_lo(v.x);
              now[1] += bf_hi(v.x);
              now[2] += bf_lo(v.y);
              now[3] += bf_hi(v.y);
            }
          }
          warp_arrive(&sm.empty[s]);
          const bool full = kt % 64 == 63 || kt == steps - 1;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            block[i] += now[i];
            if (full) {
              part[i] += block[i];
              block[i] = 0.f;
            }
          }
          if (++s == kStages) {
            s = 0;
            ++use;
          }
        }
        if (g.i0 != 0) continue;
        const int w = l >> 5;
        float4& mine = *reinterpret_cast<float4*>(&sm.sums[w & 1][4 * lane]);
        if (w >= 2) mine = make_float4(part[0], part[1], part[2], part[3]);
        asm volatile("bar.sync 3, 128;" ::: "memory");
        if (w < 2) mine = make_float4(part[0] + mine.x, part[1] + mine.y, part[2] + mine.z, part[3] + mine.w);
        asm volatile("bar.sync 3, 128;" ::: "memory");
        const int n = g.f0 + rank * kPairM + l;
        if (ok && n < p.N) p.dbias[static_cast<size_t>(g.e) * p.N + n] = sm.sums[0][l] + sm.sums[1][l];
        asm volatile("bar.sync 3, 128;" ::: "memory");
      }
    } else if (kBackW && warp == 3) {
      if (sm.deal) deal_tiles(p, sm, pair, pairs, tiles);
    }
  }

  tc_fence_before();
  __syncthreads();
  if (tid == 0 && sm.abort) {   // of either CTA, for both
    st_cluster_u32(dsmem_addr(smem_u32(&sm.gave_up), 0), 1u);
    st_cluster_u32(dsmem_addr(smem_u32(&sm.gave_up), 1), 1u);
  }
  cluster_sync();   // no role of the pair starts a copy or a product any more
  if (warp == 1) drain_wait_pair(&sm.fin, 0);
  __syncwarp();
  if (sm.gave_up) {
    if (rank == 0 && tid == 0) drain_copies<kStages, kGather>(sm);
    __syncwarp();
    cluster_sync();
  }
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc_pair(tm, 512);
  }
  if (tid == 0 && sm.abort) atomicOr(p.status, kExpertTimeout);
}

// Forward with few slots (single tokens being served): the weights' rows are all there is
// to read and the pair kernel's set-up and pipeline latency most of its time.  One warp
// per two features of a slot reads them once, 16 bytes a lane; slots of the same expert
// read them again, from the L2.
constexpr int kFewSlots = 16;
constexpr int kFewThreads = 256;
constexpr int kFewFeatures = 2;

__global__ void __launch_bounds__(kFewThreads) sc_expert_few_kernel(
    const __grid_constant__ ExpertLinearParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, s = blockIdx.y;
  const int n = (blockIdx.x * (kFewThreads / 32) + warp) * kFewFeatures;
  pdl_wait();
  pdl_launch_dependents();
  if (n >= p.N) return;
  int e = -1;
  for (int e0 = 0; e0 < p.E && e < 0; e0 += 32) {
    int lo = 0, hi = 0;
    if (e0 + lane < p.E) expert_range(p, e0 + lane, lo, hi);
    const uint32_t has = __ballot_sync(0xffffffffu, s >= lo && s < hi);
    if (has != 0u) e = e0 + __ffs(has) - 1;
  }
  if (e < 0) return;   // a slot that is not in use
  const uint4* x = reinterpret_cast<const uint4*>(p.x + expert_row(p, s) * p.ldx);
  const uint4* w = reinterpret_cast<const uint4*>(p.w + (static_cast<size_t>(e) * p.N + n) * p.K);
  const int vecs = p.K / 8;
  float a[kFewFeatures] = {};
#pragma unroll 4
  for (int i = lane; i < vecs; i += 32) {
    const uint4 xv = __ldg(x + i);
    const uint32_t xs[4] = {xv.x, xv.y, xv.z, xv.w};
#pragma unroll
    for (int f = 0; f < kFewFeatures; ++f) {
      const uint4 wv = __ldg(w + f * vecs + i);
      const uint32_t ws[4] = {wv.x, wv.y, wv.z, wv.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        a[f] = fmaf(bf_lo(xs[q]), bf_lo(ws[q]), a[f]);
        a[f] = fmaf(bf_hi(xs[q]), bf_hi(ws[q]), a[f]);
      }
    }
  }
#pragma unroll
  for (int f = 0; f < kFewFeatures; ++f)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) a[f] += __shfl_xor_sync(0xffffffffu, a[f], off);
  if (lane != 0) return;
  if (p.bias != nullptr)
#pragma unroll
    for (int f = 0; f < kFewFeatures; ++f) a[f] += __ldg(p.bias + static_cast<size_t>(e) * p.N + n + f);
  const size_t at = static_cast<size_t>(s) * p.N + n;
  if (p.pre != nullptr) *reinterpret_cast<uint32_t*>(p.pre + at) = pack_bf16x2(a[0], a[1]);
  if (p.gelu) gelu2<false>(a[0], a[1]);
  if (p.out_f32) *reinterpret_cast<float2*>(static_cast<float*>(p.out) + at) = make_float2(a[0], a[1]);
  else *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at) = pack_bf16x2(a[0], a[1]);
}

// Forward and back (input) with few slots an expert: the weights' bytes bound it, and the
// pair kernel leaves SMs idle (96 tiles for 76 pairs: 400 slots of 16 experts, 768 -> 1536)
// and takes 8 us for its set-up and one tile alone.  Here a CTA of four warps has 64
// features x up to 32 slots of an expert, four CTAs share an SM, and the hardware deals
// them out; products by warp-level MMA (the tensor rate does not matter), operands through
// four stages of 64 of the contraction by 16-byte copies (six stages, three CTAs an SM:
// 14.3 us; three and five: 13.1; four and four: 11.4; the pair kernel 15.2).
constexpr int kSmallThreads = 128;
constexpr int kSmallF = 64, kSmallS = 32, kSmallStages = 4;
constexpr uint32_t kSmallABytes = kSmallF * 128, kSmallStage = kSmallABytes + kSmallS * 128;
constexpr uint32_t kSmallDyn = kSmallStages * kSmallStage + 1024;

template <ExpertProduct kWhat>
__global__ void __launch_bounds__(kSmallThreads, 4)
    sc_expert_small_kernel(const __grid_constant__ ExpertLinearParams p) {
  constexpr bool kFwd = kWhat == ExpertProduct::kForward;
  extern __shared__ uint8_t dyn_raw[];
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(dyn_raw) + 1023) &
                                             ~static_cast<uintptr_t>(1023));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int f0 = blockIdx.x * kSmallF;
  const int width = kFwd ? p.N : p.K, depth = kFwd ? p.K : p.N;
  pdl_wait();
  pdl_launch_dependents();
  // the expert and slots of tile blockIdx.y
  int e = -1, lo = 0, hi = 0, before = 0;
  for (int e0 = 0; e0 < p.E; e0 += 32) {
    int a = 0, b = 0;
    if (e0 + lane < p.E) expert_range(p, e0 + lane, a, b);
    const int mine = (b - a + kSmallS - 1) / kSmallS;
    int x = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {   // inclusive scan
      const int y = __shfl_up_sync(0xffffffffu, x, off);
      if (lane >= off) x += y;
    }
    const int t = static_cast<int>(blockIdx.y) - before;
    const uint32_t has = __ballot_sync(0xffffffffu, t >= x - mine && t < x);
    if (has != 0u) {
      const int l = __ffs(has) - 1;
      e = e0 + l;
      lo = __shfl_sync(0xffffffffu, a + (t - x + mine) * kSmallS, l);
      hi = __shfl_sync(0xffffffffu, b, l);
      break;
    }
    before += __shfl_sync(0xffffffffu, x, 31);
  }
  if (e < 0) return;
  const int n = min(kSmallS, hi - lo);

  // copies: piece c (16 bytes) of rows r0 + 16 i; weights: 64 rows of features (forward)
  // or of the contraction, the other side: 32 slots, the last one again past the end
  const int c = tid & 7, r0 = tid >> 3;
  const uint16_t* const w = p.w + static_cast<size_t>(e) * p.N * p.K;
  const uint16_t* rows[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lo + min(r0 + 16 * i, n - 1);
    rows[i] = kFwd ? p.x + expert_row(p, s) * p.ldx : p.dy + s * p.ldy;
  }
  const int steps = (depth + 63) / 64;
  const auto copy = [&](int kt) {
    const uint32_t at = smem_u32(base) + (kt % kSmallStages) * kSmallStage;
    const int k = 64 * kt + 8 * c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + 16 * i;
      const int row = kFwd ? f0 + r : 64 * kt + r, col = kFwd ? k : f0 + 8 * c;
      const bool in = row < p.N && col < p.K;
      cp_async16(at + sw128_offset(r, c), w + (in ? static_cast<size_t>(row) * p.K + col : 0), in);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      cp_async16(at + kSmallABytes + sw128_offset(r0 + 16 * i, c), rows[i] + (k < depth ? k : 0), k < depth);
  };
#pragma unroll
  for (int i = 0; i < kSmallStages - 1; ++i) {
    if (i < steps) copy(i);
    cp_async_commit();
  }
  // slots 8 j ..; sum: see kSpan, for fp32 outputs stage by stage (2048 deep: 1.3e-7, as torch's
  // fp32 product, where eight stages had 4.7e-7; 12.0 us for 400 slots of 16 experts, 11.9 before)
  float acc[4][4] = {}, sum[4][4] = {};
  const int f = 16 * warp;                // this warp's features of the tile
#pragma unroll 1
  for (int kt = 0; kt < steps; ++kt) {
    cp_async_wait<kSmallStages - 2>();
    __syncthreads();   // the stage is there, and the one before it has been read by all
    if (kt + kSmallStages - 1 < steps) copy(kt + kSmallStages - 1);
    cp_async_commit();
    const uint32_t a = smem_u32(base) + (kt % kSmallStages) * kSmallStage, b = a + kSmallABytes;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t av[4], bv[2][4];
      if constexpr (kFwd)
        ldmatrix4(a + sw128_offset(f + (lane & 15), 2 * k + (lane >> 4)), av);
      else
        ldmatrix4_trans(a + sw128_offset(16 * k + (lane & 7) + 8 * (lane >> 4), f / 8 + ((lane >> 3) & 1)), av);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        ldmatrix4(b + sw128_offset(16 * j + (lane & 7) + 8 * (lane >> 4), 2 * k + ((lane >> 3) & 1)), bv[j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) mma_bf16(acc[j], av, bv[j >> 1][2 * (j & 1)], bv[j >> 1][2 * (j & 1) + 1]);
    }
    if (p.out_f32 || kt % kSpan == kSpan - 1 || kt == steps - 1) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          sum[j][i] += acc[j][i];
          acc[j][i] = 0.f;
        }
    }
  }
  // the lane has features fr, fr + 8 of slots 8 j + 2 (lane % 4), + 1
  const int fr = f0 + f + (lane >> 2);
  cp_async_wait_all();
  __syncthreads();
  // staging: 32 slots x 64 features in bf16, 128-byte rows; of `pre` and of the output
  uint8_t* const stg_pre = base;
  uint8_t* const stg = base + kSmallS * 128;
  const auto at = [&](int j) {   // this lane's row of fragments of slots 8 j .. 8 j + 15
    return sw128_offset(8 * j + (lane & 7) + 8 * (lane >> 4), f / 8 + ((lane >> 3) & 1));
  };
  const auto store = [&](uint8_t* to) {
#pragma unroll
    for (int j = 0; j < 4; j += 2)
      stmatrix4_trans(smem_u32(to) + at(j), pack_bf16x2(sum[j][0], sum[j][1]), pack_bf16x2(sum[j][2], sum[j][3]),
                      pack_bf16x2(sum[j + 1][0], sum[j + 1][1]), pack_bf16x2(sum[j + 1][2], sum[j + 1][3]));
  };
  const auto flush = [&](const uint8_t* from, uint16_t* out) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = r0 + 16 * i;
      if (r < n && f0 + 8 * c < width)
        *reinterpret_cast<uint4*>(out + static_cast<size_t>(lo + r) * width + f0 + 8 * c) =
            *reinterpret_cast<const uint4*>(from + sw128_offset(r, c));
    }
  };
  if constexpr (kFwd) {
    if (p.bias != nullptr)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float bias = fr + 8 * h < p.N ? __ldg(p.bias + static_cast<size_t>(e) * p.N + fr + 8 * h) : 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sum[j][2 * h] += bias;
          sum[j][2 * h + 1] += bias;
        }
      }
    if (p.pre != nullptr) store(stg_pre);
    if (p.gelu)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        gelu2<false>(sum[j][0], sum[j][1]);
        gelu2<false>(sum[j][2], sum[j][3]);
      }
  } else if (p.pre_in != nullptr) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = r0 + 16 * i;
      const bool in = r < n && f0 + 8 * c < width;
      cp_async16(smem_u32(stg_pre) + sw128_offset(r, c),
                 p.pre_in + (in ? static_cast<size_t>(lo + r) * width + f0 + 8 * c : 0), in);
    }
    cp_async_wait_all();
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      uint32_t z[4];
      ldmatrix4_trans(smem_u32(stg_pre) + at(j), z);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        gelu_slope2<false>(bf_lo(z[i]), bf_hi(z[i]), sum[j + (i >> 1)][2 * (i & 1)], sum[j + (i >> 1)][2 * (i & 1) + 1]);
    }
  }
  if (p.out_f32) {
    // eight lanes write 32 consecutive bytes of a slot
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int s = 8 * j + 2 * (lane & 3) + (i & 1), x = fr + 8 * (i >> 1);
        if (s < n && x < width)
          static_cast<float*>(p.out)[static_cast<size_t>(lo + s) * width + x] = sum[j][i];
      }
  } else {
    store(stg);
  }
  __syncthreads();
  if (!p.out_f32) flush(stg, static_cast<uint16_t*>(p.out));
  if (kFwd && p.pre != nullptr) flush(stg_pre, p.pre);
}

// It runs for up to this many slots an expert on average, and while the pair kernel's tiles
// would be at most two rounds: us here and there, the weights read anew,
//   768 -> 1536,   8 experts,  16, 32, 64, 128 slots each: 8.3 10.5 11.3 15.8; 10.3 10.5 11.5 13.6
//   768 -> 1536,  16 experts,  25, 64 slots each: 11.4 17.0; 15.2 17.1
//   1024 -> 2048, 64 experts,  8, 32, 64 slots each (seven rounds): 46 62 88; 47 51 53
constexpr int kSmallRows = 48;

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------
// bf16 rows of `cols` elements, `ld` apart, as a tensor map of 64-column boxes with the
// 128-byte swizzle; with experts > 0, that many matrices of `rows` rows each (3-D).
static bool encode_rows(CUtensorMap* m, const void* base, long long rows, int cols, long long ld,
                        int experts, int box_rows) {
  const auto enc = api_tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dim[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                             static_cast<cuuint64_t>(experts > 0 ? experts : 1)};
  const cuuint64_t stride[2] = {static_cast<cuuint64_t>(ld) * 2,
                                static_cast<cuuint64_t>(ld) * 2 * static_cast<cuuint64_t>(rows)};
  const cuuint32_t box[3] = {64u, static_cast<cuuint32_t>(box_rows), 1u}, one[3] = {1u, 1u, 1u};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, experts > 0 ? 3 : 2, const_cast<void*>(base), dim,
             stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// An output of rows x cols (x experts), in boxes of 32 x 32.
static bool encode_out(CUtensorMap* m, void* base, bool f32, long long rows, int cols, int experts) {
  const auto enc = api_tensor_map_encoder();
  if (!enc) return false;
  const cuuint64_t dim[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows),
                             static_cast<cuuint64_t>(experts > 0 ? experts : 1)};
  const cuuint64_t row = static_cast<cuuint64_t>(cols) * (f32 ? 4 : 2);
  const cuuint64_t stride[2] = {row, row * static_cast<cuuint64_t>(rows)};
  const cuuint32_t box[3] = {32u, 32u, 1u}, one[3] = {1u, 1u, 1u};
  return enc(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
             experts > 0 ? 3 : 2, base, dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
             f32 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
             CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <ExpertProduct kWhat, bool kGather, bool kF32, bool kPre>
static cudaError_t launch_pair(const PairParams& P, long long most_tiles, cudaStream_t st) {
  using Kind = PairKind<kWhat, kGather, kF32, kPre>;
  const int sms = api_device_sms();
  if (sms < 2) return cudaErrorInvalidDevice;
  const long long pairs = most_tiles < sms / 2 ? most_tiles : sms / 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(2 * pairs));
  cfg.blockDim = dim3(Kind::kThreads);
  cfg.dynamicSmemBytes = Kind::kDyn;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, sc_expert_pair_kernel<kWhat, kGather, kF32, kPre>, P);
}

template <ExpertProduct kWhat, bool kGather>
static cudaError_t launch_pair(const PairParams& P, long long most_tiles, cudaStream_t st) {
  // (the fp32 kernels have the room anyway)
  if (P.p.out_f32 || (kWhat == ExpertProduct::kBackWeight && P.p.M > kLongSlots))
    return launch_pair<kWhat, kGather, true, true>(P, most_tiles, st);
  if constexpr (kWhat != ExpertProduct::kBackWeight) {
    if (P.p.pre != nullptr || P.p.pre_in != nullptr)
      return launch_pair<kWhat, kGather, false, true>(P, most_tiles, st);
  }
  return launch_pair<kWhat, kGather, false, false>(P, most_tiles, st);
}

cudaError_t launch_expert_linear(ExpertProduct what, const ExpertLinearParams& p, cudaStream_t st) {
  if (what == ExpertProduct::kForward && p.M <= kFewSlots) {
    constexpr int per = kFewThreads / 32 * kFewFeatures;
    return launch_chained(sc_expert_few_kernel, dim3((p.N + per - 1) / per, p.M), dim3(kFewThreads), 0, st, p);
  }
  const int width = what == ExpertProduct::kBackInput ? p.K : p.N;
  if (what != ExpertProduct::kBackWeight && p.M <= static_cast<long long>(kSmallRows) * p.E &&
      (p.E < p.M ? p.E : p.M) * ((width + 255) / 256) <= api_device_sms() / 2 * 2) {
    const dim3 grid((width + kSmallF - 1) / kSmallF, p.M / kSmallS + (p.E < p.M ? p.E : p.M));
    return launch_chained(what == ExpertProduct::kForward ? sc_expert_small_kernel<ExpertProduct::kForward>
                                                          : sc_expert_small_kernel<ExpertProduct::kBackInput>,
                          grid, dim3(kSmallThreads), kSmallDyn, st, p);
  }
  PairParams P;
  P.p = p;
  const bool gather = p.token != nullptr;
  // no more tiles of slots than full ones and two begun for each expert
  const long long slot_tiles = p.M / kPairN + 2ll * (p.E < p.M ? p.E : p.M);
  bool ok;
  if (what == ExpertProduct::kForward) {
    ok = encode_rows(&P.map_a, p.w, p.N, p.K, p.K, p.E, kPairM) &&
         (gather || (encode_rows(&P.map_b, p.x, p.M, p.K, p.ldx, 0, kPairN / 2) &&
                     encode_rows(&P.map_b32, p.x, p.M, p.K, p.ldx, 0, 32))) &&
         encode_out(&P.map_out, p.out, p.out_f32, p.M, p.N, 0) &&
         (p.pre == nullptr || encode_out(&P.map_pre, p.pre, false, p.M, p.N, 0));
    if (!ok) return cudaErrorInvalidValue;
    const long long tiles = slot_tiles * ((p.N + 255) / 256);
    return gather ? launch_pair<ExpertProduct::kForward, true>(P, tiles, st)
                  : launch_pair<ExpertProduct::kForward, false>(P, tiles, st);
  }
  if (what == ExpertProduct::kBackInput) {
    ok = encode_rows(&P.map_a, p.w, p.N, p.K, p.K, p.E, kPairStep) &&
         encode_rows(&P.map_b, p.dy, p.M, p.N, p.ldy, 0, kPairN / 2) &&
         encode_rows(&P.map_b32, p.dy, p.M, p.N, p.ldy, 0, 32) &&
         encode_out(&P.map_out, p.out, p.out_f32, p.M, p.K, 0);
    if (!ok) return cudaErrorInvalidValue;
    return launch_pair<ExpertProduct::kBackInput, false>(P, slot_tiles * ((p.K + 255) / 256), st);
  }
  ok = encode_rows(&P.map_a, p.dy, p.M, p.N, p.ldy, 0, kPairStep) &&
       (gather || encode_rows(&P.map_b, p.x, p.M, p.K, p.ldx, 0, kPairStep)) &&
       encode_out(&P.map_out, p.out, p.out_f32, p.N, p.K, p.E);
  if (!ok) return cudaErrorInvalidValue;
  const long long tiles = static_cast<long long>(p.E) * ((p.N + 255) / 256) * ((p.K + kPairN - 1) / kPairN);
  return gather ? launch_pair<ExpertProduct::kBackWeight, true>(P, tiles, st)
                : launch_pair<ExpertProduct::kBackWeight, false>(P, tiles, st);
}

// The register shares of the fp32 kernels sum up to what they are launched with: a
// warpgroup that asks for more would wait for ever.
template <ExpertProduct kWhat, bool kGather>
static cudaError_t check_registers() {
  using Kind = PairKind<kWhat, kGather, true, true>;
  if (!Kind::kSplit) return cudaSuccess;
  cudaFuncAttributes a;
  const cudaError_t e = cudaFuncGetAttributes(&a, sc_expert_pair_kernel<kWhat, kGather, true, true>);
  if (e != cudaSuccess) return e;
  const int others = Kind::kThreads - 128 - 32 * Kind::kEpiWarps;
  const int want = 32 * Kind::kEpiWarps * Kind::kEpiRegs + 128 * Kind::kFirstRegs + others * Kind::kAuxRegs;
  return want <= a.numRegs * Kind::kThreads ? cudaSuccess : cudaErrorInvalidConfiguration;
}

template <ExpertProduct kWhat, bool kGather, bool kF32, bool kPre>
static cudaError_t configure_room() {
  return cudaFuncSetAttribute(sc_expert_pair_kernel<kWhat, kGather, kF32, kPre>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(PairKind<kWhat, kGather, kF32, kPre>::kDyn));
}

template <ExpertProduct kWhat, bool kGather>
static cudaError_t configure_pair() {
  cudaError_t e = check_registers<kWhat, kGather>();
  if (e == cudaSuccess) e = configure_room<kWhat, kGather, true, true>();
  if (e == cudaSuccess) e = configure_room<kWhat, kGather, false, false>();
  if constexpr (kWhat != ExpertProduct::kBackWeight)
    if (e == cudaSuccess) e = configure_room<kWhat, kGather, false, true>();
  return e;
}

cudaError_t configure_expert() {
  cudaError_t e = configure_combine();
  if (e == cudaSuccess) e = configure_pair<ExpertProduct::kForward, false>();
  if (e == cudaSuccess) e = configure_pair<ExpertProduct::kForward, true>();
  if (e == cudaSuccess) e = configure_pair<ExpertProduct::kBackInput, false>();
  if (e == cudaSuccess) e = configure_pair<ExpertProduct::kBackWeight, false>();
  if (e == cudaSuccess) e = configure_pair<ExpertProduct::kBackWeight, true>();
  const auto attr = cudaFuncAttributeMaxDynamicSharedMemorySize;
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(sc_expert_small_kernel<ExpertProduct::kForward>, attr, static_cast<int>(kSmallDyn));
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(sc_expert_small_kernel<ExpertProduct::kBackInput>, attr, static_cast<int>(kSmallDyn));
  return e;
}

}  // namespace sc
