// sc_expert_combine.cu -- the end of an expert feed-forward block: the experts'
// rows summed under their gates, the scaled residual, and a layer norm, in one pass.
//
//   S[t] = a res[t] + sum_j g[t][j] Y[slot[t][j]],   out[t] = LN(S[t])
// Backward, from dOut and dSum (either may be absent), with S, its mean and
// 1 / sigma computed again from the inputs and h = (S - mean) / sigma:
//   dh = dOut gamma;  dS = (dh - mean(dh) - h mean(dh h)) / sigma + dSum
//   dY[slot] = g dS;  dg = dS . Y[slot];  dres = a dS
//   dgamma = sum_t dOut h;  dbeta = sum_t dOut   (rows in a fixed order)
// All sums in fp32; the norm takes the unrounded S; outputs are rounded once.
//
// Bound by memory.  Each thread copies the 16-byte vectors that it will use itself, a
// row ahead, into shared memory of its own (cp.async), so that a whole row more than the
// one at work is on its way per warp, whatever the registers hold, and no thread waits for
// another's copies.  A warp has a row of up to 1024 features; wider rows have several
// warps, whose sums meet in shared memory.  Rows in registers, loaded when they were
// needed, kept too little on its way: 8192 rows x 1024, k = 4, gradient 155 us with a
// warp a row, 106 us with a thread per eight features; now 37 us and 6 for the sums of
// dgamma and dbeta (201 MB, 5.4 TB/s).
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_expert.cuh"
#include "sm103_primitives.cuh"

namespace sc {

constexpr int kCombineWarps = 8;       // most of a CTA
constexpr int kWarpFeatures = 1024;    // most of a warp
constexpr int kCombineChunk = 4;       // choices whose dot products are summed together
constexpr int kPlanRows = 4;           // rows whose slots and gates a warp loads at once
constexpr int kUnused = -2;
static_assert(kPlanRows * kMaxChoices == 32, "a lane a choice");
static_assert(kMaxChoices == 2 * kCombineChunk, "two loads of slots");

// Eight bf16 as four fp32 pairs, and back: the arithmetic runs on pairs (one instruction
// each), because a gradient's row has some fifty operations a pair.
__device__ __forceinline__ void unpack8(const uint4& v, uint64_t (&f)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = f2_pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}

__device__ __forceinline__ uint4 pack8(const uint64_t (&f)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    f2_unpack(f[i], lo, hi);
    w[i] = pack_bf16x2(lo, hi);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float f2_sum(uint64_t v) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return lo + hi;
}

template <int N>
struct Choices {
  static constexpr int value = N;
};

// How a launch is cut: warps of a row, rows of a CTA at a time, copied tensors of a row,
// rows on their way per row group (two, or one where two do not fit).
struct CombineCut {
  int warps, groups, segs, ctas;
  float inv_d;   // 1 / D (a division in the chain of a row costs as much as its sum)
};

struct CombineSmem {
  float red[2][kCombineChunk][kCombineWarps];   // the warps' sums, two in turn
  // per warp: slots and gates of two times four rows (kUnused: a row that is not in use)
  alignas(16) int slot[kCombineWarps][2 * kPlanRows][kMaxChoices];
  alignas(16) float gate[kCombineWarps][2 * kPlanRows][kMaxChoices];
};

// Sums of N values over a row's threads, the same in each of them; its warps in order.
template <bool kWide, int N>
__device__ __forceinline__ void row_sum(const CombineCut& cut, CombineSmem& sm, int group, int w, int& turn,
                                        float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], off);
  if (!kWide) return;
  turn ^= 1;   // the other half was read before the last meeting
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) sm.red[turn][i][group * cut.warps + w] = v[i];
  asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(32 * cut.warps) : "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float* const of = &sm.red[turn][i][group * cut.warps];
    v[i] = of[0];
    for (int o = 1; o < cut.warps; ++o) v[i] += of[o];
  }
}

// V vectors of 8 features a thread; kRows rows on their way per row group; kWide: several
// warps a row (where it is one, a thread's vectors lie at constant distances).
template <bool kBack, int V, int kRows, bool kWide>
__global__ void __launch_bounds__(32 * kCombineWarps, kBack ? 1 : 2)
    sc_combine_kernel(const __grid_constant__ CombineParams p, const CombineCut cut) {
  __shared__ CombineSmem sm;
  extern __shared__ uint4 fifo[];   // per warp [kRows][segs][V][32], then gamma (and beta)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int warps = kWide ? cut.warps : 1;
  const int group = warp / warps, w = warp - group * warps;
  const int vecs = p.D / 8;
  // gamma and beta, the first four and the last four features of each vector apart (one
  // load each from global memory was 32 bytes from the next lane's: 23 us of 8192 x 768)
  float4* const gam = reinterpret_cast<float4*>(
      fifo + static_cast<size_t>(cut.warps) * cut.groups * kRows * cut.segs * V * 32);
  float4* const bet = gam + 2 * vecs;
  uint4* const mine = fifo + static_cast<size_t>(warp) * kRows * cut.segs * V * 32 + lane;
  // this thread's vector v is number 32 (w + v warps) + lane of a row
  const int at0 = 32 * w + lane, at_step = 32 * warps;
  const bool norm = p.gamma != nullptr;
  const bool need_y = !kBack || norm || p.dgate != nullptr;
  const bool need_res = p.res != nullptr && (!kBack || norm);
  // segments after the choices'
  const int seg_res = p.k, seg_dout = seg_res + (need_res ? 1 : 0);
  const long long step = static_cast<long long>(gridDim.x) * cut.groups;
  pdl_wait();
  pdl_launch_dependents();
  const auto param = [&](const float4* v, int at, uint64_t (&f)[4]) {
    const float4 a = v[at], b = v[vecs + at];
    f[0] = f2_pack(a.x, a.y), f[1] = f2_pack(a.z, a.w), f[2] = f2_pack(b.x, b.y), f[3] = f2_pack(b.z, b.w);
  };

  // Slots and gates come for four rows of this group at once, a lane a choice (row by row
  // they were a quarter of the instructions), while the four rows before them are at work.
  const int plan_row = lane / kMaxChoices, plan_j = lane % kMaxChoices;
  int plan_slot = kUnused;
  float plan_gate = 0.f;
  const auto load_plan = [&](long long t0) {
    const long long t = t0 + plan_row * step;
    plan_slot = kUnused;
    plan_gate = 0.f;
    if (t >= p.T) return;
    // (all three loads before the first use; a row not in use has a slot entry too)
    int used = 1;
    if (p.rows != nullptr) {
      const unsigned b = static_cast<unsigned>(t) / static_cast<unsigned>(p.L);   // t < 2^31
      used = __ldg(p.rows + b) - static_cast<int>(static_cast<unsigned>(t) - b * p.L);
    }
    int slot = -1;
    float gate = 1.f;
    if (plan_j < p.k) {
      slot = __ldg(p.slot + t * p.k + plan_j);
      if (p.gate != nullptr) gate = __ldg(p.gate + t * p.k + plan_j);
    }
    if (used <= 0) return;
    const bool in = slot >= 0 && slot < p.M;
    plan_slot = in ? slot : -1;
    plan_gate = in ? gate : 0.f;
  };
  // All vectors of a thread but its last one lie within the row (the fewest that hold it).
  const bool last = at0 + (V - 1) * at_step < vecs;
  const auto inside = [&](int v) { return v < V - 1 || last; };
  const auto copy = [&](uint32_t to, const uint16_t* row, bool there) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      cp_async16(to + 512 * v, row + (inside(v) ? 8 * (at0 + v * at_step) : 0), there && inside(v));
  };
  // starts the copies of row i of this group, row t of all, into place r
  const auto start = [&](int i, long long t, int r) {
    const int half = i & kPlanRows, at = i % (2 * kPlanRows);
    if (i % kPlanRows == 0) {
      __syncwarp();   // the plans in this half have been read
      sm.slot[warp][half + plan_row][plan_j] = plan_slot;
      sm.gate[warp][half + plan_row][plan_j] = plan_gate;
      load_plan(t + kPlanRows * step);
      __syncwarp();
    }
    const int4* const slots = reinterpret_cast<const int4*>(sm.slot[warp][at]);
    const int4 s0 = slots[0];
    if (s0.x != kUnused) {
      const uint32_t seg = 512 * V;
      uint32_t to = smem_u32(mine) + r * cut.segs * seg;
      if (need_y) {
        const auto choice = [&](int s) {   // zeros where there is none
          copy(to, p.y + static_cast<size_t>(max(s, 0)) * p.D, s >= 0);
          to += seg;
        };
        choice(s0.x);
        if (p.k > 1) choice(s0.y);
        if (p.k > 2) choice(s0.z);
        if (p.k > 3) choice(s0.w);
        if (p.k > 4) {
          const int4 s1 = slots[1];
          choice(s1.x);
          if (p.k > 5) choice(s1.y);
          if (p.k > 6) choice(s1.z);
          if (p.k > 7) choice(s1.w);
        }
      } else {
        to += p.k * seg;
      }
      const auto row = [&](const uint16_t* of) {
        copy(to, of + t * p.D, true);
        to += seg;
      };
      if (need_res) row(p.res);
      if (kBack && norm) row(p.dout);
    }
    cp_async_commit();
  };
  const auto piece = [&](int r, int seg, int v, uint64_t (&f)[4]) {
    unpack8(mine[(r * cut.segs + seg) * V * 32 + 32 * v], f);
  };

  uint64_t dgam[kBack ? V : 1][4], dbet[kBack ? V : 1][4];
#pragma unroll
  for (int v = 0; v < (kBack ? V : 1); ++v)
#pragma unroll
    for (int q = 0; q < 4; ++q) dgam[v][q] = dbet[v][q] = f2_both(0.f);
  int turn = 0;
  long long t = static_cast<long long>(blockIdx.x) * cut.groups + group;
  load_plan(t);
  start(0, t, 0);
  if (norm) {
    for (int i = threadIdx.x; i < p.D; i += blockDim.x) {
      const int to = ((i >> 2 & 1) * vecs + (i >> 3)) * 4 + (i & 3);
      reinterpret_cast<float*>(gam)[to] = __ldg(p.gamma + i);
      if (!kBack) reinterpret_cast<float*>(bet)[to] = __ldg(p.beta + i);
    }
    __syncthreads();
  }
  for (int i = 0, r = 0; t < p.T; t += step, ++i, r = kRows == 2 ? r ^ 1 : 0) {
    const int* const slot_of = sm.slot[warp][i % (2 * kPlanRows)];
    const float* const gate_of = sm.gate[warp][i % (2 * kPlanRows)];
    if (kRows == 2) {
      start(i + 1, t + step, r ^ 1);
      cp_async_wait<1>();
    } else {
      cp_async_wait<0>();
    }
    if (slot_of[0] != kUnused) {
      // dSum is needed last: loads of now (a copy a row ahead took the room of a seventh of
      // the rows at work)
      uint4 dsum[kBack ? V : 1];
      if constexpr (kBack)
#pragma unroll
        for (int v = 0; v < V; ++v)
          dsum[v] = p.dsum != nullptr && inside(v)
                        ? __ldg(reinterpret_cast<const uint4*>(p.dsum + t * p.D) + at0 + v * at_step)
                        : make_uint4(0u, 0u, 0u, 0u);
      // S, and its normal form
      uint64_t s[V][4];
      float inv = 0.f;
      if (!kBack || norm) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
          for (int q = 0; q < 4; ++q) s[v][q] = f2_both(0.f);
          if (need_res) {
            piece(r, seg_res, v, s[v]);
#pragma unroll
            for (int q = 0; q < 4; ++q) s[v][q] = f2_mul(s[v][q], f2_both(p.res_scale));
          }
        }
#pragma unroll 2
        for (int j = 0; j < p.k; ++j) {
          const uint64_t g = f2_both(gate_of[j]);
#pragma unroll
          for (int v = 0; v < V; ++v) {
            uint64_t f[4];
            piece(r, j, v, f);
#pragma unroll
            for (int q = 0; q < 4; ++q) s[v][q] = f2_fma(g, f[q], s[v][q]);
          }
        }
        if (!kBack && p.sum != nullptr)
#pragma unroll
          for (int v = 0; v < V; ++v)
            if (inside(v))
              reinterpret_cast<uint4*>(p.sum + t * p.D)[at0 + v * at_step] = pack8(s[v]);
      }
      if (norm) {
        // two sums, so that a mean far from 0 costs no digits of the variance
        uint64_t a2 = f2_both(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int q = 0; q < 4; ++q) a2 = f2_add(a2, s[v][q]);
        float a[1] = {f2_sum(a2)};
        row_sum<kWide>(cut, sm, group, w, turn, a);
        const float mean = a[0] * cut.inv_d;
        a2 = f2_both(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
          // (features past D are and stay 0)
          const uint64_t shift = f2_both(inside(v) ? -mean : 0.f);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            s[v][q] = f2_add(s[v][q], shift);
            a2 = f2_fma(s[v][q], s[v][q], a2);
          }
        }
        a[0] = f2_sum(a2);
        row_sum<kWide>(cut, sm, group, w, turn, a);
        inv = rsqrtf(fmaf(a[0], cut.inv_d, p.eps));
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
          for (int q = 0; q < 4; ++q) s[v][q] = f2_mul(s[v][q], f2_both(inv));
      }
      if constexpr (!kBack) {
        if (norm)
#pragma unroll
          for (int v = 0; v < V; ++v) {
            const int at = at0 + v * at_step;
            if (!inside(v)) continue;
            uint64_t ga[4], be[4];
            param(gam, at, ga);
            param(bet, at, be);
#pragma unroll
            for (int q = 0; q < 4; ++q) s[v][q] = f2_fma(s[v][q], ga[q], be[q]);
            reinterpret_cast<uint4*>(p.out + t * p.D)[at] = pack8(s[v]);
          }
      } else {
        uint64_t ds[V][4], ab0 = f2_both(0.f), ab1 = f2_both(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v) {
#pragma unroll
          for (int q = 0; q < 4; ++q) ds[v][q] = f2_both(0.f);
          const int at = at0 + v * at_step;
          if (!norm || !inside(v)) continue;
          uint64_t f[4], ga[4];
          piece(r, seg_dout, v, f);
          param(gam, at, ga);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            dgam[v][q] = f2_fma(f[q], s[v][q], dgam[v][q]);
            dbet[v][q] = f2_add(dbet[v][q], f[q]);
            ds[v][q] = f2_mul(f[q], ga[q]);
            ab0 = f2_add(ab0, ds[v][q]);
            ab1 = f2_fma(ds[v][q], s[v][q], ab1);
          }
        }
        if (norm) {
          float ab[2] = {f2_sum(ab0), f2_sum(ab1)};
          row_sum<kWide>(cut, sm, group, w, turn, ab);
          // (dh - ma - h mb) / sigma
          const float by = -cut.inv_d * inv;
          const uint64_t i2 = f2_both(inv), ma = f2_both(ab[0] * by), mb = f2_both(ab[1] * by);
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int q = 0; q < 4; ++q) ds[v][q] = f2_fma(s[v][q], mb, f2_fma(ds[v][q], i2, ma));
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int at = at0 + v * at_step;
          uint64_t f[4];
          unpack8(dsum[v], f);
#pragma unroll
          for (int q = 0; q < 4; ++q) ds[v][q] = f2_add(ds[v][q], f[q]);
          if (p.dres != nullptr && inside(v)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) f[q] = f2_mul(ds[v][q], f2_both(p.res_scale));
            reinterpret_cast<uint4*>(p.dres + t * p.D)[at] = pack8(f);
          }
        }
        // N choices together (past the last one again that one, unwritten): dY and dot products
        const auto choices = [&](int j0, auto n) {
          constexpr int N = decltype(n)::value;
          float dot[N];
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int j = min(j0 + i, p.k - 1);
            const int sl = j0 + i < p.k ? slot_of[j] : -1;
            const uint64_t g = f2_both(gate_of[j]);
            uint4* const dy = reinterpret_cast<uint4*>(p.dy + static_cast<size_t>(max(sl, 0)) * p.D);
            uint64_t dot2 = f2_both(0.f);
#pragma unroll
            for (int v = 0; v < V; ++v) {
              const int at = at0 + v * at_step;
              uint64_t f[4];
              if (p.dgate != nullptr) {
                piece(r, j, v, f);
#pragma unroll
                for (int q = 0; q < 4; ++q) dot2 = f2_fma(ds[v][q], f[q], dot2);
              }
#pragma unroll
              for (int q = 0; q < 4; ++q) f[q] = f2_mul(g, ds[v][q]);
              if (sl >= 0 && inside(v)) dy[at] = pack8(f);
            }
            dot[i] = f2_sum(dot2);
          }
          if (p.dgate != nullptr) {
            row_sum<kWide>(cut, sm, group, w, turn, dot);
#pragma unroll
            for (int i = 0; i < N; ++i)
              if (w == 0 && lane == 0 && j0 + i < p.k)
                p.dgate[t * p.k + j0 + i] = slot_of[j0 + i] >= 0 ? dot[i] : 0.f;
          }
        };
        if (p.k <= 2) {
          choices(0, Choices<2>());
        } else {
          for (int j0 = 0; j0 < p.k; j0 += kCombineChunk) choices(j0, Choices<kCombineChunk>());
        }
      }
    } else if (kBack && p.dgate != nullptr && w == 0 && lane < p.k) {
      p.dgate[t * p.k + lane] = 0.f;
    }
    if (kRows == 1) start(i + 1, t + step, 0);
  }
  if constexpr (kBack) {
    cp_async_wait_all();
    if (p.dgamma == nullptr) return;
    // the CTA's row groups in order, through the copies' place
    float* const part = reinterpret_cast<float*>(fifo);
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int at = at0 + v * at_step;
      if (!inside(v)) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        *reinterpret_cast<uint64_t*>(part + (2 * group) * p.D + 8 * at + 2 * q) = dgam[v][q];
        *reinterpret_cast<uint64_t*>(part + (2 * group + 1) * p.D + 8 * at + 2 * q) = dbet[v][q];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.D; i += blockDim.x) {
      float x = part[i];
      for (int o = 1; o < cut.groups; ++o) x += part[o * 2 * p.D + i];
      p.part[static_cast<long long>(blockIdx.x) * 2 * p.D + i] = x;
    }
  } else {
    cp_async_wait_all();
  }
}

// dgamma and dbeta: the CTAs' parts, 32 features a CTA, its 32 warps every 32nd part in
// order, then the warps in order.
__global__ void __launch_bounds__(1024) sc_combine_reduce_kernel(const __grid_constant__ CombineParams p,
                                                                 int parts) {
  __shared__ float red[32][33];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int f = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (f < 2 * p.D)
#pragma unroll 8
    for (int c = w; c < parts; c += 32) v += __ldcg(p.part + static_cast<long long>(c) * 2 * p.D + f);
  red[w][lane] = v;
  __syncthreads();
  if (w != 0 || f >= 2 * p.D) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) v += red[i][lane];
  if (f < p.D) p.dgamma[f] = v;
  else p.dbeta[f - p.D] = v;
}

// ---------------------------------------------------------------------------
// launch
// ---------------------------------------------------------------------------
constexpr size_t kCombineBytes = 216 * 1024;   // shared memory for copies per SM
static_assert(kCombineBytes + sizeof(CombineSmem) <= 227 * 1024, "one CTA's shared memory");

template <bool kBack, int V, int kRows, bool kWide>
static cudaError_t launch_cut(const CombineParams& p, const CombineCut& cut, size_t smem, cudaStream_t st) {
  return launch_chained(sc_combine_kernel<kBack, V, kRows, kWide>, dim3(cut.ctas),
                        dim3(32 * cut.warps * cut.groups), smem, st, p, cut);
}

// A row of one warp always has room for two (20 KB at most); one of several warps has three
// or four vectors a thread, three up to 2304 features, where there is room for two rows too.
template <bool kBack>
static cudaError_t launch_vecs(const CombineParams& p, const CombineCut& cut, int vecs, int rows, size_t smem,
                               cudaStream_t st) {
  if (cut.warps > 1) {
    if (rows == 1) return launch_cut<kBack, 4, 1, true>(p, cut, smem, st);
    return vecs == 3 ? launch_cut<kBack, 3, 2, true>(p, cut, smem, st)
                     : launch_cut<kBack, 4, 2, true>(p, cut, smem, st);
  }
  return vecs == 1   ? launch_cut<kBack, 1, 2, false>(p, cut, smem, st)
         : vecs == 2 ? launch_cut<kBack, 2, 2, false>(p, cut, smem, st)
         : vecs == 3 ? launch_cut<kBack, 3, 2, false>(p, cut, smem, st)
                     : launch_cut<kBack, 4, 2, false>(p, cut, smem, st);
}

template <bool kBack>
static cudaError_t combine(const CombineParams& p, cudaStream_t st) {
  const bool norm = p.gamma != nullptr;
  CombineCut cut;
  // a warp a row up to 1024 features (two, of as many rows at work: forward of 768 features
  // 14.0 us instead of 10.5, gradient of 1024 49 us instead of 44: plan, addresses and sums
  // are a warp's, whatever it has of the row)
  cut.inv_d = 1.f / static_cast<float>(p.D);
  cut.warps = (p.D + kWarpFeatures - 1) / kWarpFeatures;
  const int vecs = (p.D + 256 * cut.warps - 1) / (256 * cut.warps);
  cut.segs = p.k + (p.res != nullptr && (!kBack || norm) ? 1 : 0) +
             (kBack && norm ? 1 : 0);
  // as many row groups as the shared memory has room for two rows each: two CTAs an SM
  // (the gradient, which has more registers: one); one row where even one group has not
  const size_t row = static_cast<size_t>(cut.segs) * vecs * cut.warps * 512;
  const size_t params = norm ? sizeof(float) * p.D * (kBack ? 1 : 2) : 0;
  const size_t most = (kBack ? kCombineBytes : kCombineBytes / 2) - params;
  const int rows = row * 2 <= most ? 2 : 1;
  cut.groups = kCombineWarps / cut.warps;
  while (cut.groups > 1 && row * rows * cut.groups > most) --cut.groups;
  const int sms = api_device_sms();
  if (sms < 1) return cudaErrorInvalidDevice;
  const long long want = (p.T + cut.groups - 1) / cut.groups;
  const long long room = kBack ? (sms < kCombineMaxParts ? sms : kCombineMaxParts) : 2ll * sms;
  cut.ctas = static_cast<int>(want < room ? want : room);
  const size_t smem = row * rows * cut.groups + params;
  const cudaError_t e = launch_vecs<kBack>(p, cut, vecs, rows, smem, st);
  if (e != cudaSuccess || !kBack || !norm) return e;
  return launch_chained(sc_combine_reduce_kernel, dim3((2 * p.D + 31) / 32), dim3(1024), 0, st, p, cut.ctas);
}

template <bool kBack, int V, int kRows, bool kWide>
static cudaError_t configure_cut() {
  return cudaFuncSetAttribute(sc_combine_kernel<kBack, V, kRows, kWide>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              static_cast<int>(kCombineBytes));
}

template <bool kBack>
static cudaError_t configure_cuts() {
  cudaError_t e = configure_cut<kBack, 1, 2, false>();
  if (e == cudaSuccess) e = configure_cut<kBack, 2, 2, false>();
  if (e == cudaSuccess) e = configure_cut<kBack, 3, 2, false>();
  if (e == cudaSuccess) e = configure_cut<kBack, 4, 2, false>();
  if (e == cudaSuccess) e = configure_cut<kBack, 3, 2, true>();
  if (e == cudaSuccess) e = configure_cut<kBack, 4, 2, true>();
  if (e == cudaSuccess) e = configure_cut<kBack, 4, 1, true>();
  return e;
}

cudaError_t configure_combine() {
  const cudaError_t e = configure_cuts<false>();
  return e == cudaSuccess ? configure_cuts<true>() : e;
}

cudaError_t launch_combine(const CombineParams& p, cudaStream_t st) { return combine<false>(p, st); }
cudaError_t launch_combine_back(const CombineParams& p, cudaStream_t st) { return combine<true>(p, st); }

}  // namespace sc
