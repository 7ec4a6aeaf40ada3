// sc_cache_evict.cu -- eviction from a pruned key-value cache by accumulated weight.
//
// A list keeps the k = budget slots that rank highest (protected ones, then by acc, ties to the lower slot).
// Survivors below k stay; the others fill the places that are free below k, in order.  Sources are
// at k or above and destinations below, so the rows move in place, in any order, all at once, and no
// more of them than are free: at most min(k, n - k), where closing the gaps in order would move
// nearly every row behind the first one (half of 8192 slots: 2048 rows instead of 4096).
//
// Two launches:
//   pick   a CTA a list: the cut by a radix search over 32-bit keys, eight bits at a time (acc's bits in
//          an order-preserving form), then ranks of ties, free places and their fillers from ballots: warps
//          have consecutive stretches of slots, so that ranks follow the slots
//   move   the rows of K and V, bound by memory
#include <algorithm>
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_cache.cuh"
#include "sc_expert.cuh"

namespace sc {

constexpr int kPickThreads = 1024;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kMoveThreads = 256;
constexpr uint32_t kProtected = 0xffffffffu;

// What a slot ranks by: protected, then acc in order (-0 as 0); a NaN, or a slot without a position, last.
__device__ __forceinline__ uint32_t rank_key(const EvictParams& p, float acc, int pos, int late) {
  if (pos < 0) return 0u;
  if (pos < p.sinks || pos >= late) return kProtected;
  if (acc != acc) return 0u;
  const uint32_t u = __float_as_uint(acc + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;   // 0x007fffff (-inf) .. 0xff800000 (+inf)
}

struct PickSmem {
  uint32_t hist[256];
  int warp_sum[kPickWarps][2];
  int found[2];   // digit, how many of it are still to take
};

// Exclusive prefixes over the warps of two sums, and their totals.
__device__ __forceinline__ void scan_warps(PickSmem& sm, int a, int b, int& before_a, int& before_b, int& all_a, int& all_b) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0) {
    sm.warp_sum[warp][0] = a;
    sm.warp_sum[warp][1] = b;
  }
  __syncthreads();
  const int va = sm.warp_sum[lane][0], vb = sm.warp_sum[lane][1];
  before_a = __reduce_add_sync(0xffffffffu, lane < warp ? va : 0);
  before_b = __reduce_add_sync(0xffffffffu, lane < warp ? vb : 0);
  all_a = __reduce_add_sync(0xffffffffu, va);
  all_b = __reduce_add_sync(0xffffffffu, vb);
}

__global__ void __launch_bounds__(kPickThreads) evict_pick_kernel(const EvictParams p) {
  __shared__ PickSmem sm;
  pdl_wait();
  pdl_launch_dependents();
  const int list = blockIdx.x, b = list / p.G, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long base = static_cast<long long>(list) * p.C;
  const float* acc = p.acc + base;
  const int32_t* pos = p.pos + base;
  const int n = min(max(__ldcg(p.len + list), 0), p.C), k = p.budget;
  const int late = __ldg(p.seen + b) - p.recent;
  const bool apart_acc = p.acc_out != p.acc, apart_pos = p.pos_out != p.pos;
  if (n <= k || n - k <= p.slack) {
    for (int j = tid; j < n; j += kPickThreads) {
      if (apart_acc) p.acc_out[base + j] = acc[j];
      if (apart_pos) p.pos_out[base + j] = pos[j];
    }
    __syncthreads();   // len is read
    if (tid == 0) {
      p.moved[list] = 0;
      p.len_out[list] = n;
    }
    return;
  }
  // the cut: keys above it survive, and the first `ties` of those equal to it
  uint32_t cut = 0, mask = 0;
  int ties = k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (tid < 256) sm.hist[tid] = 0;
    __syncthreads();
    for (int j = tid; j < n; j += kPickThreads) {
      const uint32_t key = rank_key(p, acc[j], pos[j], late);
      if ((key & mask) == cut) atomicAdd(&sm.hist[(key >> shift) & 255], 1u);
    }
    __syncthreads();
    if (warp == 0) {   // lane l has digits 255 - 8 l .. 248 - 8 l, the largest first
      int own[8], total = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) total += own[i] = static_cast<int>(sm.hist[255 - 8 * lane - i]);
      int upto = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      int before = upto - total;
      if (before < ties && ties <= upto) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (before < ties && ties <= before + own[i]) {
            sm.found[0] = 255 - 8 * lane - i;
            sm.found[1] = ties - before;
          }
          before += own[i];
        }
      }
    }
    __syncthreads();
    cut |= static_cast<uint32_t>(sm.found[0]) << shift;
    mask |= 255u << shift;
    ties = sm.found[1];
    __syncthreads();
  }
  // ranks: each warp a stretch of slots
  const int stretch = ((n + kPickWarps - 1) / kPickWarps + 31) & ~31;
  const int j0 = min(warp * stretch, n), j1 = min(j0 + stretch, n);
  int equal = 0, tied, unused, all, none;
  for (int j = j0 + lane; j - lane < j1; j += 32)
    equal += __popc(__ballot_sync(0xffffffffu, j < j1 && rank_key(p, acc[j], pos[j], late) == cut));
  scan_warps(sm, equal, 0, tied, unused, all, none);
  // (a lambda over the warp's stretch: survivors' ballots in order)
  const uint32_t below = (1u << lane) - 1u;
  auto over = [&](auto&& each) {
    int run = tied;
    for (int j = j0 + lane; j - lane < j1; j += 32) {
      const uint32_t key = j < j1 ? rank_key(p, acc[j], pos[j], late) : 0u;
      const uint32_t eq = __ballot_sync(0xffffffffu, j < j1 && key == cut);
      const bool keep = j < j1 && (key > cut || (key == cut && run + __popc(eq & below) < ties));
      run += __popc(eq);
      each(j, j < j1 && j < k && !keep, keep && j >= k);
    }
  };
  int free_ = 0, fill = 0;
  over([&](int, bool is_free, bool is_fill) {
    free_ += __popc(__ballot_sync(0xffffffffu, is_free));
    fill += __popc(__ballot_sync(0xffffffffu, is_fill));
  });
  int free_at, fill_at, all_free, all_fill;
  scan_warps(sm, free_, fill, free_at, fill_at, all_free, all_fill);
  int2* pairs = p.pairs + list * p.pair_pitch;
  over([&](int j, bool is_free, bool is_fill) {
    const uint32_t f = __ballot_sync(0xffffffffu, is_free), g = __ballot_sync(0xffffffffu, is_fill);
    if (is_free) pairs[free_at + __popc(f & below)].x = j;
    if (is_fill) pairs[fill_at + __popc(g & below)].y = j;
    free_at += __popc(f);
    fill_at += __popc(g);
  });
  __syncthreads();
  // acc and pos: places that stay, then the filled ones
  if (apart_acc || apart_pos) {
    for (int j = tid; j < k; j += kPickThreads) {
      if (apart_acc) p.acc_out[base + j] = acc[j];
      if (apart_pos) p.pos_out[base + j] = pos[j];
    }
    __syncthreads();
  }
  for (int i = tid; i < all_free; i += kPickThreads) {
    const int2 m = pairs[i];
    const float a = acc[m.y];
    const int q = pos[m.y];
    p.acc_out[base + m.x] = a;
    p.pos_out[base + m.x] = q;
  }
  if (tid == 0) {
    p.moved[list] = all_free;
    p.len_out[list] = k;
  }
}

// A CTA has every chunks-th piece of the moves of a head; d / 8 lanes a row, K and V together.
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p, int chunks) {
  pdl_wait();
  pdl_launch_dependents();
  const int unit = blockIdx.x / chunks, chunk = blockIdx.x - unit * chunks;
  const int b = unit / p.Hk, hk = unit - b * p.Hk, list = b * p.G + hk / (p.Hk / p.G);
  const int m = __ldcg(p.moved + list), lanes = p.d / 8, at_once = kMoveThreads / lanes;
  const int c = threadIdx.x % lanes, r = threadIdx.x / lanes;
  if (r >= at_once) return;
  const int2* pairs = p.pairs + list * p.pair_pitch;
  uint16_t* kh = p.k + b * p.stride_b + hk * p.stride_h + c * 8;
  uint16_t* vh = p.v + b * p.stride_b + hk * p.stride_h + c * 8;
  constexpr int kBatch = 4;
  const int step = chunks * at_once;
  for (int i0 = chunk * at_once + r; i0 < m; i0 += step * kBatch) {
    uint4 k[kBatch], v[kBatch];
    int to[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = i0 + u * step;
      to[u] = -1;
      if (i >= m) continue;
      const int2 at = __ldcg(pairs + i);
      to[u] = at.x;
      k[u] = *reinterpret_cast<const uint4*>(kh + at.y * p.stride_c);
      v[u] = *reinterpret_cast<const uint4*>(vh + at.y * p.stride_c);
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (to[u] < 0) continue;
      *reinterpret_cast<uint4*>(kh + to[u] * p.stride_c) = k[u];
      *reinterpret_cast<uint4*>(vh + to[u] * p.stride_c) = v[u];
    }
  }
}

cudaError_t launch_evict(const EvictParams& p, cudaStream_t st) {
  cudaError_t e = launch_chained(evict_pick_kernel, dim3(p.B * p.G), dim3(kPickThreads), 0, st, p);
  if (e != cudaSuccess || p.budget >= p.C) return e;   // (no list is over its budget)
  const long long units = static_cast<long long>(p.B) * p.Hk;
  const int most = std::min(p.budget, p.C - p.budget), rows = 4 * (kMoveThreads / (p.d / 8));
  const long long want = std::max<long long>(1, kCacheSms * 8 / units);
  const int chunks = static_cast<int>(std::min<long long>(want, (most + rows - 1) / rows));
  return launch_chained(evict_move_kernel, dim3(static_cast<unsigned>(units * chunks)), dim3(kMoveThreads), 0, st, p, chunks);
}

}  // namespace sc
