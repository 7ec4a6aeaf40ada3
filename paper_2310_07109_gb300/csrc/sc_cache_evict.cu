// sc_cache_evict.cu -- eviction from a pruned key-value cache by accumulated weight.
//
// A list keeps the k = budget slots that rank highest (protected ones, then by acc, ties to the lower slot).
// Survivors below k stay; the others fill the places that are free below k, in order.  Sources are
// at k or above and destinations below, so the rows move in place, in any order, all at once, and no
// more of them than are free: at most min(k, n - k), where closing the gaps in order would move
// nearly every row behind the first one (half of 8192 slots: 2048 rows instead of 4096).
//
// Two launches:
//   pick   a CTA a list, or a cluster of up to eight with a stretch of a long list each.  Its slots' 32-bit keys (acc's
//          bits in an order-preserving form) go into shared memory; the cut is found in passes over them, each of
//          which cuts the range that holds it into at most 256 equal parts (by bits of the difference to its lower end:
//          keys are logarithms nearly, so weights spread over the parts; digits of the keys themselves put most of
//          them into two or three, whose additions wait for one another).  Then a bit a slot, and ranks of ties, free places and
//          their fillers from prefix sums over the bits, put together in shared memory.  128 lists of 7400 to 8192 slots, a CTA
//          each: 13 us with cold caches (the first version, with digits: 29)
//   move   the rows of K and V, bound by memory, and acc and pos.  Half of the same lists' slots go, 128 features: 45 us with
//          cold caches, 220 MB of DRAM traffic (4.9 TB/s); the call 55.6
#include <algorithm>
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_cache.cuh"
#include "sc_expert.cuh"

namespace sc {

constexpr int kPickThreads = 1024;
constexpr int kPickWarps = kPickThreads / 32;
constexpr int kMoveThreads = 256;
constexpr int kMoveSlots = 1024;   // whose acc and pos a CTA moves
constexpr uint32_t kProtected = 0xffffffffu;
// Slots of a CTA where there are SMs for more CTAs: eight lists of 12000 take 14.8 us with two CTAs each and 14.3 with one, of 16384
// 16.2 and 16.7, of 20000 17.4 with four and 20.2 with two.  An SM holds one of these CTAs: 128 lists of 8224 take 51 us with
// two CTAs each (two waves), 40 with one.
constexpr int kPickSlots = 8192;
constexpr int kMostSlots = SC_MAX_CACHE / 8;
constexpr int kParts = 256;

// What a slot ranks by: protected, then acc in order (-0 as 0); a NaN, or a slot without a position, last.
__device__ __forceinline__ uint32_t rank_key(const EvictParams& p, float acc, int pos, int late) {
  if (pos < 0) return 0u;
  if (pos < p.sinks || pos >= late) return kProtected;
  if (acc != acc) return 0u;
  const uint32_t u = __float_as_uint(acc + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;   // 0x007fffff (-inf) .. 0xff800000 (+inf)
}

struct PickSmem {
  alignas(16) uint32_t hist[2][kParts];   // of every other pass: the cluster's CTAs read one while the next is cleared
  uint32_t low[kPickWarps], high[kPickWarps];
  int count[kPickWarps][2];
  uint32_t range[4];   // of the CTA: lowest and highest key, protected ones, those that rank last
  int ties;            // of the CTA
  uint32_t places;     // of the CTA: free ones, fillers << 16
  int found[3];        // part, how many of it are still to take, how many it has
};

// A word of the shared memory of the cluster's CTA `rank`.
__device__ __forceinline__ uint32_t of_rank(const void* word, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(dsmem_addr(smem_u32(word), rank)) : "memory");
  return v;
}

// Exclusive prefix over the CTA's threads of two counts (each below 2^16 in all, packed; or of one), and their totals.
__device__ __forceinline__ uint32_t scan_cta(PickSmem& sm, uint32_t v, uint32_t& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  uint32_t upto = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += x;
  }
  __syncthreads();   // (the last one's have been read)
  if (lane == 31) sm.low[warp] = upto;
  __syncthreads();
  const uint32_t w = sm.low[lane];
  all = __reduce_add_sync(0xffffffffu, w);
  return __reduce_add_sync(0xffffffffu, lane < warp ? w : 0u) + upto - v;
}

// Shared memory of a CTA in words: keys of its share of a list, two bits a slot up to a multiple of 16 bytes, and
// the cluster's counts.
template <int kCtas>
__host__ __device__ constexpr int pick_room(int C) {
  return ((C + kCtas - 1) / kCtas + 31) & ~31;
}
__host__ __device__ constexpr int pick_bits_end(int room) { return (room + room / 16 + 3) & ~3; }
template <int kCtas>
constexpr size_t pick_bytes(int C) {
  return sizeof(uint32_t) * (pick_bits_end(pick_room<kCtas>(C)) + (kCtas > 1 ? kParts : 0));
}

template <int kCtas>
__global__ void __launch_bounds__(kPickThreads, 1) evict_pick_kernel(const EvictParams p) {
  static_assert(kPickWarps == 32, "a lane a warp");
  __shared__ PickSmem sm;
  extern __shared__ __align__(16) uint32_t held[];   // keys, then two bits a slot, then the cluster's counts
  pdl_wait();
  pdl_launch_dependents();
  const int list = blockIdx.x / kCtas, rank = blockIdx.x % kCtas, b = list / p.G, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long base = static_cast<long long>(list) * p.C;
  const int n = min(max(__ldcg(p.len + list), 0), p.C), k = p.budget;
  const int late = p.seen[b] - p.recent;
  auto sync = [&]() {
    if (kCtas > 1)
      cluster_sync();
    else
      __syncthreads();
  };
  if (n <= k || n - k <= p.slack) {   // (of all CTAs of the list)
    sync();   // len is read
    if (tid == 0 && rank == 0) {
      p.moved[list] = 0;
      p.len_out[list] = n;
    }
    return;
  }
  // this CTA's slots first .. first + own - 1
  const int stretch = (((n + kCtas - 1) / kCtas) + 31) & ~31, first = min(rank * stretch, n), own = min(stretch, n - first);
  const float* acc = p.acc + base + first;
  const int32_t* pos = p.pos + base + first;
  const int room = pick_room<kCtas>(p.C);
  uint32_t* above = held + room;
  uint32_t* tied = above + room / 32;
  uint32_t* cluster_hist = held + pick_bits_end(room);
  if (tid < kParts) sm.hist[0][tid] = 0;
  // protected ones and those that rank last apart, the range of the others' keys
  uint32_t low = 0xffffffffu, high = 0;
  int safe = 0, none = 0;
  constexpr int kBatch = 8;
  for (int j0 = tid; j0 < own; j0 += kBatch * kPickThreads) {
    float a[kBatch];
    int q[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int j = j0 + u * kPickThreads;
      a[u] = 0.f;
      q[u] = -1;
      if (j < own) {
        a[u] = __ldcg(acc + j);
        q[u] = __ldcg(pos + j);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int j = j0 + u * kPickThreads;
      if (j >= own) break;
      const uint32_t key = rank_key(p, a[u], q[u], late);
      held[j] = key;
      safe += key == kProtected;
      none += key == 0;
      if (key != kProtected && key != 0) {
        low = min(low, key);
        high = max(high, key);
      }
    }
  }
  low = __reduce_min_sync(0xffffffffu, low);
  high = __reduce_max_sync(0xffffffffu, high);
  safe = __reduce_add_sync(0xffffffffu, safe);
  none = __reduce_add_sync(0xffffffffu, none);
  if (lane == 0) {
    sm.low[warp] = low;
    sm.high[warp] = high;
    sm.count[warp][0] = safe;
    sm.count[warp][1] = none;
  }
  __syncthreads();
  low = __reduce_min_sync(0xffffffffu, sm.low[lane]);
  high = __reduce_max_sync(0xffffffffu, sm.high[lane]);
  safe = __reduce_add_sync(0xffffffffu, sm.count[lane][0]);
  none = __reduce_add_sync(0xffffffffu, sm.count[lane][1]);
  if (kCtas > 1) {
    if (tid == 0) {
      sm.range[0] = low;
      sm.range[1] = high;
      sm.range[2] = safe;
      sm.range[3] = none;
    }
    cluster_sync();
    const uint32_t r = lane < kCtas ? lane : 0;
    low = __reduce_min_sync(0xffffffffu, of_rank(&sm.range[0], r));
    high = __reduce_max_sync(0xffffffffu, of_rank(&sm.range[1], r));
    const uint32_t s = of_rank(&sm.range[2], r), z = of_rank(&sm.range[3], r);
    safe = __reduce_add_sync(0xffffffffu, lane < kCtas ? s : 0);
    none = __reduce_add_sync(0xffffffffu, lane < kCtas ? z : 0);
  }
  // keys above `high` survive, and the first `want` of the `count` ones from low to high: all of them, or low is high
  int want = k - safe, count = n - safe - none;
  if (want <= 0) {
    low = high = kProtected;
    want = k;
    count = safe;
  } else if (want > count) {
    low = high = 0;
    want -= count;
    count = none;
  }
  for (int pass = 0; low != high && want != count; pass ^= 1) {
    uint32_t* hist = sm.hist[pass];
    const int shift = max(0, 24 - __clz(high - low));   // at most 256 parts of 2^shift
#pragma unroll 4
    for (int j = tid; j < own; j += kPickThreads) {
      const uint32_t key = held[j];
      if (key >= low && key <= high) atomicAdd(&hist[(key - low) >> shift], 1u);
    }
    sync();
    if (tid < kParts) {
      if (kCtas > 1) {
        uint32_t all = 0;
#pragma unroll
        for (int r = 0; r < kCtas; ++r) all += of_rank(&hist[tid], r);
        cluster_hist[tid] = all;
      }
      sm.hist[pass ^ 1][tid] = 0;
    }
    const uint32_t* counts = kCtas > 1 ? cluster_hist : hist;
    if (kCtas > 1) __syncthreads();
    if (warp == 0) {   // lane l has parts 255 - 8 l .. 248 - 8 l, the largest first
      int mine[8], total = 0;
      const uint4 hi = reinterpret_cast<const uint4*>(counts)[63 - 2 * lane], lo = reinterpret_cast<const uint4*>(counts)[62 - 2 * lane];
      const uint32_t eight[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
#pragma unroll
      for (int i = 0; i < 8; ++i) total += mine[i] = static_cast<int>(eight[i]);
      int upto = total;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      int before = upto - total;
      if (before < want && want <= upto) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (before < want && want <= before + mine[i]) {
            sm.found[0] = 255 - 8 * lane - i;
            sm.found[1] = want - before;
            sm.found[2] = mine[i];
          }
          before += mine[i];
        }
      }
    }
    __syncthreads();
    low += static_cast<uint32_t>(sm.found[0]) << shift;
    high = low + min(high - low, (1u << shift) - 1u);   // (the part's own end may lie beyond 2^32)
    want = sm.found[1];
    count = sm.found[2];
  }
  // a bit a slot
#pragma unroll 4
  for (int j0 = 0; j0 < own; j0 += kPickThreads) {
    const int j = j0 + tid;
    const uint32_t key = j < own ? held[j] : 0;
    const uint32_t over = __ballot_sync(0xffffffffu, j < own && key > high);
    const uint32_t in = __ballot_sync(0xffffffffu, j < own && key >= low && key <= high);
    if (lane == 0 && j < own) {
      above[j / 32] = over;
      tied[j / 32] = in;
    }
  }
  __syncthreads();
  const uint8_t* above8 = reinterpret_cast<const uint8_t*>(above);
  uint8_t* tied8 = reinterpret_cast<uint8_t*>(tied);
  const int bytes = (own + 7) / 8;
  if (want != count) {   // the first `want` of equal ones
    int done = 0;
    if (kCtas > 1) {   // those of the CTAs before this one
      int mine = 0;
      for (int i = tid; i < bytes; i += kPickThreads) mine += __popc(tied8[i]);
      uint32_t all;
      scan_cta(sm, mine, all);
      if (tid == 0) sm.ties = static_cast<int>(all);
      cluster_sync();
      const uint32_t c = of_rank(&sm.ties, lane < kCtas ? lane : 0);
      done = __reduce_add_sync(0xffffffffu, lane < rank ? c : 0);
    }
    for (int i0 = 0; i0 < bytes; i0 += kPickThreads) {
      const int i = i0 + tid;
      uint32_t in = i < bytes ? tied8[i] : 0u, all;
      const int before = done + static_cast<int>(scan_cta(sm, __popc(in), all));
      for (int left = want - before; __popc(in) > max(left, 0);) in &= ~(1u << (31 - __clz(in)));
      if (i < bytes) tied8[i] = static_cast<uint8_t>(in);
      done += static_cast<int>(all);
    }
  }
  // free places below k and survivors from k on, in order
  int2* pairs = p.pairs + list * p.pair_pitch;
  uint8_t* free8 = p.free_places + list * p.free_pitch + first / 8;
  auto of_byte = [&](int i, uint32_t& places, uint32_t& fills, uint32_t& low_ones) {
    const int j = first + 8 * i;
    const uint32_t keep = i < bytes ? above8[i] | tied8[i] : 0u;
    low_ones = j >= k ? 0u : k - j >= 8 ? 0xffu : (1u << (k - j)) - 1u;   // slots below k
    places = i < bytes ? ~keep & low_ones : 0u;
    fills = keep & ~low_ones & 0xffu;
  };
  int free_at = 0, fill_at = 0, all_free = 0;
  if (kCtas > 1) {   // those of the CTAs before this one (its own are at most 2^15 each)
    uint32_t mine = 0, all, places, fills, low_ones;
    for (int i = tid; i < bytes; i += kPickThreads) {
      of_byte(i, places, fills, low_ones);
      mine += __popc(places) | __popc(fills) << 16;
    }
    scan_cta(sm, mine, all);
    if (tid == 0) sm.places = all;
    cluster_sync();
    const uint32_t c = of_rank(&sm.places, lane < kCtas ? lane : 0);
    free_at = __reduce_add_sync(0xffffffffu, lane < rank ? c & 0xffffu : 0);
    fill_at = __reduce_add_sync(0xffffffffu, lane < rank ? c >> 16 : 0);
    all_free = __reduce_add_sync(0xffffffffu, lane < kCtas ? c & 0xffffu : 0);
  }
  // (the keys are done with: places from their start on, fillers from their end back)
  int my_free = 0, my_fill = 0;
  for (int i0 = 0; i0 < bytes; i0 += kPickThreads) {
    const int i = i0 + tid, j = first + 8 * i;
    uint32_t places, fills, low_ones, all;
    of_byte(i, places, fills, low_ones);
    const uint32_t before = scan_cta(sm, __popc(places) | __popc(fills) << 16, all);
    if (low_ones != 0 && i < bytes) free8[i] = static_cast<uint8_t>(places);
    for (int at = my_free + static_cast<int>(before & 0xffffu); places != 0; places &= places - 1) held[at++] = j + __ffs(places) - 1;
    for (int at = room - 1 - my_fill - static_cast<int>(before >> 16); fills != 0; fills &= fills - 1) held[at--] = j + __ffs(fills) - 1;
    my_free += static_cast<int>(all & 0xffffu);
    my_fill += static_cast<int>(all >> 16);
  }
  __syncthreads();
  // As many are free as fill them, min(k, n - k) at most, which a plan has room for; none goes beyond it all the same.
  const int plan = static_cast<int>(p.pair_pitch);
  if (kCtas == 1) {
    my_free = min(my_free, plan);
    for (int i = tid; i < my_free; i += kPickThreads) pairs[i] = make_int2(held[i], held[room - 1 - i]);
  } else {
    for (int i = tid; i < min(my_free, plan - free_at); i += kPickThreads) pairs[free_at + i].x = held[i];
    for (int i = tid; i < min(my_fill, plan - fill_at); i += kPickThreads) pairs[fill_at + i].y = held[room - 1 - i];
  }
  if (kCtas > 1) cluster_sync();   // (all have read all; len too)
  if (tid == 0 && rank == 0) {
    p.moved[list] = kCtas > 1 ? min(all_free, plan) : my_free;
    p.len_out[list] = k;
  }
}

// acc and pos of 1024 slots of a list: those that stay (where the outputs lie apart), and as many that move.
__device__ __forceinline__ void move_weights(const EvictParams& p, int id, int chunks) {
  const int list = id / chunks, i0 = (id - list * chunks) * kMoveSlots;
  const int m = __ldcg(p.moved + list), n = __ldcg(p.len_out + list);
  const long long base = static_cast<long long>(list) * p.C;
  const bool apart_acc = p.acc_out != p.acc, apart_pos = p.pos_out != p.pos;
  const uint8_t* free8 = p.free_places + list * p.free_pitch;
  const int2* pairs = p.pairs + list * p.pair_pitch;
  constexpr int kBatch = kMoveSlots / kMoveThreads;
  int2 at[kBatch];
  float acc[kBatch], moved_acc[kBatch];
  int pos[kBatch], moved_pos[kBatch];
  bool stays[kBatch];
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int i = i0 + u * kMoveThreads + static_cast<int>(threadIdx.x);
    stays[u] = (apart_acc || apart_pos) && i < n && (m == 0 || !(__ldcg(free8 + i / 8) >> (i & 7) & 1));
    if ((apart_acc || apart_pos) && i < n) {
      acc[u] = __ldcg(p.acc + base + i);
      pos[u] = __ldcg(p.pos + base + i);
    }
    if (i < m) at[u] = __ldcg(pairs + i);
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    if (i0 + u * kMoveThreads + static_cast<int>(threadIdx.x) >= m) continue;
    moved_acc[u] = __ldcg(p.acc + base + at[u].y);
    moved_pos[u] = __ldcg(p.pos + base + at[u].y);
  }
#pragma unroll
  for (int u = 0; u < kBatch; ++u) {
    const int i = i0 + u * kMoveThreads + static_cast<int>(threadIdx.x);
    if (stays[u] && apart_acc) p.acc_out[base + i] = acc[u];
    if (stays[u] && apart_pos) p.pos_out[base + i] = pos[u];
    if (i < m) {
      p.acc_out[base + at[u].x] = moved_acc[u];
      p.pos_out[base + at[u].x] = moved_pos[u];
    }
  }
}

// The first CTAs move acc and pos; of the others each has every chunks-th piece of the moves of a head, d / 8 lanes a
// row, K and V together.
__global__ void __launch_bounds__(kMoveThreads) evict_move_kernel(const EvictParams p, int chunks, int weight_chunks) {
  pdl_wait();
  pdl_launch_dependents();
  const int weight_ctas = p.B * p.G * weight_chunks, id = static_cast<int>(blockIdx.x) - weight_ctas;
  if (id < 0) return move_weights(p, blockIdx.x, weight_chunks);
  const int unit = id / chunks, chunk = id - unit * chunks;
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

namespace {

template <int kCtas>
cudaError_t launch_pick(const EvictParams& p, cudaStream_t st) {
  const cudaError_t e = allow_shared<evict_pick_kernel<kCtas>>(pick_bytes<kCtas>(std::min(SC_MAX_CACHE, kMostSlots * kCtas)));
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.B * p.G * kCtas);
  cfg.blockDim = dim3(kPickThreads);
  cfg.dynamicSmemBytes = pick_bytes<kCtas>(p.C);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kCtas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = kCtas > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, evict_pick_kernel<kCtas>, p);
}

}  // namespace

cudaError_t launch_evict(const EvictParams& p, cudaStream_t st) {
  // CTAs of a list: as many as its slots need, and twice as many while there are SMs for these
  int n = 1;
  while (n < 8 && ((p.C + n - 1) / n > kMostSlots ||
                   ((p.C + n - 1) / n > kPickSlots && static_cast<long long>(p.B) * p.G * n * 2 <= kCacheSms)))
    n *= 2;
  cudaError_t e = n == 1 ? launch_pick<1>(p, st) : n == 2 ? launch_pick<2>(p, st) : n == 4 ? launch_pick<4>(p, st) : launch_pick<8>(p, st);
  const bool evicts = p.budget < p.C, apart = p.acc_out != p.acc || p.pos_out != p.pos;
  if (e != cudaSuccess || (!evicts && !apart)) return e;
  const long long units = static_cast<long long>(p.B) * p.Hk;
  int chunks = 0;
  if (evicts) {
    const int most = std::min(p.budget, p.C - p.budget), rows = 4 * (kMoveThreads / (p.d / 8));
    chunks = static_cast<int>(std::min<long long>(std::max<long long>(1, kCacheSms * 8 / units), (most + rows - 1) / rows));
  }
  const long long slots = std::min<long long>(p.C, static_cast<long long>(p.budget) + p.slack);
  const int weight_chunks = static_cast<int>((slots + kMoveSlots - 1) / kMoveSlots);
  const long long ctas = units * chunks + static_cast<long long>(p.B) * p.G * weight_chunks;
  return launch_chained(evict_move_kernel, dim3(static_cast<unsigned>(ctas)), dim3(kMoveThreads), 0, st, p, chunks, weight_chunks);
}

}  // namespace sc
