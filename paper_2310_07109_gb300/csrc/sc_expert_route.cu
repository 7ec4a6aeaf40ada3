// sc_expert_route.cu -- routing of the rows of a batch to experts: the choice
// of k of E experts a token, the gates, and the expert-sorted slots.
//
// For token t with logits l_e: the chosen experts are the k largest l_e above
// -inf (ties: the lowest e; NaN counts as -inf; fewer where fewer are above
// -inf), in descending order.  With m = max_e l_e the gate of choice j is
//   exp(l_j - m) / sum exp(l_i - m),
// the sum over the chosen experts (renormalize) or over all E.  A difference is
// taken as 0 where both sides are equal, so that +inf and the type's lowest
// value are ordinary logits.  Slots are numbered by (expert, token): expert e
// has slots offsets[e] .. offsets[e + 1], its tokens in increasing order.
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_expert.cuh"
#include "sm103_primitives.cuh"

namespace sc {

// Few values and short work per token: latency bounds both kernels (16384 tokens, E = 64,
// k = 8: 5 MB).  Hence 32 warps a CTA with the logits of a warp's four tokens on their way
// together, counts added up by all threads, and one kernel where one CTA has every token.
constexpr int kRouteThreads = 1024;
constexpr int kRouteBackThreads = 256;
constexpr int kRouteWords = kRouteTokens / 32;
constexpr int kRoutePerWarp = kRouteTokens / (kRouteThreads / 32);   // tokens of a warp per chunk
static_assert(kRouteTokens * kMaxChoices <= kRouteThreads, "an item a thread");
// Eight lanes have a token, four tokens a warp: the search for the next choice costs a
// warp's instructions once for all four (a warp a token and `redux`, four tokens in turn:
// 16384 tokens, E = 64, k = 8, 13.1 us instead of 11.5; 8192 tokens, E = 16, k = 2, 6.4
// instead of 4.7).
constexpr int kRouteLanes = 8;
static_assert(kRoutePerWarp == 32 / kRouteLanes && kMaxChoices <= kRouteLanes, "a lane a choice");

// Order-preserving map of a float to an unsigned number; 0 below every value that
// may be chosen (NaN, -inf).
__device__ __forceinline__ uint32_t route_key(float x) {
  if (!(x > -INFINITY)) return 0u;
  x += 0.f;   // -0 and +0 tie
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The float of a key that is not 0.
__device__ __forceinline__ float route_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key);
}

// exp(x - m), m >= x the maximum of the row; 1 where x equals m.
__device__ __forceinline__ float route_exp(float x, float m) { return x == m ? 1.f : expf(x - m); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

// Over the lanes that share a token.
__device__ __forceinline__ uint32_t token_max(uint32_t v) {
#pragma unroll
  for (int off = kRouteLanes / 2; off > 0; off >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}
__device__ __forceinline__ int token_min(int v) {
#pragma unroll
  for (int off = kRouteLanes / 2; off > 0; off >>= 1) v = min(v, __shfl_xor_sync(0xffffffffu, v, off));
  return v;
}
__device__ __forceinline__ float token_sum(float v) {
#pragma unroll
  for (int off = kRouteLanes / 2; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

__device__ __forceinline__ bool token_in_use(const int32_t* rows, int L, int t) {
  if (rows == nullptr) return true;
  const int b = t / L;
  return t - b * L < __ldg(rows + b);
}

// Exclusive sums of v[0 .. n), n <= kMaxExperts, added to `to`; the total to *total.  One warp.
__device__ __forceinline__ void scan_experts(const int* v, int n, int* to, int* total) {
  const int lane = threadIdx.x & 31;
  int run = 0;
  for (int e0 = 0; e0 < n; e0 += 32) {
    const int e = e0 + lane, mine = e < n ? v[e] : 0;
    int x = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, x, off);
      if (lane >= off) x += y;
    }
    if (e < n) to[e] += run + x - mine;
    run += __shfl_sync(0xffffffffu, x, 31);
  }
  if (lane == 0) *total = run;
}

// Where items (token x choice) i0 .. i1 go, from their ranks: slots, and the slots' tokens.
// `expert` and `rank`: of item i0 + threadIdx.x, loaded before.
__device__ __forceinline__ void place_items(const RouteParams& p, const int* base, int total, int i0, int i1,
                                            int expert, int rank) {
  for (int i = i0 + threadIdx.x; i < i1; i += kRouteThreads) {
    if (i >= i0 + kRouteThreads) {
      expert = p.expert[i];
      rank = p.slot[i];
    }
    if (expert >= 0) {
      const int s = base[expert] + rank;
      p.slot[i] = s;
      p.token[s] = i / p.k;
    }
    if (i >= total) p.token[i] = -1;
  }
}

// V logits a lane (its number of the eight + 8 v).  Writes the choices, the
// gates and, in `slot`, each choice's rank among the CTA's tokens with the same
// expert: the tokens of a chunk that chose an expert are bits of its mask, so the
// rank is a count of lower bits, whatever order the warps come in.  Where there is
// one CTA it goes on to the slots.
template <int V>
__global__ void __launch_bounds__(kRouteThreads) sc_route_choose_kernel(
    const __grid_constant__ RouteParams p) {
  __shared__ int count[kMaxExperts], base[kMaxExperts], total;   // count: before this chunk
  __shared__ int16_t pick[kRouteTokens * kMaxChoices];
  extern __shared__ uint32_t mask[];                             // [E][kRouteWords]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, own = lane % kRouteLanes;
  for (int i = tid; i < p.E * kRouteWords; i += kRouteThreads) mask[i] = 0;
  for (int i = tid; i < p.E; i += kRouteThreads) count[i] = base[i] = 0;
  pdl_wait();
  pdl_launch_dependents();
  __syncthreads();
  const int t0 = blockIdx.x * p.per_cta;
  const int t1 = static_cast<int>(min(static_cast<long long>(t0) + p.per_cta, p.T));
  int first_expert = -1, first_rank = -1;
  for (int c0 = t0; c0 < t1; c0 += kRouteTokens) {
    const int n = min(t1 - c0, kRouteTokens);
    const int i = warp * kRoutePerWarp + lane / kRouteLanes, t = c0 + i;
    const bool in = i < n && token_in_use(p.rows, p.L, t);
    float x[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = own + kRouteLanes * v;
      x[v] = in && e < p.E ? __ldg(p.logits + t * p.ld + e) : -INFINITY;
    }
    uint32_t key[V], mine = 0u;   // mine: lane j's is choice j's key, 0 where none is left
    int my_expert = -1;
#pragma unroll
    for (int v = 0; v < V; ++v) key[v] = route_key(x[v]);
    for (int j = 0; j < p.k; ++j) {
      uint32_t best = key[0];
#pragma unroll
      for (int v = 1; v < V; ++v) best = max(best, key[v]);
      best = token_max(best);
      int first = kMaxExperts;   // the lowest expert with it
#pragma unroll
      for (int v = V - 1; v >= 0; --v)
        if (key[v] == best) first = own + kRouteLanes * v;
      const int at = token_min(first);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (at == own + kRouteLanes * v) key[v] = 0u;
      if (own == j) mine = best, my_expert = at;
    }
    const bool chosen = mine != 0u;
    const uint32_t most = __shfl_sync(0xffffffffu, mine, 0, kRouteLanes);   // choice 0
    const float top = route_value(most);
    const float part = chosen ? route_exp(route_value(mine), top) : 0.f;
    float sum = part;
    if (!p.renormalize && most != 0u) {
      sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        // (more than 64 experts: loaded once more, the choices need the registers)
        const int e = own + kRouteLanes * v;
        const float l = V <= 8 ? x[v] : e < p.E ? __ldg(p.logits + t * p.ld + e) : -INFINITY;
        if (l > -INFINITY) sum += route_exp(l, top);
      }
    }
    sum = token_sum(sum);
    if (own < p.k && i < n) {
      pick[i * p.k + own] = static_cast<int16_t>(chosen ? my_expert : -1);
      p.gate[t * p.k + own] = chosen ? part / sum : 0.f;
      if (chosen) atomicOr(&mask[my_expert * kRouteWords + (i >> 5)], 1u << (i & 31));
    }
    __syncthreads();
    for (int i = tid; i < n * p.k; i += kRouteThreads) {
      const int e = pick[i], r = i / p.k;
      int rank = -1;
      if (e >= 0) {
        rank = count[e];
        for (int q = 0; q < (r >> 5); ++q) rank += __popc(mask[e * kRouteWords + q]);
        rank += __popc(mask[e * kRouteWords + (r >> 5)] & ((1u << (r & 31)) - 1u));
      }
      p.expert[c0 * p.k + i] = e;
      p.slot[c0 * p.k + i] = rank;
      first_expert = e;   // (one chunk of at most 1024 items: this thread's only one)
      first_rank = rank;
    }
    __syncthreads();
    for (int e = tid; e < p.E; e += kRouteThreads) {
      int c = count[e];
#pragma unroll
      for (int q = 0; q < kRouteWords; ++q) {
        c += __popc(mask[e * kRouteWords + q]);
        mask[e * kRouteWords + q] = 0;
      }
      count[e] = c;
    }
    __syncthreads();
  }
  if (gridDim.x > 1) {
    for (int e = tid; e < p.E; e += kRouteThreads) p.counts[blockIdx.x * p.E + e] = count[e];
    return;
  }
  if (warp == 0) scan_experts(count, p.E, base, &total);
  __syncthreads();
  for (int e = tid; e <= p.E; e += kRouteThreads) p.offsets[e] = e < p.E ? base[e] : total;
  place_items(p, base, total, t0 * p.k, t1 * p.k, first_expert, first_rank);
}

// Adds up the counts: an expert's first slot, and within it this CTA's; then turns
// the ranks into slots.  One CTA per choosing CTA, over the same tokens.
__global__ void __launch_bounds__(kRouteThreads) sc_route_place_kernel(
    const __grid_constant__ RouteParams p) {
  __shared__ int base[kMaxExperts], all[kMaxExperts];
  __shared__ int total;
  const int tid = threadIdx.x;
  for (int e = tid; e < p.E; e += kRouteThreads) base[e] = all[e] = 0;
  pdl_wait();
  pdl_launch_dependents();
  const int i0 = blockIdx.x * p.per_cta * p.k;
  const int i1 = static_cast<int>(min(static_cast<long long>(i0) + p.per_cta * p.k, p.T * p.k));
  int expert = -1, rank = -1;
  if (i0 + tid < i1) {
    expert = p.expert[i0 + tid];
    rank = p.slot[i0 + tid];
  }
  __syncthreads();
  // thread: expert tid % E of every (threads / E)-th CTA; whole numbers, any order
  const int per = kRouteThreads / p.E, e = tid % p.E, g = tid / p.E;
  if (g < per) {
    int before = 0, sum = 0;
#pragma unroll 8
    for (int c = g; c < static_cast<int>(gridDim.x); c += per) {
      const int v = __ldcg(p.counts + c * p.E + e);
      before += c < static_cast<int>(blockIdx.x) ? v : 0;
      sum += v;
    }
    if (before != 0) atomicAdd(&base[e], before);
    if (sum != 0) atomicAdd(&all[e], sum);
  }
  __syncthreads();
  if (tid < 32) scan_experts(all, p.E, base, &total);
  __syncthreads();
  if (blockIdx.x == 0)   // its own slots begin where the experts' do
    for (int o = tid; o <= p.E; o += kRouteThreads) p.offsets[o] = o < p.E ? base[o] : total;
  place_items(p, base, total, i0, i1, expert, rank);
}

// d logits of the gates.  With inner = sum_j g_j dg_j: at a chosen expert
// g_j (dg_j - inner) and 0 elsewhere (renormalize), or p_e ([e chosen] dg_e - inner)
// with p the softmax over all E.  A token without a choice has gradient 0.
template <int V>
__global__ void __launch_bounds__(kRouteBackThreads) sc_route_back_kernel(
    const __grid_constant__ RouteBackParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long t = static_cast<long long>(blockIdx.x) * (kRouteBackThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.T) return;
  const bool in = token_in_use(p.rows, p.L, static_cast<int>(t));
  int e = -1;
  float g = 0.f, dg = 0.f;
  if (lane < p.k && in) {
    e = __ldg(p.expert + t * p.k + lane);
    if (e >= 0) {
      g = __ldg(p.gate + t * p.k + lane);
      dg = __ldg(p.dgate + t * p.k + lane);
    }
  }
  const float inner = warp_sum(g * dg);
  const bool some = __any_sync(0xffffffffu, e >= 0);
  float d[V], pr[V];
  float top = -INFINITY;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int at = lane + 32 * v;
    d[v] = 0.f;
    pr[v] = !p.renormalize && some && at < p.E ? __ldg(p.logits + t * p.ld + at) : -INFINITY;
    if (!(pr[v] > -INFINITY)) pr[v] = -INFINITY;   // NaN is masked
    top = fmaxf(top, pr[v]);
  }
  if (!p.renormalize) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    float s = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      pr[v] = pr[v] > -INFINITY ? route_exp(pr[v], top) : 0.f;
      s += pr[v];
    }
    s = warp_sum(s);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      pr[v] = some ? pr[v] / s : 0.f;
      d[v] = -inner * pr[v];
    }
  }
  for (int j = 0; j < p.k; ++j) {
    const int ej = __shfl_sync(0xffffffffu, e, j);
    const float gj = __shfl_sync(0xffffffffu, g, j), dgj = __shfl_sync(0xffffffffu, dg, j);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (ej == lane + 32 * v) d[v] = p.renormalize ? gj * (dgj - inner) : pr[v] * (dgj - inner);
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (lane + 32 * v < p.E) p.dlogits[t * p.E + lane + 32 * v] = d[v];
}

static int route_ctas(long long T, int* per_cta) {
  const long long chunks = (T + kRouteTokens - 1) / kRouteTokens;
  const long long each = (chunks + kRouteMaxCtas - 1) / kRouteMaxCtas;
  *per_cta = static_cast<int>(each * kRouteTokens);
  return static_cast<int>((chunks + each - 1) / each);
}

cudaError_t launch_route(const RouteParams& in, cudaStream_t st) {
  RouteParams p = in;
  const int ctas = route_ctas(p.T, &p.per_cta);
  const size_t smem = static_cast<size_t>(p.E) * kRouteWords * 4;
  auto choose = p.E <= 8     ? sc_route_choose_kernel<1>
                : p.E <= 16  ? sc_route_choose_kernel<2>
                : p.E <= 32  ? sc_route_choose_kernel<4>
                : p.E <= 64  ? sc_route_choose_kernel<8>
                : p.E <= 128 ? sc_route_choose_kernel<16>
                             : sc_route_choose_kernel<32>;
  const cudaError_t e = launch_chained(choose, dim3(ctas), dim3(kRouteThreads), smem, st, p);
  if (e != cudaSuccess || ctas == 1) return e;
  return launch_chained(sc_route_place_kernel, dim3(ctas), dim3(kRouteThreads), 0, st, p);
}

cudaError_t launch_route_back(const RouteBackParams& p, cudaStream_t st) {
  constexpr int per = kRouteBackThreads / 32;
  const dim3 grid(static_cast<unsigned>((p.T + per - 1) / per));
  auto k = p.E <= 32 ? sc_route_back_kernel<1>
           : p.E <= 64 ? sc_route_back_kernel<2>
           : p.E <= 128 ? sc_route_back_kernel<4> : sc_route_back_kernel<8>;
  return launch_chained(k, grid, dim3(kRouteBackThreads), 0, st, p);
}

}  // namespace sc
