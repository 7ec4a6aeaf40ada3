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

constexpr int kRouteThreads = 256;
constexpr int kRouteWords = kRouteTokens / 32;

// Order-preserving map of a float to an unsigned number; 0 below every value that
// may be chosen (NaN, -inf).
__device__ __forceinline__ uint32_t route_key(float x) {
  if (!(x > -INFINITY)) return 0u;
  x += 0.f;   // -0 and +0 tie
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// exp(x - m), m >= x the maximum of the row; 1 where x equals m.
__device__ __forceinline__ float route_exp(float x, float m) { return x == m ? 1.f : expf(x - m); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
  return v;
}

__device__ __forceinline__ bool token_in_use(const int32_t* rows, int L, long long t) {
  if (rows == nullptr) return true;
  const long long b = t / L;
  return t - b * L < __ldg(rows + b);
}

// One warp per token, V logits a lane (expert lane + 32 v).  Writes the choices, the
// gates and, in `slot`, each choice's rank among the CTA's tokens with the same
// expert: the tokens of a chunk that chose an expert are bits of its mask, so the
// rank is a count of lower bits, whatever order the warps come in.
template <int V>
__global__ void __launch_bounds__(kRouteThreads) sc_route_choose_kernel(
    const __grid_constant__ RouteParams p) {
  extern __shared__ uint32_t route_smem[];
  uint32_t* mask = route_smem;                              // [E][kRouteWords]
  int* count = reinterpret_cast<int*>(mask + p.E * kRouteWords);   // [E] before this chunk
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  for (int i = tid; i < p.E * kRouteWords; i += kRouteThreads) mask[i] = 0;
  for (int i = tid; i < p.E; i += kRouteThreads) count[i] = 0;
  pdl_wait();
  pdl_launch_dependents();
  __syncthreads();
  const long long t0 = static_cast<long long>(blockIdx.x) * p.per_cta;
  const long long t1 = min(t0 + p.per_cta, p.T);
  for (long long c0 = t0; c0 < t1; c0 += kRouteTokens) {
    const int n = static_cast<int>(min(t1 - c0, static_cast<long long>(kRouteTokens)));
    for (int i = warp; i < n; i += kRouteThreads / 32) {
      const long long t = c0 + i;
      float x[V];
      uint32_t key[V];
      const bool in = token_in_use(p.rows, p.L, t);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int e = lane + 32 * v;
        x[v] = in && e < p.E ? __ldg(p.logits + t * p.ld + e) : -INFINITY;
        key[v] = route_key(x[v]);
        if (key[v] == 0u) x[v] = -INFINITY;
      }
      float top = 0.f, total = 0.f, mine = 0.f;
      int my_expert = -1;
      for (int j = 0; j < p.k; ++j) {
        uint32_t best = key[0];
#pragma unroll
        for (int v = 1; v < V; ++v) best = max(best, key[v]);
        best = __reduce_max_sync(0xffffffffu, best);
        if (best == 0u) break;
        int at = 0x7fffffff;
        float val = 0.f;
#pragma unroll
        for (int v = V - 1; v >= 0; --v)
          if (key[v] == best) at = lane + 32 * v, val = x[v];
        const int e = __reduce_min_sync(0xffffffffu, at);
        val = __shfl_sync(0xffffffffu, val, e & 31);
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (e == lane + 32 * v) key[v] = 0u;
        if (j == 0) {
          top = val;
          if (!p.renormalize) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) s += route_exp(x[v], top);
            total = warp_sum(s);
          }
        }
        const float w = route_exp(val, top);
        if (p.renormalize) total += w;
        if (lane == j) mine = w, my_expert = e;
      }
      if (lane < p.k) {
        p.expert[t * p.k + lane] = my_expert;
        p.gate[t * p.k + lane] = my_expert >= 0 ? mine / total : 0.f;
        if (my_expert >= 0)
          atomicOr(&mask[my_expert * kRouteWords + (i >> 5)], 1u << (i & 31));
      }
    }
    __syncthreads();
    for (int i = tid; i < n * p.k; i += kRouteThreads) {
      const long long at = c0 * p.k + i;
      const int e = p.expert[at], r = i / p.k;
      int rank = -1;
      if (e >= 0) {
        rank = count[e];
        for (int q = 0; q < (r >> 5); ++q) rank += __popc(mask[e * kRouteWords + q]);
        rank += __popc(mask[e * kRouteWords + (r >> 5)] & ((1u << (r & 31)) - 1u));
      }
      p.slot[at] = rank;
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
  for (int e = tid; e < p.E; e += kRouteThreads)
    p.counts[static_cast<long long>(blockIdx.x) * p.E + e] = count[e];
}

// Adds up the counts: an expert's first slot, and within it this CTA's; then turns
// the ranks into slots.  One CTA per choosing CTA, over the same tokens.
__global__ void __launch_bounds__(kRouteThreads) sc_route_place_kernel(
    const __grid_constant__ RouteParams p) {
  __shared__ int base[kMaxExperts], all[kMaxExperts];
  __shared__ int total;
  const int tid = threadIdx.x;
  pdl_wait();
  pdl_launch_dependents();
  if (tid < p.E) {
    int before = 0, sum = 0;
    for (unsigned c = 0; c < gridDim.x; ++c) {
      const int v = __ldcg(p.counts + static_cast<long long>(c) * p.E + tid);
      if (c < blockIdx.x) before += v;
      sum += v;
    }
    base[tid] = before;
    all[tid] = sum;
  }
  __syncthreads();
  if (tid == 0) {
    int run = 0;
    for (int e = 0; e < p.E; ++e) {
      base[e] += run;
      if (blockIdx.x == 0) p.offsets[e] = run;
      run += all[e];
    }
    if (blockIdx.x == 0) p.offsets[p.E] = run;
    total = run;
  }
  __syncthreads();
  const long long i0 = static_cast<long long>(blockIdx.x) * p.per_cta * p.k;
  const long long i1 = min(i0 + static_cast<long long>(p.per_cta) * p.k, p.T * p.k);
  for (long long i = i0 + tid; i < i1; i += kRouteThreads) {
    const int e = p.expert[i];
    if (e >= 0) {
      const int s = base[e] + p.slot[i];
      p.slot[i] = s;
      p.token[s] = static_cast<int>(i / p.k);
    }
    if (i >= total) p.token[i] = -1;
  }
}

// d logits of the gates.  With inner = sum_j g_j dg_j: at a chosen expert
// g_j (dg_j - inner) and 0 elsewhere (renormalize), or p_e ([e chosen] dg_e - inner)
// with p the softmax over all E.  A token without a choice has gradient 0.
template <int V>
__global__ void __launch_bounds__(kRouteThreads) sc_route_back_kernel(
    const __grid_constant__ RouteBackParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long t = static_cast<long long>(blockIdx.x) * (kRouteThreads / 32) + (threadIdx.x >> 5);
  if (t >= p.T) return;
  const bool in = token_in_use(p.rows, p.L, t);
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

int route_ctas(long long T, int* per_cta) {
  const long long chunks = (T + kRouteTokens - 1) / kRouteTokens;
  const long long each = (chunks + kRouteMaxCtas - 1) / kRouteMaxCtas;
  *per_cta = static_cast<int>(each * kRouteTokens);
  return static_cast<int>((chunks + each - 1) / each);
}

cudaError_t launch_route(const RouteParams& in, cudaStream_t st) {
  RouteParams p = in;
  const int ctas = route_ctas(p.T, &p.per_cta);
  const size_t smem = static_cast<size_t>(p.E) * (kRouteWords + 1) * 4;
  auto choose = p.E <= 32 ? sc_route_choose_kernel<1>
                : p.E <= 64 ? sc_route_choose_kernel<2>
                : p.E <= 128 ? sc_route_choose_kernel<4> : sc_route_choose_kernel<8>;
  const cudaError_t e = launch_chained(choose, dim3(ctas), dim3(kRouteThreads), smem, st, p);
  if (e != cudaSuccess) return e;
  return launch_chained(sc_route_place_kernel, dim3(ctas), dim3(kRouteThreads), 0, st, p);
}

cudaError_t launch_route_back(const RouteBackParams& p, cudaStream_t st) {
  constexpr int per = kRouteThreads / 32;
  const dim3 grid(static_cast<unsigned>((p.T + per - 1) / per));
  auto k = p.E <= 32 ? sc_route_back_kernel<1>
           : p.E <= 64 ? sc_route_back_kernel<2>
           : p.E <= 128 ? sc_route_back_kernel<4> : sc_route_back_kernel<8>;
  return launch_chained(k, grid, dim3(kRouteThreads), 0, st, p);
}

}  // namespace sc
