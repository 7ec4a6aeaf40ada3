// sc_expert_linear.cu -- matrix products grouped by expert, ragged sizes known on
// the device alone.  Expert e has the slots offsets[e] .. offsets[e + 1]:
//   forward       out[s][n]   = act(sum_k x[row(s)][k] W_e[n][k] + b_e[n])
//   back (input)  out[s][k]   = (sum_n dy[s][n] W_e[n][k]) GELU'(pre[s][k])
//   back (weight) out[e][n][k] = sum_s dy[s][n] x[row(s)][k],  db_e[n] = sum_s dy[s][n]
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_expert.cuh"
#include "sm103_primitives.cuh"

namespace sc {

constexpr int kSimpleTile = 64, kSimpleDepth = 16, kSimpleThreads = 256;

__device__ __forceinline__ float bf(uint16_t v) {
  return __uint_as_float(static_cast<uint32_t>(v) << 16);
}

__device__ __forceinline__ float gelu_exact(float x) {
  return 0.5f * x * (1.f + erff(x * 0.70710678118654752f));
}
__device__ __forceinline__ float gelu_slope(float x) {
  return 0.5f * (1.f + erff(x * 0.70710678118654752f)) +
         x * expf(-0.5f * x * x) * 0.3989422804014327f;
}

// 64 x 64 outputs a CTA, 4 x 4 a thread, operands through shared memory in fp32.
template <ExpertProduct kWhat>
__global__ void __launch_bounds__(kSimpleThreads) sc_expert_simple_kernel(
    const __grid_constant__ ExpertLinearParams p) {
  __shared__ float as[kSimpleDepth][kSimpleTile + 1], bs[kSimpleDepth][kSimpleTile + 1];
  pdl_wait();
  pdl_launch_dependents();
  const int tid = threadIdx.x;
  int e = 0, lo = 0, hi = 0, i0, ni;
  const int j0 = blockIdx.x * kSimpleTile, nj = kWhat == ExpertProduct::kForward ? p.N : p.K;
  if constexpr (kWhat == ExpertProduct::kBackWeight) {
    e = blockIdx.z;
    expert_range(p, e, lo, hi);
    i0 = blockIdx.y * kSimpleTile;
    ni = p.N;
  } else {
    int t = blockIdx.y;
    for (;; ++e) {
      if (e == p.E) return;
      expert_range(p, e, lo, hi);
      const int tiles = (hi - lo + kSimpleTile - 1) / kSimpleTile;
      if (t < tiles) break;
      t -= tiles;
    }
    i0 = t * kSimpleTile;
    ni = hi - lo;
  }
  const uint16_t* w = p.w + static_cast<long long>(e) * p.N * p.K;
  const int depth = kWhat == ExpertProduct::kForward ? p.K
                    : kWhat == ExpertProduct::kBackInput ? p.N : hi - lo;
  float acc[4][4] = {};
  float rows = 0.f;   // kBackWeight: the sum over the slots of row i0 + tid of dy^T
  for (int d0 = 0; d0 < depth; d0 += kSimpleDepth) {
    for (int q = tid; q < kSimpleTile * kSimpleDepth; q += kSimpleThreads) {
      // i and j of the operands along the unit stride of their memory
      int d, i;
      if constexpr (kWhat == ExpertProduct::kBackWeight) i = q % kSimpleTile, d = q / kSimpleTile;
      else d = q % kSimpleDepth, i = q / kSimpleDepth;
      float a = 0.f, b = 0.f;
      if (d0 + d < depth && i0 + i < ni) {
        if constexpr (kWhat == ExpertProduct::kForward)
          a = bf(p.x[static_cast<long long>(expert_row(p, lo + i0 + i)) * p.ldx + d0 + d]);
        else if constexpr (kWhat == ExpertProduct::kBackInput)
          a = bf(p.dy[static_cast<long long>(lo + i0 + i) * p.ldy + d0 + d]);
        else
          a = bf(p.dy[static_cast<long long>(lo + d0 + d) * p.ldy + i0 + i]);
      }
      as[d][i] = a;
      if constexpr (kWhat == ExpertProduct::kBackInput) i = q % kSimpleTile, d = q / kSimpleTile;
      if (d0 + d < depth && j0 + i < nj) {
        if constexpr (kWhat == ExpertProduct::kForward)
          b = bf(w[static_cast<long long>(j0 + i) * p.K + d0 + d]);
        else if constexpr (kWhat == ExpertProduct::kBackInput)
          b = bf(w[static_cast<long long>(d0 + d) * p.K + j0 + i]);
        else
          b = bf(p.x[static_cast<long long>(expert_row(p, lo + d0 + d)) * p.ldx + j0 + i]);
      }
      bs[d][i] = b;
    }
    __syncthreads();
#pragma unroll
    for (int d = 0; d < kSimpleDepth; ++d) {
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v)
          acc[u][v] = fmaf(as[d][(tid / 16) + 16 * u], bs[d][(tid % 16) + 16 * v], acc[u][v]);
      if (kWhat == ExpertProduct::kBackWeight && tid < kSimpleTile) rows += as[d][tid];
    }
    __syncthreads();
  }
  if constexpr (kWhat == ExpertProduct::kBackWeight) {
    if (p.dbias != nullptr && blockIdx.x == 0 && tid < kSimpleTile && i0 + tid < ni)
      p.dbias[static_cast<long long>(e) * p.N + i0 + tid] = rows;
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int i = i0 + tid / 16 + 16 * u, j = j0 + tid % 16 + 16 * v;
      if (i >= ni || j >= nj) continue;
      float y = acc[u][v];
      long long at;
      if constexpr (kWhat == ExpertProduct::kForward) {
        at = static_cast<long long>(lo + i) * p.N + j;
        if (p.bias != nullptr) y += p.bias[static_cast<long long>(e) * p.N + j];
        if (p.pre != nullptr) p.pre[at] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
        if (p.gelu) y = gelu_exact(y);
      } else if constexpr (kWhat == ExpertProduct::kBackInput) {
        at = static_cast<long long>(lo + i) * p.K + j;
        if (p.pre_in != nullptr) y *= gelu_slope(bf(p.pre_in[at]));
      } else {
        at = (static_cast<long long>(e) * p.N + i) * p.K + j;
      }
      if (p.out_f32) static_cast<float*>(p.out)[at] = y;
      else static_cast<uint16_t*>(p.out)[at] = __bfloat16_as_ushort(__float2bfloat16_rn(y));
    }
}

cudaError_t launch_expert_linear(ExpertProduct what, const ExpertLinearParams& p, cudaStream_t st) {
  const auto tiles = [](int n) { return static_cast<unsigned>((n + kSimpleTile - 1) / kSimpleTile); };
  if (what == ExpertProduct::kBackWeight)
    return launch_chained(sc_expert_simple_kernel<ExpertProduct::kBackWeight>,
                          dim3(tiles(p.K), tiles(p.N), p.E), dim3(kSimpleThreads), 0, st, p);
  // no more tiles than full ones and one begun for each expert
  const unsigned rows = static_cast<unsigned>(p.M / kSimpleTile + (p.E < p.M ? p.E : p.M));
  if (what == ExpertProduct::kForward)
    return launch_chained(sc_expert_simple_kernel<ExpertProduct::kForward>, dim3(tiles(p.N), rows),
                          dim3(kSimpleThreads), 0, st, p);
  return launch_chained(sc_expert_simple_kernel<ExpertProduct::kBackInput>, dim3(tiles(p.K), rows),
                        dim3(kSimpleThreads), 0, st, p);
}

cudaError_t configure_combine();

cudaError_t configure_expert() { return configure_combine(); }

}  // namespace sc
