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
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_expert.cuh"
#include "sm103_primitives.cuh"

namespace sc {

constexpr int kCombineThreads = 256;
constexpr int kCombineVecs = 4;   // 16-byte vectors of 8 features per thread: D <= 32 x threads of a row

__device__ __forceinline__ void unpack8(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                    pack_bf16x2(f[6], f[7]));
}

// Sums of two values over the kRow threads of a row (a warp, or the whole CTA).
template <int kRow>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* red) {
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) {
    a += __shfl_xor_sync(0xffffffffu, a, off);
    b += __shfl_xor_sync(0xffffffffu, b, off);
  }
  if constexpr (kRow > 32) {
    __syncthreads();   // the previous sum has been read
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < kRow / 32; ++w) {
      a += red[w].x;
      b += red[w].y;
    }
  }
  return make_float2(a, b);
}

__device__ __forceinline__ int clamp_slot(const CombineParams& p, int s) {
  return s >= 0 && s < p.M ? s : -1;
}

// S of row t, this thread's features (vector c + i kRow of 8).
template <int kRow>
__device__ __forceinline__ void combine_sum(const CombineParams& p, long long t, int c, int vecs,
                                            float (&s)[kCombineVecs][8]) {
#pragma unroll
  for (int i = 0; i < kCombineVecs; ++i) {
    const int at = c + i * kRow;
#pragma unroll
    for (int q = 0; q < 8; ++q) s[i][q] = 0.f;
    if (p.res != nullptr && at < vecs) {
      float f[8];
      unpack8(__ldg(reinterpret_cast<const uint4*>(p.res + t * p.D) + at), f);
#pragma unroll
      for (int q = 0; q < 8; ++q) s[i][q] = p.res_scale * f[q];
    }
  }
  for (int j = 0; j < p.k; ++j) {
    const int sl = clamp_slot(p, __ldg(p.slot + t * p.k + j));
    if (sl < 0) continue;
    const float g = p.gate ? __ldg(p.gate + t * p.k + j) : 1.f;
    const uint4* y = reinterpret_cast<const uint4*>(p.y + static_cast<long long>(sl) * p.D);
#pragma unroll
    for (int i = 0; i < kCombineVecs; ++i) {
      const int at = c + i * kRow;
      if (at >= vecs) continue;
      float f[8];
      unpack8(__ldg(y + at), f);
#pragma unroll
      for (int q = 0; q < 8; ++q) s[i][q] = fmaf(g, f[q], s[i][q]);
    }
  }
}

// Mean and 1 / sigma of a row (two passes over the registers).
template <int kRow>
__device__ __forceinline__ float2 row_moments(const CombineParams& p, int c, int vecs,
                                              const float (&s)[kCombineVecs][8], float2* red) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < kCombineVecs; ++i)
#pragma unroll
    for (int q = 0; q < 8; ++q) a += s[i][q];   // features past D are 0
  const float mean = row_sum2<kRow>(a, 0.f, red).x / static_cast<float>(p.D);
  float b = 0.f;
#pragma unroll
  for (int i = 0; i < kCombineVecs; ++i)
    if (c + i * kRow < vecs)
#pragma unroll
      for (int q = 0; q < 8; ++q) b += (s[i][q] - mean) * (s[i][q] - mean);
  const float var = row_sum2<kRow>(b, 0.f, red).x / static_cast<float>(p.D);
  return make_float2(mean, 1.f / sqrtf(var + p.eps));
}

__device__ __forceinline__ bool row_in_use(const CombineParams& p, long long t) {
  if (p.rows == nullptr) return true;
  const long long b = t / p.L;
  return t - b * p.L < __ldg(p.rows + b);
}

template <int kRow>
__global__ void __launch_bounds__(kCombineThreads) sc_combine_kernel(
    const __grid_constant__ CombineParams p) {
  __shared__ float2 red[kCombineThreads / 32];
  pdl_wait();
  pdl_launch_dependents();
  const int c = threadIdx.x % kRow;
  const long long t = static_cast<long long>(blockIdx.x) * (kCombineThreads / kRow) + threadIdx.x / kRow;
  if (t >= p.T || !row_in_use(p, t)) return;
  const int vecs = p.D / 8;
  float s[kCombineVecs][8];
  combine_sum<kRow>(p, t, c, vecs, s);
  if (p.sum != nullptr)
#pragma unroll
    for (int i = 0; i < kCombineVecs; ++i)
      if (c + i * kRow < vecs) reinterpret_cast<uint4*>(p.sum + t * p.D)[c + i * kRow] = pack8(s[i]);
  if (p.gamma == nullptr) return;
  const float2 m = row_moments<kRow>(p, c, vecs, s, red);
#pragma unroll
  for (int i = 0; i < kCombineVecs; ++i) {
    const int at = c + i * kRow;
    if (at >= vecs) continue;
    float o[8];
#pragma unroll
    for (int q = 0; q < 8; ++q)
      o[q] = (s[i][q] - m.x) * m.y * __ldg(p.gamma + 8 * at + q) + __ldg(p.beta + 8 * at + q);
    reinterpret_cast<uint4*>(p.out + t * p.D)[at] = pack8(o);
  }
}

template <int kRow>
__global__ void __launch_bounds__(kCombineThreads) sc_combine_back_kernel(
    const __grid_constant__ CombineParams p) {
  __shared__ float2 red[kCombineThreads / 32];
  extern __shared__ float part[];   // [rows of the CTA][2][D]
  pdl_wait();
  pdl_launch_dependents();
  constexpr int kRows = kCombineThreads / kRow;
  const int c = threadIdx.x % kRow, r = threadIdx.x / kRow;
  const int vecs = p.D / 8;
  float dgam[kCombineVecs][8] = {}, dbet[kCombineVecs][8] = {};
  for (long long t = static_cast<long long>(blockIdx.x) * kRows + r; t < p.T;
       t += static_cast<long long>(gridDim.x) * kRows) {
    if (!row_in_use(p, t)) {
      if (c < p.k && p.dgate) p.dgate[t * p.k + c] = 0.f;
      continue;
    }
    float ds[kCombineVecs][8];
#pragma unroll
    for (int i = 0; i < kCombineVecs; ++i)
#pragma unroll
      for (int q = 0; q < 8; ++q) ds[i][q] = 0.f;
    if (p.dout != nullptr) {
      float s[kCombineVecs][8];
      combine_sum<kRow>(p, t, c, vecs, s);
      const float2 m = row_moments<kRow>(p, c, vecs, s, red);
      float a = 0.f, b = 0.f;
#pragma unroll
      for (int i = 0; i < kCombineVecs; ++i) {
        const int at = c + i * kRow;
        if (at >= vecs) continue;
        unpack8(__ldg(reinterpret_cast<const uint4*>(p.dout + t * p.D) + at), ds[i]);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          s[i][q] = (s[i][q] - m.x) * m.y;
          dgam[i][q] += ds[i][q] * s[i][q];
          dbet[i][q] += ds[i][q];
          ds[i][q] *= __ldg(p.gamma + 8 * at + q);
          a += ds[i][q];
          b += ds[i][q] * s[i][q];
        }
      }
      const float2 ab = row_sum2<kRow>(a, b, red);
      const float ma = ab.x / static_cast<float>(p.D), mb = ab.y / static_cast<float>(p.D);
#pragma unroll
      for (int i = 0; i < kCombineVecs; ++i)
#pragma unroll
        for (int q = 0; q < 8; ++q) ds[i][q] = m.y * (ds[i][q] - ma - s[i][q] * mb);
    }
#pragma unroll
    for (int i = 0; i < kCombineVecs; ++i) {
      const int at = c + i * kRow;
      if (at >= vecs) continue;
      if (p.dsum != nullptr) {
        float f[8];
        unpack8(__ldg(reinterpret_cast<const uint4*>(p.dsum + t * p.D) + at), f);
#pragma unroll
        for (int q = 0; q < 8; ++q) ds[i][q] += f[q];
      }
      if (p.dres != nullptr) {
        float f[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = p.res_scale * ds[i][q];
        reinterpret_cast<uint4*>(p.dres + t * p.D)[at] = pack8(f);
      }
    }
    for (int j = 0; j < p.k; ++j) {
      const int sl = clamp_slot(p, __ldg(p.slot + t * p.k + j));
      if (sl < 0) {
        if (c == 0 && p.dgate) p.dgate[t * p.k + j] = 0.f;
        continue;
      }
      const float g = p.gate ? __ldg(p.gate + t * p.k + j) : 1.f;
      const uint4* y = reinterpret_cast<const uint4*>(p.y + static_cast<long long>(sl) * p.D);
      uint4* dy = reinterpret_cast<uint4*>(p.dy + static_cast<long long>(sl) * p.D);
      float dot = 0.f;
#pragma unroll
      for (int i = 0; i < kCombineVecs; ++i) {
        const int at = c + i * kRow;
        if (at >= vecs) continue;
        float f[8], o[8];
        if (p.dgate) {
          unpack8(__ldg(y + at), f);
#pragma unroll
          for (int q = 0; q < 8; ++q) dot = fmaf(ds[i][q], f[q], dot);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = g * ds[i][q];
        dy[at] = pack8(o);
      }
      if (p.dgate) {
        dot = row_sum2<kRow>(dot, 0.f, red).x;
        if (c == 0) p.dgate[t * p.k + j] = dot;
      }
    }
  }
  if (p.dgamma == nullptr) return;
  // the CTA's rows, in order, into its part of the workspace
#pragma unroll
  for (int i = 0; i < kCombineVecs; ++i) {
    const int at = c + i * kRow;
    if (at >= vecs) continue;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      part[(r * 2) * p.D + 8 * at + q] = dgam[i][q];
      part[(r * 2 + 1) * p.D + 8 * at + q] = dbet[i][q];
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 2 * p.D; i += kCombineThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kRows; ++w) v += part[w * 2 * p.D + i];
    p.part[static_cast<long long>(blockIdx.x) * 2 * p.D + i] = v;
  }
}

// dgamma and dbeta: the CTAs' parts in order.  32 features a CTA, its eight warps take
// every eighth part.
__global__ void __launch_bounds__(256) sc_combine_reduce_kernel(
    const __grid_constant__ CombineParams p, int parts) {
  __shared__ float red[8][32];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int f = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (f < 2 * p.D)
    for (int c = w; c < parts; c += 8) v += __ldcg(p.part + static_cast<long long>(c) * 2 * p.D + f);
  red[w][lane] = v;
  __syncthreads();
  if (w != 0 || f >= 2 * p.D) return;
  for (int i = 1; i < 8; ++i) v += red[i][lane];
  if (f < p.D) p.dgamma[f] = v;
  else p.dbeta[f - p.D] = v;
}

static bool row_per_warp(const CombineParams& p) { return p.D <= 32 * 8 * kCombineVecs; }

cudaError_t launch_combine(const CombineParams& p, cudaStream_t st) {
  const int per = row_per_warp(p) ? kCombineThreads / 32 : 1;
  const dim3 grid(static_cast<unsigned>((p.T + per - 1) / per));
  return launch_chained(row_per_warp(p) ? sc_combine_kernel<32> : sc_combine_kernel<kCombineThreads>,
                        grid, dim3(kCombineThreads), 0, st, p);
}

cudaError_t launch_combine_back(const CombineParams& p, cudaStream_t st) {
  const int per = row_per_warp(p) ? kCombineThreads / 32 : 1;
  const long long want = (p.T + per - 1) / per;
  const int ctas = static_cast<int>(want < kCombineMaxCtas ? want : kCombineMaxCtas);
  const size_t smem = p.dgamma ? sizeof(float) * 2 * p.D * per : 0;
  cudaError_t e = launch_chained(
      row_per_warp(p) ? sc_combine_back_kernel<32> : sc_combine_back_kernel<kCombineThreads>,
      dim3(ctas), dim3(kCombineThreads), smem, st, p);
  if (e != cudaSuccess || p.dgamma == nullptr) return e;
  return launch_chained(sc_combine_reduce_kernel, dim3((2 * p.D + 31) / 32), dim3(256), 0, st, p, ctas);
}

cudaError_t configure_combine() {
  const cudaError_t e = cudaFuncSetAttribute(sc_combine_back_kernel<32>,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(sc_combine_back_kernel<kCombineThreads>,
                              cudaFuncAttributeMaxDynamicSharedMemorySize, 65536);
}

}  // namespace sc
