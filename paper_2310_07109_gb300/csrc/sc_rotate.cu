// sc_rotate.cu -- norm and rotation of query and key heads in one pass, its gradient,
// and the same pass with keys and values going into a cache.
//
// For a head x of d features, a token at position p:
//   y = x rsqrt(mean x^2 + eps) gamma;   (y_i, y_i') -> m (y_i cos a - y_i' sin a, y_i' cos a + y_i sin a)
//   with a = p f for each pair.  Backward: the rotation's transpose gives dy, then
//   h = x rsqrt(..);  dx = rsqrt(..) (dy gamma - h mean(dy gamma h));  dgamma = sum dy h.
//
// Angles: a pair's frequency is kept as the fraction of a turn that one position adds, in
// units of 2^-64.  An integer product with the position wraps at whole turns by itself, so
// its top 32 bits are the angle, whatever the position (an fp32 product is off by 0.06 rad at
// position 10^6).
//
// Bound by memory: each value is read once and written once.  A lane has the two 16-byte vectors
// of a head that hold both members of its eight pairs, so rotating takes no exchange between
// lanes and a norm's sum is a few shuffles; a warp has 32 / W heads of a token at once and
// loads kBatch such groups before it works on the first.  A token's angles are computed once for all
// its heads, one pair a lane, and passed on through shared memory.
#include <cuda_runtime.h>
#include <algorithm>
#include <cstdint>

#include "sc_cache.cuh"
#include "sc_expert.cuh"
#include "sc_internal.cuh"

namespace sc {

constexpr int kRotateWarps = 8;
constexpr int kRotateThreads = kRotateWarps * 32;
constexpr int kMaxPairs = SC_MAX_HEAD_WIDTH / 2;
constexpr int kPairsLane = kMaxPairs / 32;

struct RotateSmem {
  float2 turn[kRotateWarps][kMaxPairs];        // m cos, m sin of the warp's token
  float gamma[2][SC_MAX_HEAD_WIDTH];
};

// The fraction of a turn that one position adds, in 2^-64.
__device__ __forceinline__ uint64_t turn_of(double freq) {
  double t = freq * 0.15915494309189533577;   // 1 / (2 pi)
  t -= floor(t);
  return __double2ull_rn(t * 18446744073709551616.0);
}

// cos and sin of `pos` times that fraction.
__device__ __forceinline__ float2 turned(uint64_t turn, int pos, float m) {
  const uint64_t at = turn * static_cast<uint64_t>(static_cast<int64_t>(pos));
  const int top = static_cast<int>((at + 0x80000000ull) >> 32);   // of half a turn, in 2^-31
  float s, c;
  sincospif(static_cast<float>(top) * 4.656612873077393e-10f, &s, &c);
  return make_float2(m * c, m * s);
}

template <class T>
__device__ __forceinline__ void unpack16(const uint4& a, const uint4& b, float (&x)[16]) {
  T::unpack(a.x, x[0], x[1]);
  T::unpack(a.y, x[2], x[3]);
  T::unpack(a.z, x[4], x[5]);
  T::unpack(a.w, x[6], x[7]);
  T::unpack(b.x, x[8], x[9]);
  T::unpack(b.y, x[10], x[11]);
  T::unpack(b.z, x[12], x[13]);
  T::unpack(b.w, x[14], x[15]);
}

template <class T>
__device__ __forceinline__ uint4 pack8(const float* x) {
  return make_uint4(T::pack(x[0], x[1]), T::pack(x[2], x[3]), T::pack(x[4], x[5]), T::pack(x[6], x[7]));
}

template <int W>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// What a lane has of every head: vectors va and vb, both members of pairs 8 q .. 8 q + 7.
struct LaneShare {
  int va, vb;
  bool live, turns, inter;
  __device__ LaneShare(const RotateParams& p, int q) {
    const int half = p.rot / 16;
    live = q < p.d / 16;
    turns = live && q < half;
    inter = p.interleaved != 0;
    const bool apart = turns && !inter;
    va = apart ? q : 2 * q;
    vb = apart ? q + half : 2 * q + 1;
  }
};

// A token's angles into the warp's table.
__device__ __forceinline__ void table(const RotateParams& p, const uint64_t (&turn)[kPairsLane], int pos,
                                      float2* to, int lane) {
  __syncwarp();
#pragma unroll
  for (int i = 0; i < kPairsLane; ++i)
    if (i * 32 + lane < p.rot / 2) to[i * 32 + lane] = turned(turn[i], pos, p.mscale);
  __syncwarp();
}

// Rotates the pairs of x, which hold (a, b) as x[i], x[8 + i], or as x[2 i], x[2 i + 1].
template <bool kBack>
__device__ __forceinline__ void rotate16(float (&x)[16], const LaneShare& s, const float2* turn) {
  if (!s.turns) return;
  const float4* t4 = reinterpret_cast<const float4*>(turn);
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    const float4 f = t4[i / 2];
    const float2 cs[2] = {make_float2(f.x, kBack ? -f.y : f.y), make_float2(f.z, kBack ? -f.w : f.w)};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int k = i + j;
      if (s.inter) {
        const float a = x[2 * k], b = x[2 * k + 1];
        x[2 * k] = a * cs[j].x - b * cs[j].y;
        x[2 * k + 1] = b * cs[j].x + a * cs[j].y;
      } else {
        const float a = x[k], b = x[8 + k];
        x[k] = a * cs[j].x - b * cs[j].y;
        x[8 + k] = b * cs[j].x + a * cs[j].y;
      }
    }
  }
}

__device__ __forceinline__ void gamma16(const float* gamma, const LaneShare& s, float (&g)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 a = reinterpret_cast<const float4*>(gamma)[2 * s.va + i];
    const float4 b = reinterpret_cast<const float4*>(gamma)[2 * s.vb + i];
    g[4 * i] = a.x; g[4 * i + 1] = a.y; g[4 * i + 2] = a.z; g[4 * i + 3] = a.w;
    g[8 + 4 * i] = b.x; g[8 + 4 * i + 1] = b.y; g[8 + 4 * i + 2] = b.z; g[8 + 4 * i + 3] = b.w;
  }
}

__device__ __forceinline__ void load_gamma(const RotateParams& p, RotateSmem& sm) {
  for (int i = threadIdx.x; i < p.d; i += kRotateThreads) {
    sm.gamma[0][i] = p.gamma_q != nullptr ? __ldg(p.gamma_q + i) : 0.f;
    sm.gamma[1][i] = p.gamma_k != nullptr ? __ldg(p.gamma_k + i) : 0.f;
  }
}

__device__ __forceinline__ int cache_len(const RotateParams& p, int list) {
  return min(max(__ldcg(p.len + list), 0), p.C);
}

// Forward, and append where cache_k is set.  A warp's work: the groups of heads `part`, part + parts, ...
// of a token; with few tokens several warps share one.
template <class T, int W>
__global__ void __launch_bounds__(kRotateThreads) rotate_kernel(const RotateParams p, int parts) {
  constexpr int kAtOnce = 32 / W;   // heads of a group
  constexpr int kBatch = 4;         // groups whose loads are under way together
  __shared__ RotateSmem sm;
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int q = lane & (W - 1), sub = lane / W;
  const LaneShare share(p, q);
  const bool append = p.cache_k != nullptr;
  const int gq = (p.Hq + kAtOnce - 1) / kAtOnce, gk = (p.Hk + kAtOnce - 1) / kAtOnce;
  const int groups = gq + gk + (append ? gk : 0);
  uint64_t turn[kPairsLane];
#pragma unroll
  for (int i = 0; i < kPairsLane; ++i)
    turn[i] = i * 32 + lane < p.rot / 2 ? turn_of(__ldg(p.freq + i * 32 + lane)) : 0;
  load_gamma(p, sm);
  __syncthreads();
  const unsigned L = static_cast<unsigned>(p.L);
  const long long items = p.T * parts, step = static_cast<long long>(gridDim.x) * kRotateWarps;
  for (long long it = static_cast<long long>(blockIdx.x) * kRotateWarps + warp; it < items; it += step) {
    const unsigned t = static_cast<unsigned>(it / parts);
    const int part = static_cast<int>(it - static_cast<long long>(t) * parts);
    const int b = static_cast<int>(t / L), r = static_cast<int>(t - b * L);
    if (p.rows != nullptr && r >= __ldg(p.rows + b)) continue;
    const int pos = append ? __ldcg(p.seen + b) + r : p.pos != nullptr ? __ldg(p.pos + t) : r;
    table(p, turn, pos, sm.turn[warp], lane);
    for (int g0 = part; g0 < groups; g0 += parts * kBatch) {
      uint4 va[kBatch], vb[kBatch];
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int g = g0 + u * parts;
        const int side = g < gq ? 0 : g < gq + gk ? 1 : 2;
        const int head = (g - (side == 0 ? 0 : side == 1 ? gq : gq + gk)) * kAtOnce + sub;
        const HeadsIn in = side == 0 ? p.q : side == 1 ? p.k : p.v;
        va[u] = vb[u] = make_uint4(0, 0, 0, 0);
        if (g < groups && share.live && head < (side == 0 ? p.Hq : p.Hk)) {
          const uint4* src = reinterpret_cast<const uint4*>(in.p + t * in.ld + static_cast<long long>(head) * p.d);
          va[u] = src[share.va];
          vb[u] = src[share.vb];
        }
      }
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        const int g = g0 + u * parts;
        if (g >= groups) break;
        const int side = g < gq ? 0 : g < gq + gk ? 1 : 2;
        const int head = (g - (side == 0 ? 0 : side == 1 ? gq : gq + gk)) * kAtOnce + sub;
        const bool live = share.live && head < (side == 0 ? p.Hq : p.Hk);
        if (side < 2) {
          float x[16];
          unpack16<T>(va[u], vb[u], x);
          if ((side == 0 ? p.gamma_q : p.gamma_k) != nullptr) {
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
            const float inv = rsqrtf(sum_lanes<W>(ss) / static_cast<float>(p.d) + p.eps);
            if (share.live) {
              float gm[16];
              gamma16(sm.gamma[side], share, gm);
#pragma unroll
              for (int i = 0; i < 16; ++i) x[i] *= inv * gm[i];
            }
          }
          rotate16<false>(x, share, sm.turn[warp] + 8 * q);
          va[u] = pack8<T>(x);
          vb[u] = pack8<T>(x + 8);
        }
        if (!live) continue;
        uint16_t* to;
        if (side == 0) {
          to = p.q_out.p + t * p.q_out.ld + static_cast<long long>(head) * p.d;
        } else if (!append) {
          to = p.k_out.p + t * p.k_out.ld + static_cast<long long>(head) * p.d;
        } else {
          const int of = p.Hk / p.G, list = b * p.G + head / of;
          const int slot = cache_len(p, list) + r;
          if (slot >= p.C) continue;
          to = (side == 1 ? p.cache_k : p.cache_v) + b * p.stride_b + head * p.stride_h + slot * p.stride_c;
          if (side == 1 && q == 0 && head % of == 0) {
            p.acc[static_cast<long long>(list) * p.C + slot] = 0.f;
            p.slot_pos[static_cast<long long>(list) * p.C + slot] = pos;
          }
        }
        reinterpret_cast<uint4*>(to)[share.va] = va[u];
        reinterpret_cast<uint4*>(to)[share.vb] = vb[u];
      }
    }
  }
  if (!append) return;
  // The last CTA to be done with len and seen moves them on.
  __shared__ bool last;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicInc(p.done, gridDim.x - 1) == gridDim.x - 1;   // back to 0 after the last
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  for (int i = threadIdx.x; i < p.B * p.G; i += kRotateThreads) {
    const int b = i / p.G;
    const int come = p.rows != nullptr ? min(max(__ldg(p.rows + b), 0), p.L) : p.L;
    const long long n = static_cast<long long>(cache_len(p, i)) + come;
    if (n > p.C) atomicOr(p.status, kStatusFull);
    p.len_out[i] = static_cast<int>(min(n, static_cast<long long>(p.C)));
  }
  for (int b = threadIdx.x; b < p.B; b += kRotateThreads)
    p.seen_out[b] = __ldcg(p.seen + b) + (p.rows != nullptr ? min(max(__ldg(p.rows + b), 0), p.L) : p.L);
}

// Gradient.  dgamma: a lane adds up its features over its heads and tokens, the CTA its lanes, in order;
// the parts of the CTAs are added, in order, by rotate_gamma_kernel.
template <class T, int W>
__global__ void __launch_bounds__(kRotateThreads, 2) rotate_back_kernel(const RotateParams p) {
  constexpr int kAtOnce = 32 / W;
  constexpr int kBatch = 2;
  __shared__ RotateSmem sm;
  __shared__ float sums[kRotateWarps][SC_MAX_HEAD_WIDTH];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int q = lane & (W - 1), sub = lane / W;
  const LaneShare share(p, q);
  uint64_t turn[kPairsLane];
#pragma unroll
  for (int i = 0; i < kPairsLane; ++i)
    turn[i] = i * 32 + lane < p.rot / 2 ? turn_of(__ldg(p.freq + i * 32 + lane)) : 0;
  load_gamma(p, sm);
  __syncthreads();
  float total[2][16];
#pragma unroll
  for (int i = 0; i < 16; ++i) total[0][i] = total[1][i] = 0.f;
  const unsigned L = static_cast<unsigned>(p.L);
  const long long step = static_cast<long long>(gridDim.x) * kRotateWarps;
  const float over_d = 1.f / static_cast<float>(p.d);
  for (long long it = static_cast<long long>(blockIdx.x) * kRotateWarps + warp; it < p.T; it += step) {
    const unsigned t = static_cast<unsigned>(it);
    const int b = static_cast<int>(t / L), r = static_cast<int>(t - b * L);
    if (p.rows != nullptr && r >= __ldg(p.rows + b)) continue;
    table(p, turn, p.pos != nullptr ? __ldg(p.pos + t) : r, sm.turn[warp], lane);
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const int heads = side == 0 ? p.Hq : p.Hk;
      const bool norm = (side == 0 ? p.gamma_q : p.gamma_k) != nullptr;
      const HeadsIn dy = side == 0 ? p.dq : p.dk, in = side == 0 ? p.q : p.k;
      const HeadsOut out = side == 0 ? p.q_out : p.k_out;
      for (int h0 = 0; h0 < heads; h0 += kBatch * kAtOnce) {
        uint4 va[kBatch], vb[kBatch], xa[kBatch], xb[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int head = h0 + u * kAtOnce + sub;
          va[u] = vb[u] = xa[u] = xb[u] = make_uint4(0, 0, 0, 0);
          if (!share.live || head >= heads) continue;
          const uint4* src = reinterpret_cast<const uint4*>(dy.p + t * dy.ld + static_cast<long long>(head) * p.d);
          va[u] = src[share.va];
          vb[u] = src[share.vb];
          if (!norm) continue;
          src = reinterpret_cast<const uint4*>(in.p + t * in.ld + static_cast<long long>(head) * p.d);
          xa[u] = src[share.va];
          xb[u] = src[share.vb];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
          const int head = h0 + u * kAtOnce + sub;
          float g[16];
          unpack16<T>(va[u], vb[u], g);
          rotate16<true>(g, share, sm.turn[warp] + 8 * q);
          if (norm) {
            float x[16], gm[16];
            unpack16<T>(xa[u], xb[u], x);
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) ss += x[i] * x[i];
            const float inv = rsqrtf(sum_lanes<W>(ss) * over_d + p.eps);
            gamma16(sm.gamma[side], share.live ? share : LaneShare(p, 0), gm);
            float inner = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              x[i] *= inv;
              total[side][i] += g[i] * x[i];
              g[i] *= gm[i];
              inner += g[i] * x[i];
            }
            inner = sum_lanes<W>(inner) * over_d;
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = inv * (g[i] - x[i] * inner);
          }
          if (!share.live || head >= heads) continue;
          uint4* to = reinterpret_cast<uint4*>(out.p + t * out.ld + static_cast<long long>(head) * p.d);
          to[share.va] = pack8<T>(g);
          to[share.vb] = pack8<T>(g + 8);
        }
      }
    }
  }
  if (p.gamma_q == nullptr && p.gamma_k == nullptr) return;
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float v = total[side][i];
#pragma unroll
      for (int o = W; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (share.live && sub == 0) sums[warp][8 * (i < 8 ? share.va : share.vb) + (i & 7)] = v;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.d; i += kRotateThreads) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < kRotateWarps; ++w) v += sums[w][i];
      p.part[(static_cast<long long>(blockIdx.x) * 2 + side) * p.d + i] = v;
    }
    __syncthreads();
  }
}

// dgamma from the CTAs' parts: 32 features a CTA, eight warps with every eighth part each.
__global__ void __launch_bounds__(kRotateThreads) rotate_gamma_kernel(const RotateParams p, int ctas) {
  __shared__ float sums[kRotateWarps][32];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int i = blockIdx.x * 32 + lane;   // of [2][d]
  float v = 0.f;
  if (i < 2 * p.d)
    for (int c = warp; c < ctas; c += kRotateWarps) v += p.part[static_cast<long long>(c) * 2 * p.d + i];
  sums[warp][lane] = v;
  __syncthreads();
  if (warp != 0 || i >= 2 * p.d) return;
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kRotateWarps; ++w) v += sums[w][lane];
  float* to = i < p.d ? p.dgamma_q : p.dgamma_k;
  if (to != nullptr) to[i < p.d ? i : i - p.d] = v;
}

namespace {

int lanes_of(int d) {
  int w = 1;
  while (16 * w < d) w *= 2;
  return w;
}

template <class T, int W>
cudaError_t forward(const RotateParams& p, cudaStream_t st) {
  const int at_once = 32 / W;
  const int gq = (p.Hq + at_once - 1) / at_once, gk = (p.Hk + at_once - 1) / at_once;
  const int groups = gq + gk * (p.cache_k != nullptr ? 2 : 1);
  // few tokens: a warp for each group of heads, until the SMs have some warps each
  const long long want = static_cast<long long>(kCacheSms) * 32;
  int parts = 1;
  if (p.T < want) parts = static_cast<int>(std::min<long long>(groups, (want + p.T - 1) / p.T));
  const long long ctas = (p.T * parts + kRotateWarps - 1) / kRotateWarps;
  const dim3 grid(static_cast<unsigned>(std::min<long long>(ctas, kCacheSms * 6)));
  return launch_chained(rotate_kernel<T, W>, grid, dim3(kRotateThreads), 0, st, p, parts);
}

template <class T, int W>
cudaError_t backward(const RotateParams& p, cudaStream_t st) {
  const int ctas = static_cast<int>(std::min<long long>((p.T + kRotateWarps - 1) / kRotateWarps, kRotateMaxParts));
  cudaError_t e = launch_chained(rotate_back_kernel<T, W>, dim3(ctas), dim3(kRotateThreads), 0, st, p);
  if (e != cudaSuccess || (p.gamma_q == nullptr && p.gamma_k == nullptr)) return e;
  return launch_chained(rotate_gamma_kernel, dim3((2 * p.d + 31) / 32), dim3(kRotateThreads), 0, st, p, ctas);
}

template <class T>
cudaError_t forward_of(const RotateParams& p, cudaStream_t st) {
  switch (lanes_of(p.d)) {
    case 1: return forward<T, 1>(p, st);
    case 2: return forward<T, 2>(p, st);
    case 4: return forward<T, 4>(p, st);
    case 8: return forward<T, 8>(p, st);
    default: return forward<T, 16>(p, st);
  }
}

template <class T>
cudaError_t backward_of(const RotateParams& p, cudaStream_t st) {
  switch (lanes_of(p.d)) {
    case 1: return backward<T, 1>(p, st);
    case 2: return backward<T, 2>(p, st);
    case 4: return backward<T, 4>(p, st);
    case 8: return backward<T, 8>(p, st);
    default: return backward<T, 16>(p, st);
  }
}

}  // namespace

cudaError_t launch_rotate(const RotateParams& p, int dtype, cudaStream_t st) {
  return dtype == SC_FP16 ? forward_of<Fp16>(p, st) : forward_of<Bf16>(p, st);
}

cudaError_t launch_rotate_back(const RotateParams& p, int dtype, cudaStream_t st) {
  return dtype == SC_FP16 ? backward_of<Fp16>(p, st) : backward_of<Bf16>(p, st);
}

}  // namespace sc
