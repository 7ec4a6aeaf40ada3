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
// position 10^6).  Sine and cosine of it are the hardware's, within 2^-21.
//
// Each value is read once and written once, but a group of heads takes so few bytes that the instructions
// it takes count as much.  So all that does not change from token to token is settled before the loop: the
// heads of a token (queries, keys and, in an append, values) are one list, a warp has one group of 32 / W of
// them for all its tokens, and a lane two 16-byte vectors of a head, which hold both members of its eight
// pairs (no exchange between lanes but a norm's sum) and lie where its neighbours' do (every request has whole
// sectors).  The warps of a CTA have the groups of the same few tokens, whose angles they compute together, one for
// each pair, whatever the number of heads.  Each thread copies its own vectors of the next tokens into shared memory of
// its own (cp.async) while it works on these ones, side by side where all of a warp's are in use; the arithmetic runs
// on fp32 pairs.  16384 tokens of 20 heads of 128: 29 us (168 MB, 5.8 TB/s), gradient with norms 48 us (252 MB); 6500 tokens of
// 24 heads of 64: 13 us (40 MB), 22 with a warp a token, which settles all that for each group anew.
#include <algorithm>
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_cache.cuh"
#include "sc_expert.cuh"
#include "sc_internal.cuh"

namespace sc {

constexpr int kRotateWarps = 8;         // most of a CTA
constexpr int kRotateThreads = kRotateWarps * 32;
constexpr int kSmWarps = 16;            // an SM's: 128 registers a thread (what spills with 80 costs half of the time again)
constexpr int kWarpTokens = 4;          // most tokens of a warp at a time, forward
constexpr int kWarpTokensBack = 2;      // backward (twice the vectors)
constexpr int kTileTokens = 16;         // most tokens of a CTA at a time

// How the work is cut: `wg` warps side by side for groups, `wt` for tokens, each `nt` tokens at a time.
struct RotatePlan {
  int wg, wt, nt, ctas;
};

// The fraction of a turn that one position adds, freq / (2 pi), in 2^-64: the 53-bit significand times
// 2^66 / (2 pi) as a 117-bit product, shifted by the exponent (fp64 arithmetic would take longer than all else).
__device__ __forceinline__ unsigned long long turn_of(double freq) {
  const unsigned long long bits = static_cast<unsigned long long>(__double_as_longlong(freq));
  const unsigned long long m = (bits & 0xfffffffffffffull) | 0x10000000000000ull, c = 11743562013128004906ull;
  const unsigned long long hi = __umul64hi(m, c), lo = m * c;
  const int right = 54 + 1023 - static_cast<int>(bits >> 52 & 2047u);   // of the product, for freq = m 2^(e - 52)
  unsigned long long t;
  if (right >= 128) t = 0;
  else if (right >= 64) t = hi >> (right - 64);
  else if (right > 0) t = hi << (64 - right) | lo >> right;
  else t = right > -64 ? lo << -right : 0;
  return bits >> 63 ? 0 - t : t;
}

// First and second members of a lane's pairs as fp32 pairs, and back: the two vectors (kInter false), or
// the even and the odd values of both.
template <class T, bool kInter>
__device__ __forceinline__ void unpack(const uint4& va, const uint4& vb, uint64_t (&a)[4], uint64_t (&b)[4]) {
  const uint32_t w[8] = {va.x, va.y, va.z, va.w, vb.x, vb.y, vb.z, vb.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x0, y0, x1, y1;
    if (kInter) {
      T::unpack(w[2 * i], x0, y0);
      T::unpack(w[2 * i + 1], x1, y1);
    } else {
      T::unpack(w[i], x0, x1);
      T::unpack(w[4 + i], y0, y1);
    }
    a[i] = f2_pack(x0, x1);
    b[i] = f2_pack(y0, y1);
  }
}

template <class T, bool kInter>
__device__ __forceinline__ void pack(const uint64_t (&a)[4], const uint64_t (&b)[4], uint4& va, uint4& vb) {
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x0, x1, y0, y1;
    f2_unpack(a[i], x0, x1);
    f2_unpack(b[i], y0, y1);
    w[kInter ? 2 * i : i] = kInter ? T::pack(x0, y0) : T::pack(x0, x1);
    w[kInter ? 2 * i + 1 : 4 + i] = kInter ? T::pack(x1, y1) : T::pack(y0, y1);
  }
  va = make_uint4(w[0], w[1], w[2], w[3]);
  vb = make_uint4(w[4], w[5], w[6], w[7]);
}

template <int W>
__device__ __forceinline__ float sum_lanes(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

__device__ __forceinline__ float f2_total(uint64_t v) {
  float lo, hi;
  f2_unpack(v, lo, hi);
  return lo + hi;
}

// The sum of squares of the lane's sixteen values, over the head's lanes.
template <int W>
__device__ __forceinline__ float squares(const uint64_t (&a)[4], const uint64_t (&b)[4]) {
  uint64_t s = f2_mul(a[0], a[0]), t = f2_mul(b[0], b[0]);
#pragma unroll
  for (int i = 1; i < 4; ++i) {
    s = f2_fma(a[i], a[i], s);
    t = f2_fma(b[i], b[i], t);
  }
  return sum_lanes<W>(f2_total(f2_add(s, t)));
}

// What a lane does for every token.
struct LaneShare {
  int group, sub, q;   // its warp's group; head of the group and lane of the head
  int head;            // of the list of queries, keys and values; one that there is
  int side, of_side;   // 0 queries, 1 keys, 2 values; the head's number among them
  int va, vb;          // its vectors of the head
  bool live;           // it has a part of a head
  bool turn_a, turn_b; // which is rotated: with the layout of halves all of it or nothing, else vector by vector
  __device__ __forceinline__ LaneShare(const RotateParams& p, const RotatePlan& plan, int w, bool inter, bool append) {
    const int lane = threadIdx.x & 31, at_once = 32 / w, turned = p.Hq + p.Hk, heads = turned + (append ? p.Hk : 0);
    group = blockIdx.y * plan.wg + (threadIdx.x >> 5) % plan.wg;
    q = lane % w;
    sub = lane / w;
    const int mine = group * at_once + sub;
    head = min(mine, heads - 1);
    side = head < p.Hq ? 0 : head < turned ? 1 : 2;
    of_side = head - (side == 0 ? 0 : side == 1 ? p.Hq : turned);
    const int lanes = p.d / 16, half = p.rot / 16;
    const bool in = q < lanes;
    live = in && mine < heads;
    // halves: vectors q and q + half, and for the rest of the head those behind; else q and q + lanes
    const bool apart = !inter && q < half;
    va = !in ? 0 : inter || apart ? q : q + half;   // (lanes beyond the head read its start)
    vb = !in ? 0 : apart ? q + half : q + lanes;
    turn_a = in && (inter ? va < 2 * half : apart);
    turn_b = in && (inter ? vb < 2 * half : apart);
  }
};

// (a, b) -> (a cos - b sin, b cos + a sin), or, backward, (a cos + b sin, b cos - a sin); row: the token's in the tables
template <bool kBack, bool kInter>
__device__ __forceinline__ void rotate(uint64_t (&a)[4], uint64_t (&b)[4], const float* cos, const float* sin, const LaneShare& s) {
  if (!s.turn_a && !s.turn_b) return;
  // pairs 8 q ..., or those of the two vectors
  const int first = kInter ? 4 * s.va : 8 * s.q, then = kInter ? (s.turn_b ? 4 * s.vb : first) : 8 * s.q + 4;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const ulonglong2 c2 = *reinterpret_cast<const ulonglong2*>(cos + (h == 0 ? first : then));
    const ulonglong2 s2 = *reinterpret_cast<const ulonglong2*>(sin + (h == 0 ? first : then));
    if (kInter && !(h == 0 ? s.turn_a : s.turn_b)) continue;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = 2 * h + k;
      const uint64_t c = k == 0 ? c2.x : c2.y, sn = k == 0 ? s2.x : s2.y;
      const uint64_t x = a[i], as = f2_mul(x, sn), bs = f2_mul(b[i], sn), minus = (kBack ? as : bs) ^ 0x8000000080000000ull;
      a[i] = f2_fma(x, c, kBack ? bs : minus);
      b[i] = f2_fma(b[i], c, kBack ? minus : as);
    }
  }
}

// Shared memory: the vectors of two tiles, [warp][tile][token][vector][lane], then two tables of angles.
__host__ __device__ inline size_t ring_bytes(const RotatePlan& plan, int vectors) {
  return static_cast<size_t>(plan.wg) * plan.wt * 2 * plan.nt * vectors * 32 * sizeof(uint4);
}

// The tile of tokens of a CTA: lane i has its token t0 + i's sequence, row, position, and whether it is in use.
struct TileTokens {
  int b, r, pos;
  unsigned used;   // of all lanes
  __device__ __forceinline__ TileTokens(const RotateParams& p, long long t0, int count, bool append) {
    const int lane = threadIdx.x & 31;
    const long long t = t0 + lane;
    bool in = lane < count && t < p.T;
    b = r = pos = 0;
    if (in) {
      b = static_cast<int>(__umul64hi(static_cast<unsigned long long>(t) * 2, p.per_row));   // t / L
      r = static_cast<int>(static_cast<unsigned>(t) - static_cast<unsigned>(b) * static_cast<unsigned>(p.L));
      pos = append ? p.seen[b] + r : p.pos != nullptr ? p.pos[t] : r;
      in = p.rows == nullptr || r < p.rows[b];
    }
    used = __ballot_sync(0xffffffffu, in);
  }
};

// The tile's angles, cos and sin of [token][rot / 2]: a warp a token, a lane a pair.
__device__ __forceinline__ void angles(const RotateParams& p, const TileTokens& at, int count, const unsigned long long* turn,
                                       float* cos, float* sin) {
  const int lane = threadIdx.x & 31, pairs = p.rot / 2;
  for (int i = threadIdx.x >> 5; i < count; i += blockDim.x >> 5) {
    const long long pos = __shfl_sync(0xffffffffu, at.pos, i);
    for (int k = lane; k < pairs; k += 32) {
      const unsigned long long a = turn[k] * static_cast<unsigned long long>(pos);
      const int top = static_cast<int>((a + 0x80000000ull) >> 32);   // of half a turn, in 2^-31
      const float angle = static_cast<float>(top) * 1.4629180792671596e-9f;   // pi 2^-31
      cos[i * pairs + k] = p.mscale * __cosf(angle);
      sin[i * pairs + k] = p.mscale * __sinf(angle);
    }
  }
}

__device__ __forceinline__ void turns_of(const RotateParams& p, unsigned long long* turn) {
  for (int k = threadIdx.x; k < p.rot / 2; k += blockDim.x) turn[k] = turn_of(__ldg(p.freq + k));
  __syncthreads();
}

// gamma of the lane's first and second members (1 where there is none).
__device__ __forceinline__ void gamma_of(const float* gamma, const LaneShare& s, bool inter, uint64_t (&a)[4], uint64_t (&b)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    a[i] = b[i] = f2_both(1.f);
    if (gamma == nullptr) continue;
    const float* x = gamma + 8 * s.va;
    const float* y = gamma + 8 * s.vb;
    if (inter) {   // the sixteen values from x on, in turn
      const float* z = i < 2 ? x + 4 * i : y + 4 * (i - 2);
      a[i] = f2_pack(__ldg(z), __ldg(z + 2));
      b[i] = f2_pack(__ldg(z + 1), __ldg(z + 3));
    } else {
      a[i] = f2_pack(__ldg(x + 2 * i), __ldg(x + 2 * i + 1));
      b[i] = f2_pack(__ldg(y + 2 * i), __ldg(y + 2 * i + 1));
    }
  }
}

// (as it stands when all CTAs have read it)
__device__ __forceinline__ int cache_len(const RotateParams& p, int list) {
  return min(max(__ldcg(p.len + list), 0), p.C);
}

// Forward, and append where cache_k is set.
template <class T, int W, bool kInter, bool kNorm>
__global__ void __launch_bounds__(kRotateThreads, kSmWarps / kRotateWarps) rotate_kernel(const RotateParams p, const RotatePlan plan) {
  extern __shared__ __align__(16) char raw[];
  __shared__ unsigned long long turn[SC_MAX_HEAD_WIDTH / 2];
  float* table = reinterpret_cast<float*>(raw + ring_bytes(plan, 2));   // [2][cos, sin][wt nt][rot / 2]
  pdl_wait();
  pdl_launch_dependents();
  const bool append = p.cache_k != nullptr;
  const LaneShare s(p, plan, W, kInter, append);
  const int count = plan.wt * plan.nt, pairs = p.rot / 2, mine = (threadIdx.x >> 5) / plan.wg * plan.nt;
  const bool beyond = s.q >= p.d / 16;   // (zeros)
  const bool copies = s.group * (32 / W) >= p.Hq + p.Hk;   // a warp of values alone
  const HeadsIn in = s.side == 0 ? p.q : s.side == 1 ? p.k : p.v;
  const HeadsOut out = s.side == 0 ? p.q_out : p.k_out;
  const bool to_cache = append && s.side > 0;
  const uint16_t* src = in.p + s.of_side * p.d;
  uint16_t* dst = !to_cache ? out.p + s.of_side * p.d : (s.side == 1 ? p.cache_k : p.cache_v) + s.of_side * p.stride_h;
  const int of = p.Hk / p.G, list = to_cache ? s.of_side / of : 0;
  const bool marks = to_cache && s.live && s.side == 1 && s.q == 0 && s.of_side % of == 0;
  uint64_t ga[4], gb[4];
  const float* gamma = s.side == 0 ? p.gamma_q : s.side == 1 ? p.gamma_k : nullptr;
  if (kNorm) gamma_of(gamma, s, kInter, ga, gb);
  uint4* ring = reinterpret_cast<uint4*>(raw) + (threadIdx.x >> 5) * (2 * plan.nt * 64) + (threadIdx.x & 31);
  const unsigned every = (1u << plan.nt) - 1;   // a warp's tokens of a tile
  auto load = [&](const TileTokens& at, long long t0, int half) {
    uint32_t to = smem_u32(ring + half * plan.nt * 64);
    const uint16_t *from_a = src + (t0 + mine) * in.ld + 8 * s.va, *from_b = from_a + 8 * (s.vb - s.va);
    unsigned left = at.used >> mine & every;
    if (left == (1u << kWarpTokens) - 1) {
#pragma unroll
      for (int i = 0; i < kWarpTokens; ++i, from_a += in.ld, from_b += in.ld) {
        cp_async16(to + i * 1024, from_a, !beyond);
        cp_async16(to + i * 1024 + 512, from_b, !beyond);
      }
    } else {
      for (; left != 0; left >>= 1, to += 1024, from_a += in.ld, from_b += in.ld)
        if (left & 1u) {
          cp_async16(to, from_a, !beyond);
          cp_async16(to + 512, from_b, !beyond);
        }
    }
    cp_async_commit();
  };
  auto token = [&](const uint4* own, const float* cos, const float* sin, const TileTokens& at, int number, uint16_t* to) {
    const uint4 xa = own[0], xb = own[32];
    uint4 ya = xa, yb = xb;
    if (!copies) {
      uint64_t a[4], b[4];
      unpack<T, kInter>(xa, xb, a, b);
      if (kNorm) {
        const float ss = squares<W>(a, b);
        const uint64_t inv = f2_both(gamma != nullptr ? rsqrtf(fmaf(ss, p.over_d, p.eps)) : 1.f);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          a[k] = f2_mul(a[k], f2_mul(ga[k], inv));
          b[k] = f2_mul(b[k], f2_mul(gb[k], inv));
        }
      }
      rotate<false, kInter>(a, b, cos, sin, s);
      pack<T, kInter>(a, b, ya, yb);
    }
    bool live = s.live;
    if (append) {
      const int b_u = __shfl_sync(0xffffffffu, at.b, number), r_u = __shfl_sync(0xffffffffu, at.r, number);
      if (to_cache) {
        const int held = min(max(p.len[b_u * p.G + list], 0), p.C), room = p.C - held;
        const int c = held + min(r_u, room);   // (held + r_u may pass 2^31)
        to = dst + b_u * p.stride_b + c * p.stride_c;
        live = live && r_u < room;
        if (marks && live) {
          const long long slot = (static_cast<long long>(b_u) * p.G + list) * p.C + c;
          p.acc[slot] = 0.f;
          p.slot_pos[slot] = p.seen[b_u] + r_u;
        }
      }
      if (s.side == 2) {
        ya = xa;
        yb = xb;
      }
    }
    if (!live) return;
    reinterpret_cast<uint4*>(to)[s.va] = ya;
    reinterpret_cast<uint4*>(to)[s.vb] = yb;
  };
  const long long step = static_cast<long long>(gridDim.x) * count;
  long long t0 = static_cast<long long>(blockIdx.x) * count;
  TileTokens next(p, t0, count, append);
  load(next, t0, 0);
  turns_of(p, turn);
  for (int half = 0; t0 < p.T; t0 += step, half ^= 1) {
    const TileTokens at = next;
    next = TileTokens(p, t0 + step, count, append);
    load(next, t0 + step, half ^ 1);
    float *cos = table + half * 2 * count * pairs, *sin = cos + count * pairs;
    angles(p, at, count, turn, cos, sin);
    cp_async_wait<1>();
    __syncthreads();   // (the other table is free when all have come here again)
    cos += mine * pairs;
    sin += mine * pairs;
    const uint4* own = ring + half * plan.nt * 64;
    uint16_t* to = dst + (t0 + mine) * out.ld;
    unsigned left = at.used >> mine & every;
    if (left == (1u << kWarpTokens) - 1) {   // all of them, side by side
#pragma unroll
      for (int i = 0; i < kWarpTokens; ++i) token(own + i * 64, cos + i * pairs, sin + i * pairs, at, mine + i, to + i * out.ld);
    } else {
      for (int i = mine; left != 0; left >>= 1, ++i, own += 64, cos += pairs, sin += pairs, to += out.ld)
        if (left & 1u) token(own, cos, sin, at, i, to);
    }
  }
  if (!append) return;
  // The last CTA to be done with len and seen moves them on.
  __shared__ bool last;
  const unsigned ctas = gridDim.x * gridDim.y;
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    last = atomicInc(p.done, ctas - 1) == ctas - 1;   // back to 0 after the last
    __threadfence();
  }
  __syncthreads();
  if (!last) return;
  for (int i = threadIdx.x; i < p.B * p.G; i += blockDim.x) {
    const int b = i / p.G;
    const int come = p.rows != nullptr ? min(max(p.rows[b], 0), p.L) : p.L;
    const long long n = static_cast<long long>(cache_len(p, i)) + come;
    if (n > p.C) atomicOr(p.status, kStatusFull);
    p.len_out[i] = static_cast<int>(min(n, static_cast<long long>(p.C)));
  }
  for (int b = threadIdx.x; b < p.B; b += blockDim.x)
    p.seen_out[b] = p.seen[b] + (p.rows != nullptr ? min(max(p.rows[b], 0), p.L) : p.L);
}

// Gradient.  dgamma: a lane adds up its features of its head over its tokens, the CTA its lanes and warps, in order;
// the parts of the CTAs (blockIdx.y has groups of its own) are added, in order, by rotate_gamma_kernel.
template <class T, int W, bool kInter, bool kNorm>
__global__ void __launch_bounds__(kRotateThreads, kSmWarps / kRotateWarps) rotate_back_kernel(const RotateParams p, const RotatePlan plan) {
  constexpr int kAt = 1;   // tokens that go through the stages together (two: registers do not suffice)
  extern __shared__ __align__(16) char raw[];
  __shared__ unsigned long long turn[SC_MAX_HEAD_WIDTH / 2];
  float* table = reinterpret_cast<float*>(raw + ring_bytes(plan, 4));
  __shared__ float sums[kRotateWarps][SC_MAX_HEAD_WIDTH];
  pdl_wait();
  pdl_launch_dependents();
  const LaneShare s(p, plan, W, kInter, false);
  const int count = plan.wt * plan.nt, pairs = p.rot / 2, warp = threadIdx.x >> 5, mine = warp / plan.wg * plan.nt;
  const bool beyond = s.q >= p.d / 16;
  const HeadsIn dy = s.side == 0 ? p.dq : p.dk, in = s.side == 0 ? p.q : p.k;
  const HeadsOut out = s.side == 0 ? p.q_out : p.k_out;
  const float* gamma = s.side == 0 ? p.gamma_q : p.gamma_k;
  const uint16_t *src = dy.p + s.of_side * p.d, *src_x = in.p + s.of_side * p.d;
  uint16_t* dst = out.p + s.of_side * p.d;
  uint64_t ga[4], gb[4], total[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) total[k] = 0;
  if (kNorm) gamma_of(gamma, s, kInter, ga, gb);
  uint4* ring = reinterpret_cast<uint4*>(raw) + warp * (2 * plan.nt * 128) + (threadIdx.x & 31);
  auto load = [&](const TileTokens& at, long long t0, int half) {
    const uint32_t to = smem_u32(ring + half * plan.nt * 128);
    const uint16_t *from = src + (t0 + mine) * dy.ld, *from_x = src_x + (t0 + mine) * in.ld;
    for (int i = 0; i < plan.nt; ++i, from += dy.ld, from_x += in.ld)
      if (at.used >> (mine + i) & 1u) {
        cp_async16(to + i * 2048, from + 8 * s.va, !beyond);
        cp_async16(to + i * 2048 + 512, from + 8 * s.vb, !beyond);
        if (kNorm) {
          cp_async16(to + i * 2048 + 1024, from_x + 8 * s.va, !beyond && gamma != nullptr);
          cp_async16(to + i * 2048 + 1536, from_x + 8 * s.vb, !beyond && gamma != nullptr);
        }
      }
    cp_async_commit();
  };
  const long long step = static_cast<long long>(gridDim.x) * count;
  long long t0 = static_cast<long long>(blockIdx.x) * count;
  TileTokens next(p, t0, count, false);
  load(next, t0, 0);
  turns_of(p, turn);
  for (int half = 0; t0 < p.T; t0 += step, half ^= 1) {
    const TileTokens at = next;
    next = TileTokens(p, t0 + step, count, false);
    load(next, t0 + step, half ^ 1);
    float *cos = table + half * 2 * count * pairs, *sin = cos + count * pairs;
    angles(p, at, count, turn, cos, sin);
    cp_async_wait<1>();
    __syncthreads();
    for (int i = 0; i < plan.nt; i += kAt) {
      uint64_t a[kAt][4], b[kAt][4], x[kAt][4], y[kAt][4];
#pragma unroll
      for (int u = 0; u < kAt; ++u) {
        const uint4* own = ring + (half * plan.nt + min(i + u, plan.nt - 1)) * 128;
        unpack<T, kInter>(own[0], own[32], a[u], b[u]);
        if (kNorm) unpack<T, kInter>(own[64], own[96], x[u], y[u]);
      }
#pragma unroll
      for (int u = 0; u < kAt; ++u) {
        const int row = (mine + min(i + u, plan.nt - 1)) * pairs;
        rotate<true, kInter>(a[u], b[u], cos + row, sin + row, s);
      }
      if (kNorm) {
        float ss[kAt];
#pragma unroll
        for (int u = 0; u < kAt; ++u) ss[u] = squares<W>(x[u], y[u]);
        uint64_t inv[kAt], inner[kAt];
#pragma unroll
        for (int u = 0; u < kAt; ++u) {
          inv[u] = f2_both(gamma != nullptr ? rsqrtf(fmaf(ss[u], p.over_d, p.eps)) : 1.f);
          const bool used = i + u < plan.nt && (at.used >> (mine + i + u) & 1u);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            x[u][k] = f2_mul(x[u][k], inv[u]);
            y[u][k] = f2_mul(y[u][k], inv[u]);
          }
          if (used) {   // (of the whole warp)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              total[k] = f2_fma(a[u][k], x[u][k], total[k]);
              total[4 + k] = f2_fma(b[u][k], y[u][k], total[4 + k]);
            }
          }
          inner[u] = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            a[u][k] = f2_mul(a[u][k], ga[k]);
            b[u][k] = f2_mul(b[u][k], gb[k]);
            inner[u] = f2_fma(a[u][k], x[u][k], inner[u]);
            inner[u] = f2_fma(b[u][k], y[u][k], inner[u]);
          }
        }
#pragma unroll
        for (int u = 0; u < kAt; ++u) {
          const float mean = -sum_lanes<W>(f2_total(inner[u])) * p.over_d;
          if (gamma == nullptr) continue;   // (of the lane's head)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            a[u][k] = f2_mul(inv[u], f2_fma(x[u][k], f2_both(mean), a[u][k]));
            b[u][k] = f2_mul(inv[u], f2_fma(y[u][k], f2_both(mean), b[u][k]));
          }
        }
      }
#pragma unroll
      for (int u = 0; u < kAt; ++u) {
        const int token = mine + i + u;
        if (i + u >= plan.nt || !(at.used >> token & 1u) || !s.live) continue;
        uint4 ya, yb;
        pack<T, kInter>(a[u], b[u], ya, yb);
        uint4* to = reinterpret_cast<uint4*>(dst + (t0 + token) * out.ld);
        to[s.va] = ya;
        to[s.vb] = yb;
      }
    }
  }
  if constexpr (kNorm) {
#pragma unroll
  for (int side = 0; side < 2; ++side) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[2];
      f2_unpack(total[i], v[0], v[1]);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v[k] = s.live && s.side == side ? v[k] : 0.f;
#pragma unroll
        for (int o = W; o < 32; o <<= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        const int member = 2 * (i & 3) + k, second = i / 4;   // pair of the lane's eight
        const int feature = kInter ? 8 * (member < 4 ? s.va : s.vb) + 2 * (member & 3) + second : 8 * (second ? s.vb : s.va) + member;
        if (!beyond && s.sub == 0) sums[warp][feature] = v[k];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < p.d; i += blockDim.x) {
      float v = 0.f;
      for (int w = 0; w < static_cast<int>(blockDim.x >> 5); ++w) v += sums[w][i];
      p.part[((static_cast<long long>(blockIdx.y) * gridDim.x + blockIdx.x) * 2 + side) * p.d + i] = v;
    }
    __syncthreads();
  }
  }
}

// dgamma from the CTAs' parts: eight features a CTA, every 32nd part a thread.
__global__ void __launch_bounds__(kRotateThreads) rotate_gamma_kernel(const RotateParams p, int ctas) {
  __shared__ float sums[kRotateWarps][8];
  pdl_wait();
  pdl_launch_dependents();
  const int f = threadIdx.x & 7, i = blockIdx.x * 8 + f, from = threadIdx.x / 8, lane = threadIdx.x & 31;   // of [2][d]
  float v = 0.f;
#pragma unroll 10
  for (int c = from; c < ctas; c += 32) v += __ldcg(p.part + static_cast<long long>(c) * 2 * p.d + i);
  v += __shfl_xor_sync(0xffffffffu, v, 8);
  v += __shfl_xor_sync(0xffffffffu, v, 16);
  if (lane < 8) sums[threadIdx.x >> 5][f] = v;
  __syncthreads();
  if (threadIdx.x >= 8) return;
  v = 0.f;
#pragma unroll
  for (int w = 0; w < kRotateWarps; ++w) v += sums[w][f];
  float* to = i < p.d ? p.dgamma_q : p.dgamma_k;
  if (to != nullptr) to[i < p.d ? i : i - p.d] = v;
}

namespace {

// Lanes that a head takes: a power of two, four at least.
int lanes_of(int d) { return d <= 64 ? 4 : d <= 128 ? 8 : 16; }

// All groups of a few tokens to a CTA of three warps at least (the smaller, the more evenly they fill an SM's sixteen
// warps of 128 registers); the fewer tokens there are, the fewer at a time, until each SM has two CTAs.
RotatePlan plan_of(const RotateParams& p, int groups, int most_tokens) {
  RotatePlan plan;
  plan.wg = std::min(groups, kRotateWarps);
  plan.wt = plan.wg >= 3 ? 1 : plan.wg == 2 ? 2 : 4;
  const int columns = (groups + plan.wg - 1) / plan.wg;
  plan.nt = most_tokens;
  while (plan.nt > 1 && (p.T + plan.wt * plan.nt - 1) / (plan.wt * plan.nt) * columns < 2 * kCacheSms) plan.nt /= 2;
  while (plan.wt > 1 && (p.T + plan.wt - 1) / plan.wt * columns < kCacheSms) --plan.wt;
  const long long tiles = (p.T + plan.wt * plan.nt - 1) / (plan.wt * plan.nt);
  plan.ctas = static_cast<int>(std::min<long long>(tiles, std::max(1, kCacheSms * (kSmWarps / (plan.wg * plan.wt)) / columns)));
  return plan;
}

template <class T, int W, bool kInter, bool kNorm>
struct Rotation {
  static int groups_of(int heads) { return (heads + 32 / W - 1) / (32 / W); }
  static size_t bytes(const RotateParams& p, const RotatePlan& plan, int vectors) {
    return ring_bytes(plan, vectors) + sizeof(float) * 2 * 2 * plan.wt * plan.nt * (p.rot / 2);
  }
  // the most: the ring of eight warps, and angles of the most tokens
  static constexpr size_t kMost = kRotateWarps * 2 * kWarpTokens * 2 * 512 + 4 * 4 * kTileTokens * (SC_MAX_HEAD_WIDTH / 2);
  static_assert(kWarpTokens * 2 == kWarpTokensBack * 4, "the same bytes backward");
  static cudaError_t forward(const RotateParams& p, cudaStream_t st) {
    const int groups = groups_of(p.Hq + p.Hk * (p.cache_k != nullptr ? 2 : 1));
    const RotatePlan plan = plan_of(p, groups, kWarpTokens);
    const cudaError_t e = allow_shared<rotate_kernel<T, W, kInter, kNorm>>(kMost);
    if (e != cudaSuccess) return e;
    return launch_chained(rotate_kernel<T, W, kInter, kNorm>, dim3(plan.ctas, (groups + plan.wg - 1) / plan.wg),
                          dim3(plan.wg * plan.wt * 32), bytes(p, plan, 2), st, p, plan);
  }
  static cudaError_t backward(const RotateParams& p, cudaStream_t st) {
    const int groups = groups_of(p.Hq + p.Hk);
    const RotatePlan plan = plan_of(p, groups, kWarpTokensBack);
    const int columns = (groups + plan.wg - 1) / plan.wg;
    cudaError_t e = allow_shared<rotate_back_kernel<T, W, kInter, kNorm>>(kMost);
    if (e != cudaSuccess) return e;
    e = launch_chained(rotate_back_kernel<T, W, kInter, kNorm>, dim3(plan.ctas, columns),
                                   dim3(plan.wg * plan.wt * 32), bytes(p, plan, 4), st, p, plan);
    if (e != cudaSuccess || !kNorm) return e;
    return launch_chained(rotate_gamma_kernel, dim3(p.d / 4), dim3(kRotateThreads), 0, st, p, plan.ctas * columns);
  }
};

// what(Rotation<..>) of the lanes a head takes, the layout of its pairs, and whether there is a norm
template <class T, int W, class What>
cudaError_t of_layout(const RotateParams& p, const What& what) {
  if (p.gamma_q != nullptr || p.gamma_k != nullptr)
    return p.interleaved ? what(Rotation<T, W, true, true>()) : what(Rotation<T, W, false, true>());
  return p.interleaved ? what(Rotation<T, W, true, false>()) : what(Rotation<T, W, false, false>());
}
template <class T, class What>
cudaError_t of_width(const RotateParams& p, const What& what) {
  switch (lanes_of(p.d)) {
    case 4: return of_layout<T, 4>(p, what);
    case 8: return of_layout<T, 8>(p, what);
    default: return of_layout<T, 16>(p, what);
  }
}
template <class What>
cudaError_t of_type(int dtype, const RotateParams& p, const What& what) {
  return dtype == SC_FP16 ? of_width<Fp16>(p, what) : of_width<Bf16>(p, what);
}

}  // namespace

cudaError_t launch_rotate(const RotateParams& p, int dtype, cudaStream_t st) {
  return of_type(dtype, p, [&](auto r) { return r.forward(p, st); });
}

cudaError_t launch_rotate_back(const RotateParams& p, int dtype, cudaStream_t st) {
  return of_type(dtype, p, [&](auto r) { return r.backward(p, st); });
}

}  // namespace sc
