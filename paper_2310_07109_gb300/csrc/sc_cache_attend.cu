// sc_cache_attend.cu -- attention of the newest tokens over a pruned key-value cache,
// with the weights added up for each slot.
//
//   t = scale log2(e) q . k;   P = 2^(t - LSE);   O = P V;   acc = decay acc + sum over rows, mean over heads of P
// Three launches:
//   rows    one pass over K and V with the running reference (the largest t so far) and sum of a row's weights;
//           a CTA has up to 64 rows of a key head (tokens x query heads) and a part of the list's
//           slots, four warps of 16 rows each; S = Q K^T and P V by warp products, P in registers
//   join    the parts of a list: LSE = reference + log2(sum) of all, O scaled and rounded
//   sums    each slot's weights from K and the rows' LSE: 2^(t - LSE) summed down the key's column over
//           rows and heads in a fixed order
#include <algorithm>
#include <cuda_runtime.h>
#include <cstdint>

#include "sc_cache.cuh"
#include "sc_expert.cuh"

namespace sc {

constexpr int kAttendWarps = 4;
constexpr int kAttendThreads = kAttendWarps * 32;
constexpr int kRowTile = 16 * kAttendWarps;
constexpr int kKeyTile = 64;
constexpr int kJoinWarps = 8;

// A tile of `kKeyTile` (or kRowTile) rows of D values: 16-byte chunk c of row r lies at chunk c ^ (r & 7), so that the eight rows of
// a fragment are in eight different banks.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(uint32_t base, int row, int chunk) {
  return base + static_cast<uint32_t>(row * (D * 2) + ((chunk ^ (row & 7)) << 4));
}

__device__ __forceinline__ void cp_async4(uint32_t saddr, const void* gptr, bool copy) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(saddr), "l"(gptr), "r"(copy ? 4 : 0) : "memory");
}

// A fragment (16 rows x 16) of a tile's rows row0.., values 16 k ..
template <int D>
__device__ __forceinline__ void load_a(uint32_t base, int row0, int k, int lane, uint32_t (&a)[4]) {
  ldmatrix4(chunk_at<D>(base, row0 + (lane & 15), 2 * k + (lane >> 4)), a);
}
// B fragments of 16 keys x 16 values: b[0], b[1] of keys 0-7, b[2], b[3] of keys 8-15
template <int D>
__device__ __forceinline__ void load_b(uint32_t base, int key0, int k, int lane, uint32_t (&b)[4]) {
  ldmatrix4(chunk_at<D>(base, key0 + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), b);
}
// B fragments of 16 keys (the contraction) x 16 values of V
template <int D>
__device__ __forceinline__ void load_v(uint32_t base, int key0, int n, int lane, uint32_t (&b)[4]) {
  ldmatrix4_trans(chunk_at<D>(base, key0 + (lane & 15), 2 * n + (lane >> 4)), b);
}

struct ListOf {
  int n, rows, first;   // slots and rows in use, position of row 0
};
__device__ __forceinline__ ListOf list_of(const AttendParams& p, int b, int g) {
  ListOf l;
  l.n = min(max(__ldg(p.len + b * p.G + g), 0), p.C);
  l.rows = p.rows != nullptr ? min(max(__ldg(p.rows + b), 0), p.T) : p.T;
  l.first = __ldg(p.seen + b) - l.rows;
  return l;
}

// Rows m0 .. of key head hk into a tile; zeros beyond the rows in use.
template <int D>
__device__ __forceinline__ void load_q(const AttendParams& p, int b, int hk, int m0, int rows, uint32_t base) {
  for (int i = threadIdx.x; i < kRowTile * (D / 8); i += kAttendThreads) {
    const int row = i / (D / 8), c = i % (D / 8), m = m0 + row;
    const int tok = m / p.R, h = hk * p.R + m % p.R;
    const bool live = m < p.M && tok < rows;
    const uint16_t* src = p.q + (static_cast<long long>(b) * p.T + (live ? tok : 0)) * p.ldq +
                          static_cast<long long>(live ? h : 0) * D + c * 8;
    cp_async16(chunk_at<D>(base, row, c), src, live);
  }
}

template <int D>
__device__ __forceinline__ void load_keys(const AttendParams& p, const uint16_t* head, int j0, int n, uint32_t base) {
  for (int i = threadIdx.x; i < kKeyTile * (D / 8); i += kAttendThreads) {
    const int row = i / (D / 8), c = i % (D / 8), j = j0 + row;
    const bool live = j < n;
    cp_async16(chunk_at<D>(base, row, c), head + (live ? j : 0) * p.stride_c + c * 8, live);
  }
}

template <int D>
struct RowsSmem {
  alignas(128) uint16_t q[kRowTile * D];
  alignas(128) uint16_t k[2][kKeyTile * D];
  alignas(128) uint16_t v[2][kKeyTile * D];
  int pos[2][kKeyTile];
};

template <class T, int D>
__global__ void __launch_bounds__(kAttendThreads) attend_rows_kernel(const AttendParams p) {
  extern __shared__ char raw[];
  RowsSmem<D>& sm = *reinterpret_cast<RowsSmem<D>*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  pdl_wait();
  pdl_launch_dependents();
  const int tiles_m = (p.M + kRowTile - 1) / kRowTile;
  long long id = blockIdx.x;
  const int split = static_cast<int>(id % p.splits);
  id /= p.splits;
  const int m0 = static_cast<int>(id % tiles_m) * kRowTile;
  id /= tiles_m;
  const int hk = static_cast<int>(id % p.Hk), b = static_cast<int>(id / p.Hk);
  const int g = hk / (p.Hk / p.G);
  const ListOf l = list_of(p, b, g);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int tiles = (l.n + kKeyTile - 1) / kKeyTile, per = (tiles + p.splits - 1) / p.splits;
  const int t0 = min(split * per, tiles), t1 = m0 < l.rows * p.R ? min(t0 + per, tiles) : t0;
  const uint16_t* kh = p.k + b * p.stride_b + hk * p.stride_h;
  const uint16_t* vh = p.v + b * p.stride_b + hk * p.stride_h;
  const int32_t* pos = p.pos + (static_cast<long long>(b) * p.G + g) * p.C;
  const uint32_t sq = smem_u32(sm.q);

  auto load = [&](int tile, int s) {
    const int j0 = tile * kKeyTile;
    load_keys<D>(p, kh, j0, l.n, smem_u32(sm.k[s]));
    load_keys<D>(p, vh, j0, l.n, smem_u32(sm.v[s]));
    if (threadIdx.x < kKeyTile) {
      const int j = j0 + threadIdx.x;
      cp_async4(smem_u32(&sm.pos[s][threadIdx.x]), pos + min(j, l.n - 1), j < l.n);
    }
    cp_async_commit();
  };

  // this lane's rows of the warp's sixteen: lane / 4 and that + 8
  float o[D / 8][4], ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
  int at[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) at[u] = l.first + (m0 + warp * 16 + (lane >> 2) + 8 * u) / p.R;
  const int last = l.first + min(m0 + kRowTile - 1, l.rows * p.R - 1) / p.R;   // the latest row of the tile

  if (t0 < t1) {
    load_q<D>(p, b, hk, m0, l.rows, sq);
    load(t0, 0);
  }
  for (int tile = t0; tile < t1; ++tile) {
    const int s = (tile - t0) & 1;
    if (tile + 1 < t1) {
      load(tile + 1, s ^ 1);
      cp_async_wait<1>();
    } else {
      cp_async_wait<0>();
    }
    // a slot that no row of the tile sees may hold anything: its V is taken as 0
    bool unseen = false;
    if (threadIdx.x < kKeyTile) {
      const int at_key = sm.pos[s][threadIdx.x];
      unseen = tile * kKeyTile + threadIdx.x < l.n && (at_key < 0 || at_key > last);
    }
    if (__syncthreads_or(unseen)) {
      if (unseen)
        for (int c = 0; c < D / 8; ++c)
          *reinterpret_cast<uint4*>(reinterpret_cast<char*>(sm.v[s]) + threadIdx.x * D * 2 + c * 16) = make_uint4(0, 0, 0, 0);
      __syncthreads();
    }
    const uint32_t sk = smem_u32(sm.k[s]), sv = smem_u32(sm.v[s]);
    float c[kKeyTile / 8][4];
#pragma unroll
    for (int i = 0; i < kKeyTile / 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t a[4];
      load_a<D>(sq, warp * 16, k, lane, a);
#pragma unroll
      for (int n = 0; n < kKeyTile / 16; ++n) {
        uint32_t f[4];
        load_b<D>(sk, n * 16, k, lane, f);
        T::mma(c[2 * n], a, f[0], f[1]);
        T::mma(c[2 * n + 1], a, f[2], f[3]);
      }
    }
    float top[2] = {ref[0], ref[1]};
#pragma unroll
    for (int i = 0; i < kKeyTile / 8; ++i) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = 8 * i + 2 * (lane & 3) + (k & 1), where = sm.pos[s][key];
        const bool sees = tile * kKeyTile + key < l.n && where >= 0 && where <= at[k >> 1];
        c[i][k] = sees ? c[i][k] * p.scale2 : -INFINITY;
        top[k >> 1] = fmaxf(top[k >> 1], c[i][k] - T::kHeadroom);
      }
    }
    float keep[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 1));
      top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 2));
      keep[u] = top[u] == ref[u] ? 1.f : ex2(ref[u] - top[u]);   // (both -inf: nothing so far)
      ref[u] = top[u];
      sum[u] *= keep[u];
      top[u] = top[u] == -INFINITY ? 0.f : top[u];
    }
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      o[i][0] *= keep[0];
      o[i][1] *= keep[0];
      o[i][2] *= keep[1];
      o[i][3] *= keep[1];
    }
#pragma unroll
    for (int i = 0; i < kKeyTile / 8; ++i) {
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] = ex2(c[i][k] - top[k >> 1]);
      sum[0] += c[i][0] + c[i][1];
      sum[1] += c[i][2] + c[i][3];
    }
#pragma unroll
    for (int k = 0; k < kKeyTile / 16; ++k) {
      const uint32_t a[4] = {T::pack(c[2 * k][0], c[2 * k][1]), T::pack(c[2 * k][2], c[2 * k][3]),
                             T::pack(c[2 * k + 1][0], c[2 * k + 1][1]), T::pack(c[2 * k + 1][2], c[2 * k + 1][3])};
#pragma unroll
      for (int n = 0; n < D / 16; ++n) {
        uint32_t f[4];
        load_v<D>(sv, k * 16, n, lane, f);
        T::mma(o[2 * n], a, f[0], f[1]);
        T::mma(o[2 * n + 1], a, f[2], f[3]);
      }
    }
    __syncthreads();   // the stage is free
  }
  const long long unit = static_cast<long long>(b) * p.Hk + hk;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 1);
    sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 2);
    const int m = m0 + warp * 16 + (lane >> 2) + 8 * u;
    if (m >= l.rows * p.R) continue;
    const long long at_row = (unit * p.splits + split) * p.M + m;
    if ((lane & 3) == 0) p.ml[at_row] = make_float2(ref[u], sum[u]);
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
      *reinterpret_cast<float2*>(p.part + at_row * D + 8 * i + 2 * (lane & 3)) = make_float2(o[i][2 * u], o[i][2 * u + 1]);
  }
}

// A warp a row: its parts joined.
template <class T, int D>
__global__ void __launch_bounds__(kJoinWarps * 32) attend_join_kernel(const AttendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31;
  const long long row = static_cast<long long>(blockIdx.x) * kJoinWarps + (threadIdx.x >> 5);
  if (row >= static_cast<long long>(p.B) * p.Hk * p.M) return;
  const long long unit = row / p.M;
  const int m = static_cast<int>(row - unit * p.M), b = static_cast<int>(unit / p.Hk), hk = static_cast<int>(unit - static_cast<long long>(b) * p.Hk);
  const ListOf l = list_of(p, b, hk / (p.Hk / p.G));
  if (m >= l.rows * p.R) {
    if (lane == 0) p.lse[row] = INFINITY;
    return;
  }
  float ref = -INFINITY;
  for (int s = lane; s < p.splits; s += 32) ref = fmaxf(ref, p.ml[(unit * p.splits + s) * p.M + m].x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
  constexpr int kOwn = D / 32;
  float total = 0.f, o[kOwn] = {};
  for (int s = 0; s < p.splits; ++s) {
    const long long at = (unit * p.splits + s) * p.M + m;
    const float2 ml = p.ml[at];
    if (ml.x == -INFINITY && ml.y == 0.f) continue;   // nothing seen (a NaN is)
    const float w = ex2(ml.x - ref);
    total += w * ml.y;
#pragma unroll
    for (int i = 0; i < kOwn; i += 2) {
      const float2 f = *reinterpret_cast<const float2*>(p.part + at * D + lane * kOwn + i);
      o[i] += w * f.x;
      o[i + 1] += w * f.y;
    }
  }
  const bool none = ref == -INFINITY && total == 0.f;
  const float inv = none ? 0.f : 1.f / total;
  uint32_t* to = reinterpret_cast<uint32_t*>(p.o + (static_cast<long long>(b) * p.T + m / p.R) * p.ldo +
                                             static_cast<long long>(hk * p.R + m % p.R) * D + lane * kOwn);
#pragma unroll
  for (int i = 0; i < kOwn; i += 2) to[i / 2] = T::pack(o[i] * inv, o[i + 1] * inv);
  if (lane == 0) p.lse[row] = none ? INFINITY : ref + log2f(total);
}

template <int D>
struct SumsSmem {
  alignas(128) uint16_t k[kKeyTile * D];
  alignas(128) uint16_t q[2][kRowTile * D];
  int pos[kKeyTile];
  float sum[kAttendWarps][kKeyTile];
};

// A CTA has a tile of a list's slots: the weights of all rows of the list's heads.
template <class T, int D>
__global__ void __launch_bounds__(kAttendThreads) attend_sums_kernel(const AttendParams p) {
  extern __shared__ char raw[];
  SumsSmem<D>& sm = *reinterpret_cast<SumsSmem<D>*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  pdl_wait();
  pdl_launch_dependents();
  const int tiles = (p.C + kKeyTile - 1) / kKeyTile;
  const int tile = blockIdx.x % tiles, list = blockIdx.x / tiles, b = list / p.G, g = list - b * p.G;
  const ListOf l = list_of(p, b, g);
  const int j0 = tile * kKeyTile, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (j0 >= l.n) return;
  const long long at0 = static_cast<long long>(list) * p.C + j0;
  if (l.rows == 0) {
    if (threadIdx.x < kKeyTile && j0 + threadIdx.x < l.n) p.acc_out[at0 + threadIdx.x] = p.acc[at0 + threadIdx.x];
    return;
  }
  const int of = p.Hk / p.G, rows_m = l.rows * p.R, tiles_m = (rows_m + kRowTile - 1) / kRowTile;
  if (threadIdx.x < kKeyTile) {
    const int j = j0 + threadIdx.x;
    sm.pos[threadIdx.x] = j < l.n ? __ldg(p.pos + at0 + threadIdx.x) : -1;
  }
  float sum[kKeyTile / 8][2] = {};   // this lane's keys 2 (lane & 3), + 1 of each eight
  const int steps = of * tiles_m;
  auto load = [&](int step) {
    load_q<D>(p, b, g * of + step / tiles_m, step % tiles_m * kRowTile, l.rows, smem_u32(sm.q[step & 1]));
    cp_async_commit();
  };
  load(0);
  for (int step = 0; step < steps; ++step) {
    const int hk = g * of + step / tiles_m, m0 = step % tiles_m * kRowTile;
    if (step % tiles_m == 0) {
      load_keys<D>(p, p.k + b * p.stride_b + hk * p.stride_h, j0, l.n, smem_u32(sm.k));
      cp_async_commit();
    }
    cp_async_wait<0>();
    __syncthreads();
    if (step + 1 < steps) load(step + 1);
    const uint32_t sq = smem_u32(sm.q[step & 1]), sk = smem_u32(sm.k);
    float c[kKeyTile / 8][4];
#pragma unroll
    for (int i = 0; i < kKeyTile / 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t a[4];
      load_a<D>(sq, warp * 16, k, lane, a);
#pragma unroll
      for (int n = 0; n < kKeyTile / 16; ++n) {
        uint32_t f[4];
        load_b<D>(sk, n * 16, k, lane, f);
        T::mma(c[2 * n], a, f[0], f[1]);
        T::mma(c[2 * n + 1], a, f[2], f[3]);
      }
    }
    float lse[2];
    int at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int m = m0 + warp * 16 + (lane >> 2) + 8 * u;
      lse[u] = m < rows_m ? p.lse[(static_cast<long long>(b) * p.Hk + hk) * p.M + m] : INFINITY;
      at[u] = m < rows_m ? l.first + m / p.R : -1;
    }
#pragma unroll
    for (int i = 0; i < kKeyTile / 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int where = sm.pos[8 * i + 2 * (lane & 3) + (k & 1)];
        if (where >= 0 && where <= at[k >> 1]) sum[i][k & 1] += ex2(c[i][k] * p.scale2 - lse[k >> 1]);
      }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kKeyTile / 8; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v = sum[i][k];
      v += __shfl_xor_sync(0xffffffffu, v, 4);
      v += __shfl_xor_sync(0xffffffffu, v, 8);
      v += __shfl_xor_sync(0xffffffffu, v, 16);
      if (lane < 4) sm.sum[warp][8 * i + 2 * lane + k] = v;
    }
  __syncthreads();
  if (threadIdx.x < kKeyTile && j0 + threadIdx.x < l.n) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kAttendWarps; ++w) v += sm.sum[w][threadIdx.x];
    p.acc_out[at0 + threadIdx.x] = p.decay * p.acc[at0 + threadIdx.x] + v / static_cast<float>(p.H / p.G);
  }
}

namespace {

template <class T, int D>
cudaError_t configure_of() {
  cudaError_t e = cudaFuncSetAttribute(attend_rows_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(RowsSmem<D>) + 128);
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(attend_sums_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SumsSmem<D>) + 128);
}

template <class T, int D>
cudaError_t launch_of(const AttendParams& p, cudaStream_t st) {
  const long long units = static_cast<long long>(p.B) * p.Hk;
  const int tiles_m = (p.M + kRowTile - 1) / kRowTile;
  cudaError_t e = launch_chained(attend_rows_kernel<T, D>, dim3(static_cast<unsigned>(units * tiles_m * p.splits)),
                                 dim3(kAttendThreads), sizeof(RowsSmem<D>) + 128, st, p);
  if (e != cudaSuccess) return e;
  e = launch_chained(attend_join_kernel<T, D>, dim3(static_cast<unsigned>((units * p.M + kJoinWarps - 1) / kJoinWarps)),
                     dim3(kJoinWarps * 32), 0, st, p);
  if (e != cudaSuccess) return e;
  const long long tiles = (p.C + kKeyTile - 1) / kKeyTile;
  return launch_chained(attend_sums_kernel<T, D>, dim3(static_cast<unsigned>(tiles * p.B * p.G)), dim3(kAttendThreads),
                        sizeof(SumsSmem<D>) + 128, st, p);
}

}  // namespace

cudaError_t configure_attend() {
  cudaError_t e = configure_of<Bf16, 64>();
  if (e == cudaSuccess) e = configure_of<Bf16, 128>();
  if (e == cudaSuccess) e = configure_of<Fp16, 64>();
  if (e == cudaSuccess) e = configure_of<Fp16, 128>();
  return e;
}

cudaError_t launch_attend(const AttendParams& p, int d, int dtype, cudaStream_t st) {
  if (dtype == SC_FP16) return d == 64 ? launch_of<Fp16, 64>(p, st) : launch_of<Fp16, 128>(p, st);
  return d == 64 ? launch_of<Bf16, 64>(p, st) : launch_of<Bf16, 128>(p, st);
}

}  // namespace sc
