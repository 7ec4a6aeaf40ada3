// sc_cache_attend.cu -- attention of the newest tokens over a pruned key-value cache,
// with the weights added up for each slot.
//
//   t = scale log2(e) q . k;   P = 2^(t - LSE);   O = P V;   acc = decay acc + sum over rows, mean over heads of P
// A key head of a sequence (a unit) has M = T R rows, R query heads to a key head.  Bound by the bytes of K and V (each read
// once at M <= 32) as long as there are few rows.  Products are warp-level ones (16 rows at least, which a token of
// grouped heads does not fill; they take 25 % of the tensor pipe), with S, P and O in registers; softmax with the
// running reference (the largest t so far) and sum of each row; P meets V as two 16-bit values, one product each (as one value:
// attend_batch 76 us and 76.5 with two, attend_window 27 and 28.5, prompts an eighth less; O was then off by 1.9e-3 of 64
// bits, with two by the 1.7e-3 of its one rounding).
//   M <= 16   attend_few_kernel: the 16-slot tiles of all units dealt out to warps in equal runs, each warp with a
//             pipeline of its own.  32 streams of 3000 to 8000 slots, 16 heads over 4 of 128: the call 76.5 us
//             for 390 MB, this kernel on its own with cold caches 71 (5.5 TB/s); 252 as many rows below
//   M <= 32   attend_rows_kernel<.., 2>: a CTA a part of a unit, two pairs of warps on either half of each 64-slot
//             tile.  Four sequences of 12 heads of 64, 32 tokens, 4096 slots: the call 28.5 us, 50 as many rows below
//     both keep the scores t, 4 bytes a row and slot, and attend_stored_join_kernel joins the parts of the units
//     (LSE = reference + log2(sum) of all, O scaled and rounded) and adds 2^(t - LSE) up over the list's rows and heads
//     in a fixed order (the 32 tokens: 30 us when first built so, 37 where K is read again for the sums)
//   M > 32    attend_rows_kernel<.., 1>, attend_join_kernel, and the sums from scores kept (attend_stored_sums_kernel,
//             up to kStoredBytes) or computed again (attend_sums_kernel, attend_heads_kernel).  A prompt of 4096
//             tokens, 16 heads over 4 of 128: 946 us (145 TFLOP/s of 4 T n d H)
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

// Tiles are rows of D values: 16-byte chunk c of row r lies at chunk c ^ (r & 7), so that the eight rows of a fragment are
// in eight different banks.
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

// O += (first + second) V of 16 keys, four fragments of O at a time.
template <class T, int D>
__device__ __forceinline__ void add_values(float (&o)[D / 8][4], const uint32_t (&first)[4], const uint32_t (&second)[4], uint32_t base,
                                           int key0, int lane) {
#pragma unroll
  for (int n = 0; n < D / 16; n += 2) {
    uint32_t f[2][4];
    load_v<D>(base, key0, n, lane, f[0]);
    load_v<D>(base, key0, n + 1, lane, f[1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) T::mma(o[2 * n + i], first, f[i / 2][i % 2 * 2], f[i / 2][i % 2 * 2 + 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) T::mma(o[2 * n + i], second, f[i / 2][i % 2 * 2], f[i / 2][i % 2 * 2 + 1]);
  }
}

struct ListOf {
  int n, rows, first;   // slots and rows in use, position of row 0
};
__device__ __forceinline__ ListOf list_of(const AttendParams& p, int b, int g) {
  ListOf l;
  l.n = min(max(p.len[b * p.G + g], 0), p.C);
  l.rows = p.rows != nullptr ? min(max(p.rows[b], 0), p.T) : p.T;
  l.first = p.seen[b] - l.rows;
  return l;
}

// A lane's scores of slots j, j + 1 for the rows m0 + lane / 4 and that + 8 (the pitch is even: the second has room).
__device__ __forceinline__ void store_scores(const AttendParams& p, float* of_unit, int m0, int rows_m, int j, int n, const float (&c)[4]) {
  if (j >= n) return;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int m = m0 + static_cast<int>(threadIdx.x & 31) / 4 + 8 * u;
    if (m < rows_m) *reinterpret_cast<float2*>(of_unit + static_cast<long long>(m) * p.pitch + j) = make_float2(c[2 * u], c[2 * u + 1]);
  }
}

// Rows m0 .. of key head hk into a tile; zeros beyond the rows in use.
template <int D>
__device__ __forceinline__ void load_q(const AttendParams& p, int b, int hk, int m0, int rows, int tile_rows, uint32_t base) {
  for (int i = threadIdx.x; i < tile_rows * (D / 8); i += kAttendThreads) {
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

// Tiles on their way: as many as leave an SM room for three CTAs (two of wide heads).
template <int D>
struct RowsSmem {
  static constexpr int kStages = D == 64 ? 4 : 3;
  alignas(128) uint16_t q[kRowTile * D];
  alignas(128) uint16_t k[kStages][kKeyTile * D];
  alignas(128) uint16_t v[kStages][kKeyTile * D];
  int pos[kStages][kKeyTile];
};

// kGroups 2: at most 32 rows, which two warps have for the first half of each tile's slots and two for the second.
template <class T, int D, int kGroups>
__global__ void __launch_bounds__(kAttendThreads) attend_rows_kernel(const AttendParams p) {
  constexpr int kStages = RowsSmem<D>::kStages, kKeys = kKeyTile / kGroups, kRowWarps = kAttendWarps / kGroups;
  constexpr int kRows = 16 * kRowWarps;
  extern __shared__ char raw[];
  RowsSmem<D>& sm = *reinterpret_cast<RowsSmem<D>*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  pdl_wait();
  pdl_launch_dependents();
  const int tiles_m = (p.M + kRows - 1) / kRows;
  long long id = blockIdx.x;
  const int split = static_cast<int>(id % p.splits);
  id /= p.splits;
  const int m0 = static_cast<int>(id % tiles_m) * kRows;
  id /= tiles_m;
  const int hk = static_cast<int>(id % p.Hk), b = static_cast<int>(id / p.Hk);
  const int g = hk / (p.Hk / p.G);
  const ListOf l = list_of(p, b, g);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row0 = warp % kRowWarps * 16, key0 = warp / kRowWarps * kKeys;   // of the tiles
  const int rows_m = l.rows * p.R;
  const int tiles = (l.n + kKeyTile - 1) / kKeyTile, per = (tiles + p.splits - 1) / p.splits;
  const int t0 = min(split * per, tiles), t1 = m0 < rows_m ? min(t0 + per, tiles) : t0;
  const uint16_t* kh = p.k + b * p.stride_b + hk * p.stride_h;
  const uint16_t* vh = p.v + b * p.stride_b + hk * p.stride_h;
  const int32_t* pos = p.pos + (static_cast<long long>(b) * p.G + g) * p.C;
  const uint32_t sq = smem_u32(sm.q);
  float* scores = p.scores + (static_cast<long long>(b) * p.Hk + hk) * p.M * p.pitch;

  auto load = [&](int tile) {
    if (tile < t1) {
      const int j0 = tile * kKeyTile, s = (tile - t0) % kStages;
      load_keys<D>(p, kh, j0, l.n, smem_u32(sm.k[s]));
      load_keys<D>(p, vh, j0, l.n, smem_u32(sm.v[s]));
      if (threadIdx.x < kKeyTile) {
        const int j = j0 + threadIdx.x;
        cp_async4(smem_u32(&sm.pos[s][threadIdx.x]), pos + min(j, l.n - 1), j < l.n);
      }
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
  for (int u = 0; u < 2; ++u) at[u] = l.first + (m0 + row0 + (lane >> 2) + 8 * u) / p.R;
  const int last = l.first + min(m0 + kRows - 1, rows_m - 1) / p.R;   // the latest row of the tile,
  const int first_at = l.first + (m0 + row0) / p.R;                   // and the warp's earliest

  if (t0 < t1) load_q<D>(p, b, hk, m0, l.rows, kRows, sq);
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) load(t0 + i);
  for (int tile = t0; tile < t1; ++tile) {
    const int s = (tile - t0) % kStages;
    cp_async_wait<kStages - 2>();
    // a slot that no row of the tile sees may hold anything: its V is taken as 0
    bool unseen = false;
    if (threadIdx.x < kKeyTile) {
      const int at_key = sm.pos[s][threadIdx.x];
      unseen = tile * kKeyTile + static_cast<int>(threadIdx.x) >= l.n || at_key < 0 || at_key > last;
    }
    const int hidden = __syncthreads_count(unseen);   // (and the tile before this one is done with)
    load(tile + kStages - 1);
    if (hidden == kKeyTile) {
      if (kGroups == 2 || p.stored) {   // (the sums read every score)
        const int j = tile * kKeyTile + static_cast<int>(threadIdx.x) % kKeyTile;
        for (int m = m0 + threadIdx.x / kKeyTile; m < min(rows_m, m0 + kRows) && j < l.n; m += kAttendThreads / kKeyTile)
          scores[static_cast<long long>(m) * p.pitch + j] = -INFINITY;
      }
      continue;
    }
    if (hidden != 0) {
      if (unseen)
        for (int c = 0; c < D / 8; ++c)
          *reinterpret_cast<uint4*>(reinterpret_cast<char*>(sm.v[s]) + threadIdx.x * D * 2 + c * 16) = make_uint4(0, 0, 0, 0);
      __syncthreads();
    }
    if (m0 + row0 >= rows_m) continue;   // a warp without rows
    const uint32_t sk = smem_u32(sm.k[s]), sv = smem_u32(sm.v[s]);
    float c[kKeys / 8][4];
#pragma unroll
    for (int i = 0; i < kKeys / 8; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] = 0.f;
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t a[4];
      load_a<D>(sq, row0, k, lane, a);
#pragma unroll
      for (int n = 0; n < kKeys / 16; ++n) {
        uint32_t f[4];
        load_b<D>(sk, key0 + n * 16, k, lane, f);
        T::mma(c[2 * n], a, f[0], f[1]);
        T::mma(c[2 * n + 1], a, f[2], f[3]);
      }
    }
    float top[2] = {ref[0], ref[1]};
    // whether every row sees every slot of the tile: looked up once for the tile, not for each score
    const int w0 = sm.pos[s][lane], w1 = sm.pos[s][32 + lane];
    const bool whole = __all_sync(0xffffffffu, (tile + 1) * kKeyTile <= l.n && w0 >= 0 && w0 <= first_at && w1 >= 0 && w1 <= first_at);
#pragma unroll
    for (int i = 0; i < kKeys / 8; ++i) {
      const int key = key0 + 8 * i + 2 * (lane & 3);
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] *= p.scale2;
      if (!whole) {
        const int2 where = *reinterpret_cast<const int2*>(&sm.pos[s][key]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int w = k & 1 ? where.y : where.x;
          const bool sees = tile * kKeyTile + key + (k & 1) < l.n && w >= 0 && w <= at[k >> 1];
          c[i][k] = sees ? c[i][k] : -INFINITY;
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) top[k >> 1] = fmaxf(top[k >> 1], c[i][k] - T::kHeadroom);
      if (kGroups == 2 || p.stored) store_scores(p, scores, m0 + row0, rows_m, tile * kKeyTile + key, l.n, c[i]);
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
    if (__any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        o[i][0] *= keep[0];
        o[i][1] *= keep[0];
        o[i][2] *= keep[1];
        o[i][3] *= keep[1];
      }
    }
#pragma unroll
    for (int i = 0; i < kKeys / 8; ++i) {
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] = ex2(c[i][k] - top[k >> 1]);
      sum[0] += c[i][0] + c[i][1];
      sum[1] += c[i][2] + c[i][3];
    }
#pragma unroll
    for (int k = 0; k < kKeys / 16; ++k) {
      uint32_t a[4], rest[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) T::split(c[2 * k + i / 2][i % 2 * 2], c[2 * k + i / 2][i % 2 * 2 + 1], a[i], rest[i]);
      add_values<T, D>(o, a, rest, sv, key0 + k * 16, lane);
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 1);
    sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 2);
  }
  if (kGroups == 2) {   // the second half's warps hand theirs over
    cp_async_wait_all();
    __syncthreads();
    constexpr int kPitch = D + 8;
    float2* ends = reinterpret_cast<float2*>(sm.v);
    float* part = reinterpret_cast<float*>(sm.k);
    static_assert(sizeof(sm.k) >= kRows * kPitch * 4, "room for the second half's O");
    if (warp >= kRowWarps) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int m = row0 + (lane >> 2) + 8 * u;
        if ((lane & 3) == 0) ends[m] = make_float2(ref[u], sum[u]);
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
          *reinterpret_cast<float2*>(part + m * kPitch + 8 * i + 2 * (lane & 3)) = make_float2(o[i][2 * u], o[i][2 * u + 1]);
      }
    }
    __syncthreads();
    if (warp >= kRowWarps) return;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int m = row0 + (lane >> 2) + 8 * u;
      const float2 end = ends[m];
      const float top = fmaxf(ref[u], end.x);
      const float mine = ref[u] == top ? 1.f : ex2(ref[u] - top), other = end.x == top ? 1.f : ex2(end.x - top);
      ref[u] = top;
      sum[u] = mine * sum[u] + other * end.y;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        const float2 f = *reinterpret_cast<const float2*>(part + m * kPitch + 8 * i + 2 * (lane & 3));
        o[i][2 * u] = mine * o[i][2 * u] + other * f.x;
        o[i][2 * u + 1] = mine * o[i][2 * u + 1] + other * f.y;
      }
    }
  }
  const long long unit = static_cast<long long>(b) * p.Hk + hk;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int m = m0 + row0 + (lane >> 2) + 8 * u;
    if (m >= rows_m) continue;
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
  const int m = static_cast<int>(row - unit * p.M), b = static_cast<int>(unit / p.Hk);
  const int hk = static_cast<int>(unit - static_cast<long long>(b) * p.Hk);
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
  static constexpr int kTiles = sum_tiles(D), kSlots = kTiles * kKeyTile;
  alignas(128) uint16_t k[kSlots * D];
  alignas(128) uint16_t q[2][kRowTile * D];
  int pos[kSlots];
  int least[kTiles], most[kTiles];   // the least and the greatest position of each tile's slots
  float sum[kAttendWarps][kSlots];   // by 16 rows of a row tile
};

// A CTA has a stretch of a key head's slots: the weights of its rows, or of one of `row_parts` parts of them.  The keys
// stay in shared memory while the rows pass, a tile of them at a time.
template <class T, int D>
__global__ void __launch_bounds__(kAttendThreads) attend_sums_kernel(const AttendParams p) {
  using S = SumsSmem<D>;
  constexpr int kRows = kRowTile;
  extern __shared__ char raw[];
  S& sm = *reinterpret_cast<S*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~uintptr_t(127));
  pdl_wait();
  pdl_launch_dependents();
  const int pieces = (p.C + S::kSlots - 1) / S::kSlots;
  const int piece = blockIdx.x % pieces, part = blockIdx.x / pieces % p.row_parts, unit = blockIdx.x / pieces / p.row_parts;
  const int b = unit / p.Hk, hk = unit - b * p.Hk, list = b * p.G + hk / (p.Hk / p.G);
  const ListOf l = list_of(p, b, list - b * p.G);
  const int j0 = piece * S::kSlots, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (j0 >= l.n || l.rows == 0) return;
  const long long at0 = static_cast<long long>(list) * p.C + j0;
  const int rows_m = l.rows * p.R, tiles_m = (rows_m + kRows - 1) / kRows, per = (tiles_m + p.row_parts - 1) / p.row_parts;
  const int step0 = min(part * per, tiles_m), step1 = min(step0 + per, tiles_m);
  const int row0 = warp * 16, tiles = min(S::kTiles, (l.n - j0 + kKeyTile - 1) / kKeyTile);
  auto load = [&](int step) {
    load_q<D>(p, b, hk, step * kRows, l.rows, kRows, smem_u32(sm.q[step & 1]));
  };
  for (int t = 0; t < tiles; ++t)
    load_keys<D>(p, p.k + b * p.stride_b + hk * p.stride_h, j0 + t * kKeyTile, l.n, smem_u32(sm.k + t * kKeyTile * D));
  if (step0 < step1) load(step0);
  cp_async_commit();
  for (int t = warp; t < S::kTiles; t += kAttendWarps) {
    int least = 0x7fffffff, most = 0;
    for (int j = t * kKeyTile + lane; j < (t + 1) * kKeyTile; j += 32) {
      const int where = j0 + j < l.n ? p.pos[at0 + j] : -1;
      sm.pos[j] = where < 0 ? 0x7fffffff : where;   // (seen by no row)
      least = min(least, sm.pos[j]);
      most = max(most, sm.pos[j]);
    }
    least = __reduce_min_sync(0xffffffffu, least);
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 0) {
      sm.least[t] = least;
      sm.most[t] = most;
    }
  }
  for (int i = threadIdx.x; i < kAttendWarps * S::kSlots; i += kAttendThreads) (&sm.sum[0][0])[i] = 0.f;
  for (int step = step0; step < step1; ++step) {
    const int m0 = step * kRows;
    float lse[2];
    int at[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int m = m0 + row0 + (lane >> 2) + 8 * u;
      lse[u] = m < rows_m ? p.lse[static_cast<long long>(unit) * p.M + m] : INFINITY;
      at[u] = m < rows_m ? l.first + m / p.R : -1;
    }
    cp_async_wait_all();
    __syncthreads();
    if (step + 1 < step1) load(step + 1);
    cp_async_commit();
    const uint32_t sq = smem_u32(sm.q[step & 1]);
    const int last = l.first + min(m0 + kRows - 1, rows_m - 1) / p.R, first_at = l.first + (m0 + row0) / p.R;
    if (m0 + row0 < rows_m) {
      uint32_t a[D / 16][4];
#pragma unroll
      for (int k = 0; k < D / 16; ++k) load_a<D>(sq, row0, k, lane, a[k]);
      for (int t = 0; t < tiles; ++t) {
        if (sm.least[t] > last) continue;
        const bool whole = sm.most[t] <= first_at;   // (every row of the warp sees every slot)
        const uint32_t sk = smem_u32(sm.k + t * kKeyTile * D);
        float c[kKeyTile / 8][4];
#pragma unroll
        for (int i = 0; i < kKeyTile / 8; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) c[i][k] = 0.f;
#pragma unroll
        for (int k = 0; k < D / 16; ++k)
#pragma unroll
          for (int n = 0; n < kKeyTile / 16; ++n) {
            uint32_t f[4];
            load_b<D>(sk, n * 16, k, lane, f);
            T::mma(c[2 * n], a[k], f[0], f[1]);
            T::mma(c[2 * n + 1], a[k], f[2], f[3]);
          }
#pragma unroll
        for (int i = 0; i < kKeyTile / 8; ++i) {
          const int key = t * kKeyTile + 8 * i + 2 * (lane & 3);
          float v[2];
          if (whole) {
            v[0] = ex2(c[i][0] * p.scale2 - lse[0]) + ex2(c[i][2] * p.scale2 - lse[1]);
            v[1] = ex2(c[i][1] * p.scale2 - lse[0]) + ex2(c[i][3] * p.scale2 - lse[1]);
          } else {   // (a NaN of an unseen slot is kept out by the choice, not by a product)
            const int2 where = *reinterpret_cast<const int2*>(&sm.pos[key]);
            v[0] = (where.x <= at[0] ? ex2(c[i][0] * p.scale2 - lse[0]) : 0.f) +
                   (where.x <= at[1] ? ex2(c[i][2] * p.scale2 - lse[1]) : 0.f);
            v[1] = (where.y <= at[0] ? ex2(c[i][1] * p.scale2 - lse[0]) : 0.f) +
                   (where.y <= at[1] ? ex2(c[i][3] * p.scale2 - lse[1]) : 0.f);
          }
          // over the warp's other rows: lanes four apart
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            v[k] += __shfl_xor_sync(0xffffffffu, v[k], 4);
            v[k] += __shfl_xor_sync(0xffffffffu, v[k], 8);
            v[k] += __shfl_xor_sync(0xffffffffu, v[k], 16);
          }
          if (lane < 4) {
            float2* to = reinterpret_cast<float2*>(&sm.sum[warp][key]);
            const float2 old = *to;
            *to = make_float2(old.x + v[0], old.y + v[1]);
          }
        }
      }
    }
  }
  __syncthreads();
  for (int j = threadIdx.x; j < S::kSlots && j0 + j < l.n; j += kAttendThreads) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kAttendWarps; ++w) v += sm.sum[w][j];
    p.sums[(static_cast<long long>(unit) * p.row_parts + part) * p.pitch + j0 + j] = v;
  }
}

// A list's slots, one a thread: the sums of its heads and their parts, in order.
__global__ void __launch_bounds__(256) attend_heads_kernel(const AttendParams p) {
  pdl_wait();
  pdl_launch_dependents();
  const int pieces = (p.C + 255) / 256, list = blockIdx.x / pieces, b = list / p.G, g = list - b * p.G, of = p.Hk / p.G;
  const int j = (blockIdx.x - list * pieces) * 256 + static_cast<int>(threadIdx.x);
  const ListOf l = list_of(p, b, g);
  if (j >= l.n) return;
  const long long at = static_cast<long long>(list) * p.C + j;
  const float* sums = p.sums + (static_cast<long long>(b) * p.Hk + g * of) * p.row_parts * p.pitch + j;
  float v = 0.f;
  if (l.rows > 0) {
#pragma unroll 8
    for (int h = 0; h < of * p.row_parts; ++h) v += sums[static_cast<long long>(h) * p.pitch];
  }
  p.acc_out[at] = l.rows > 0 ? p.decay * p.acc[at] + v / static_cast<float>(p.H / p.G) : p.acc[at];
}

// Slots of a list whose scores are kept and whose rows' LSE are known: eight warps have every eighth row each of 128
// slots, and their sums are added in order.
constexpr int kStoredSlots = 128;
__global__ void __launch_bounds__(256) attend_stored_sums_kernel(const AttendParams p) {
  __shared__ float4 part[8][kStoredSlots / 4];
  pdl_wait();
  pdl_launch_dependents();
  const int pieces = (p.C + kStoredSlots - 1) / kStoredSlots, list = blockIdx.x / pieces, b = list / p.G, g = list - b * p.G;
  const int of = p.Hk / p.G, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int j0 = (blockIdx.x - list * pieces) * kStoredSlots, j = j0 + 4 * lane;
  const ListOf l = list_of(p, b, g);
  if (j0 >= l.n) return;
  const int rows_m = l.rows * p.R, rows = of * rows_m;
  const long long unit0 = static_cast<long long>(b) * p.Hk + g * of, at = static_cast<long long>(list) * p.C + j0 + threadIdx.x;
  const bool mine = threadIdx.x < kStoredSlots && j0 + static_cast<int>(threadIdx.x) < l.n;
  const float old = mine ? p.acc[at] : 0.f;
  float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int kAhead = 8;
  if (j < l.n)
    for (int r0 = warp; r0 < rows; r0 += 8 * kAhead) {
      float4 t[kAhead];
      float x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int r = r0 + 8 * u, h = r / rows_m;
        const long long row = (unit0 + h) * p.M + r - h * rows_m;
        x[u] = INFINITY;
        t[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) {
          x[u] = p.lse[row];
          t[u] = *reinterpret_cast<const float4*>(p.scores + row * p.pitch + j);
        }
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        sum.x += ex2(t[u].x - x[u]);
        sum.y += ex2(t[u].y - x[u]);
        sum.z += ex2(t[u].z - x[u]);
        sum.w += ex2(t[u].w - x[u]);
      }
    }
  part[warp][lane] = sum;
  __syncthreads();
  if (!mine) return;
  float v = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) v += reinterpret_cast<const float*>(part[w])[threadIdx.x];
  p.acc_out[at] = l.rows > 0 ? p.decay * old + v / static_cast<float>(p.H / p.G) : old;
}

// ---------------------------------------------------------------------------
// few rows: a warp's tiles
// ---------------------------------------------------------------------------
// A unit is a key head of a sequence.  The tiles of all units, one behind the other, are dealt out to the warps in
// equal runs, whatever the lengths of the lists; a warp's piece of a unit has the number warp + unit, which no
// other has (from a piece to the next one, at least one of the two goes up).
__device__ __forceinline__ int list_tiles(const AttendParams& p, int list) {
  const int rows = p.rows != nullptr ? p.rows[list / p.G] : p.T;
  const int n = min(max(p.len[list], 0), p.C);
  return rows > 0 ? (n + kFewTile - 1) / kFewTile : 0;
}

// Where a warp's run is: list, head of the list, tile of the head.
struct Cursor {
  int list, head, tile, tiles;
};

__device__ __forceinline__ void next_list(const AttendParams& p, Cursor& c) {
  const int lists = p.B * p.G;
  c.head = c.tile = 0;
  do {
    ++c.list;
    c.tiles = c.list < lists ? list_tiles(p, c.list) : 1;
  } while (c.tiles == 0);
}

__device__ __forceinline__ void advance(const AttendParams& p, int of, Cursor& c) {
  if (++c.tile < c.tiles) return;
  c.tile = 0;
  if (++c.head == of) next_list(p, c);
}

template <int D>
struct FewShape {
  static constexpr int kStages = D == 64 ? 4 : 3;
  static constexpr int kTileBytes = kFewTile * D * 2;
  static constexpr int kStageBytes = 2 * kTileBytes + kFewTile * 4;
  static constexpr int kWarpBytes = kStages * kStageBytes;
  static constexpr int kWarps = few_warps_sm(D);     // a CTA, which has an SM to itself
  static constexpr int kThreads = kWarps * 32;
  static constexpr int kPitch = D + 8;               // floats of a row of O in shared memory: rows in different banks
  static constexpr int kBytes = kWarps * kWarpBytes + 128;
};
static_assert(FewShape<64>::kWarpBytes >= kFewRows * FewShape<64>::kPitch * 4 && FewShape<64>::kBytes <= 230000 &&
              FewShape<128>::kWarpBytes >= kFewRows * FewShape<128>::kPitch * 4 && FewShape<128>::kBytes <= 230000,
              "a warp's stages hold its O, and an SM the stages");

template <class T, int D>
__global__ void __launch_bounds__(FewShape<D>::kThreads, 1) attend_few_kernel(const AttendParams p) {
  using S = FewShape<D>;
  extern __shared__ char raw[];
  __shared__ int units[S::kWarps];
  __shared__ float2 ends[S::kWarps][kFewRows];   // reference and sum of the rows of each warp's last piece
  const int lane = threadIdx.x & 31, me = threadIdx.x >> 5, warp = blockIdx.x * S::kWarps + me;
  const uint32_t all = (smem_u32(raw) + 127) & ~127u, mine = all + me * S::kWarpBytes;
  char* own = raw + (mine - smem_u32(raw));
  pdl_wait();
  pdl_launch_dependents();
  const int of = p.Hk / p.G, lists = p.B * p.G;
  // the run: all tiles, then the list in which it starts
  int total = 0;
  for (int i = lane; i < lists; i += 32) total += list_tiles(p, i);
  total = __reduce_add_sync(0xffffffffu, total) * of;
  const int share = max(kFewMinTiles, (total + p.warps - 1) / p.warps);
  if (warp == 0 && lane == 0) p.share[0] = share;
  const int from = min(warp * share, total), count = min(share, total - from);
  Cursor at{};
  if (count > 0) {
    int before = 0;   // tiles of the lists before i
    for (int i = 0;; i += 32) {
      const int t = i + lane < lists ? list_tiles(p, i + lane) * of : 0;
      int upto = t;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const unsigned there = __ballot_sync(0xffffffffu, before + upto > from);
      if (there != 0) {
        const int l = __ffs(there) - 1;
        const int tiles = __shfl_sync(0xffffffffu, t, l) / of;
        const int rest = from - before - (__shfl_sync(0xffffffffu, upto, l) - tiles * of);
        at.list = i + l;
        at.tiles = tiles;
        at.head = rest / tiles;
        at.tile = rest - at.head * tiles;
        break;
      }
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
  }
  Cursor ahead = at;
  int to_load = count, loaded = 0;
  // this lane's chunks of a tile: rows lane / (D / 8) + ..., chunk lane % (D / 8)
  constexpr int kLanesRow = D / 8, kRowsOnce = 32 / kLanesRow;
  const int row0 = lane / kLanesRow, chunk = lane % kLanesRow;
  auto load = [&]() {
    if (to_load > 0) {
      const int b = ahead.list / p.G, g = ahead.list - b * p.G, hk = g * of + ahead.head;
      const int n = min(p.len[ahead.list], p.C), j0 = ahead.tile * kFewTile;
      const uint32_t base = mine + (loaded % S::kStages) * S::kStageBytes;
      const long long head = b * p.stride_b + hk * p.stride_h + j0 * p.stride_c + chunk * 8;
#pragma unroll
      for (int i = 0; i < kFewTile / kRowsOnce; ++i) {
        const int row = row0 + i * kRowsOnce;
        const bool live = j0 + row < n;
        const long long off = live ? head + row * p.stride_c : 0;
        cp_async16(chunk_at<D>(base, row, chunk), p.k + off, live);
        cp_async16(chunk_at<D>(base + S::kTileBytes, row, chunk), p.v + off, live);
      }
      if (lane < kFewTile) {
        const bool live = j0 + lane < n;
        cp_async4(base + 2 * S::kTileBytes + lane * 4, p.pos + static_cast<long long>(ahead.list) * p.C + (live ? j0 + lane : 0), live);
      }
      --to_load;
      ++loaded;
      advance(p, of, ahead);
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < S::kStages - 1; ++i) load();

  uint32_t q[D / 16][4];
  float o[D / 8][4], ref[2], sum[2];
  int seen_to[2], last = 0, unit = -1, n = 0, rows_m = 0;
  bool fresh = true;
  for (int step = 0; step < count; ++step) {
    if (fresh) {
      fresh = false;
      const int b = at.list / p.G, g = at.list - b * p.G, hk = g * of + at.head;
      const ListOf l = list_of(p, b, g);
      unit = b * p.Hk + hk;
      n = l.n;
      rows_m = l.rows * p.R;
      last = l.first + l.rows - 1;
      if (at.tile == 0 && lane == 0) p.share[1 + unit] = from + step;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int m = (lane >> 2) + 8 * u, tok = m / p.R;
        seen_to[u] = l.first + tok;
        const bool live = m < rows_m;
        const uint32_t* src = reinterpret_cast<const uint32_t*>(
            p.q + (static_cast<long long>(b) * p.T + (live ? tok : 0)) * p.ldq + (hk * p.R + (live ? m % p.R : 0)) * D) + (lane & 3);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          q[k][u] = live ? src[8 * k] : 0u;
          q[k][2 + u] = live ? src[8 * k + 4] : 0u;
        }
        ref[u] = -INFINITY;
        sum[u] = 0.f;
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
    }
    load();
    cp_async_wait<S::kStages - 1>();
    const uint32_t sk = mine + (step % S::kStages) * S::kStageBytes, sv = sk + S::kTileBytes;
    char* stage = own + (step % S::kStages) * S::kStageBytes;
    const int j0 = at.tile * kFewTile;
    // a slot that no row sees may hold anything: its V is taken as 0
    bool unseen = false;
    if (lane < kFewTile) {
      const int where = reinterpret_cast<const int*>(stage + 2 * S::kTileBytes)[lane];
      unseen = j0 + lane < n && (where < 0 || where > last);
    }
    __syncwarp();
    const unsigned blank = __ballot_sync(0xffffffffu, unseen);
    if (blank != 0) {
      for (int r = 0; r < kFewTile; ++r)
        if (blank >> r & 1u && lane < D / 8)
          *reinterpret_cast<uint4*>(stage + S::kTileBytes + r * D * 2 + lane * 16) = make_uint4(0, 0, 0, 0);
      __syncwarp();
    }
    float c[2][4] = {};
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
      uint32_t f[4];
      load_b<D>(sk, 0, k, lane, f);
      T::mma(c[0], q[k], f[0], f[1]);
      T::mma(c[1], q[k], f[2], f[3]);
    }
    float top[2] = {ref[0], ref[1]};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int key = 8 * i + 2 * (lane & 3);
      const int2 where = *reinterpret_cast<const int2*>(stage + 2 * S::kTileBytes + key * 4);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int w = k & 1 ? where.y : where.x;
        const bool sees = j0 + key + (k & 1) < n && w >= 0 && w <= seen_to[k >> 1];
        c[i][k] = sees ? c[i][k] * p.scale2 : -INFINITY;
        top[k >> 1] = fmaxf(top[k >> 1], c[i][k] - T::kHeadroom);
      }
      store_scores(p, p.scores + static_cast<long long>(unit) * p.M * p.pitch, 0, rows_m, j0 + key, n, c[i]);
    }
    bool moved = false;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 1));
      top[u] = fmaxf(top[u], __shfl_xor_sync(0xffffffffu, top[u], 2));
      moved |= top[u] != ref[u];
    }
    if (__any_sync(0xffffffffu, moved)) {
      float keep[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        keep[u] = top[u] == ref[u] ? 1.f : ex2(ref[u] - top[u]);   // (both -inf: nothing so far)
        ref[u] = top[u];
        sum[u] *= keep[u];
      }
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        o[i][0] *= keep[0];
        o[i][1] *= keep[0];
        o[i][2] *= keep[1];
        o[i][3] *= keep[1];
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) top[u] = ref[u] == -INFINITY ? 0.f : ref[u];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int k = 0; k < 4; ++k) c[i][k] = ex2(c[i][k] - top[k >> 1]);
      sum[0] += c[i][0] + c[i][1];
      sum[1] += c[i][2] + c[i][3];
    }
    uint32_t a[4], rest[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) T::split(c[i / 2][i % 2 * 2], c[i / 2][i % 2 * 2 + 1], a[i], rest[i]);
    add_values<T, D>(o, a, rest, sv, 0, lane);
    __syncwarp();   // the stage is free
    const int was_list = at.list, was_head = at.head;
    advance(p, of, at);
    if (step + 1 == count || (at.list == was_list && at.head == was_head)) continue;
    // the unit goes on in other warps at most: what this one has of it
    fresh = true;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 1);
      sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 2);
      const int m = (lane >> 2) + 8 * u;
      if (m >= rows_m) continue;
      const long long at_row = (static_cast<long long>(warp) + unit) * p.M + m;
      if ((lane & 3) == 0) p.ml[at_row] = make_float2(ref[u], sum[u]);
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
        *reinterpret_cast<float2*>(p.part + at_row * D + 8 * i + 2 * (lane & 3)) = make_float2(o[i][2 * u], o[i][2 * u + 1]);
    }
  }
  // The warps' last pieces, joined where neighbours have the same unit: the first of them writes one piece, the
  // others' are empty.
  cp_async_wait_all();   // (none is left but empty groups)
  if (unit >= 0) {
    float* mo = reinterpret_cast<float*>(own);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 1);
      sum[u] += __shfl_xor_sync(0xffffffffu, sum[u], 2);
      const int m = (lane >> 2) + 8 * u;
      if ((lane & 3) == 0) ends[me][m] = make_float2(ref[u], sum[u]);
#pragma unroll
      for (int i = 0; i < D / 8; ++i)
        *reinterpret_cast<float2*>(mo + m * S::kPitch + 8 * i + 2 * (lane & 3)) = make_float2(o[i][2 * u], o[i][2 * u + 1]);
    }
  }
  if (lane == 0) units[me] = unit;
  __syncthreads();
  if (unit < 0) return;
  int w0 = me, w1 = me + 1;
  while (w0 > 0 && units[w0 - 1] == unit) --w0;
  while (w1 < S::kWarps && units[w1] == unit) ++w1;
  for (int m = lane; m < rows_m; m += 32)
    if (me != w0) p.ml[(static_cast<long long>(warp) + unit) * p.M + m] = make_float2(-INFINITY, 0.f);
  const float* first = reinterpret_cast<const float*>(raw + (all - smem_u32(raw)));
  const long long to_row = (static_cast<long long>(blockIdx.x) * S::kWarps + w0 + unit) * p.M;
  for (int e = (me - w0) * 32 + lane; e < rows_m * (D / 4); e += (w1 - w0) * 32) {
    const int m = e / (D / 4), c = e % (D / 4) * 4;
    float top = -INFINITY, total = 0.f;
    for (int w = w0; w < w1; ++w) top = fmaxf(top, ends[w][m].x);
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w = w0; w < w1; ++w) {
      const float2 end = ends[w][m];
      const float k = end.x == top ? 1.f : end.x == -INFINITY && end.y == 0.f ? 0.f : ex2(end.x - top);
      const float4 f = *reinterpret_cast<const float4*>(first + w * (S::kWarpBytes / 4) + m * S::kPitch + c);
      v.x += k * f.x;
      v.y += k * f.y;
      v.z += k * f.z;
      v.w += k * f.w;
      total += k * end.y;
    }
    *reinterpret_cast<float4*>(p.part + (to_row + m) * D + c) = v;
    if (c == 0) p.ml[to_row + m] = make_float2(top, total);
  }
}

// The warps that have parts of a unit: all that write one in its first and its last CTA, and the first of each CTA in
// between, which has the unit in all its warps.
template <int kWarps>
struct Pieces {
  int unit, w0, first, between, count;
  __device__ __forceinline__ Pieces(int unit_, int n, int share, int from) : unit(unit_) {
    const int tiles = (n + kFewTile - 1) / kFewTile;
    if (tiles == 0) {
      w0 = first = between = count = 0;
      return;
    }
    w0 = from / share;
    const int w1 = (from + tiles - 1) / share, c0 = w0 / kWarps, c1 = w1 / kWarps;
    first = min(w1, c0 * kWarps + kWarps - 1) - w0 + 1;
    between = c1 > c0 ? c1 - c0 - 1 : 0;
    count = first + between + (c1 > c0 ? w1 - c1 * kWarps + 1 : 0);
  }
  // the number of part i
  __device__ __forceinline__ long long at(int i) const {
    const int c = w0 / kWarps + 1;   // the CTA after the first
    const int w = i < first ? w0 + i : i < first + between ? (c + i - first) * kWarps : (c + between) * kWarps + i - first - between;
    return static_cast<long long>(w) + unit;
  }
};

// The parts that CTAs of at most 32 rows make of a unit.
struct SplitPieces {
  int unit, count;
  __device__ __forceinline__ SplitPieces(int unit_, int splits) : unit(unit_), count(splits) {}
  __device__ __forceinline__ long long at(int i) const { return static_cast<long long>(unit) * count + i; }
};
// kWarps: of attend_few_kernel's CTAs, or 0 for the parts of attend_rows_kernel
template <int kWarps>
__device__ __forceinline__ auto parts_of(const AttendParams& p, int unit, int n, int share) {
  if constexpr (kWarps == 0)
    return SplitPieces(unit, p.splits);
  else
    return Pieces<kWarps>(unit, n, share, __ldcg(p.share + 1 + unit));
}

// The first `row_ctas` CTAs join rows, one each or, with many rows (`together`), a warp a row; the others have kSumSlots
// slots of a list each, whose weights they add up over the list's rows from the scores and the rows' LSE.
constexpr int kSumThreads = 128, kSumWarps = kSumThreads / 32;
constexpr int kSumSlots = kSumThreads * 4;
constexpr int kSumAhead = 8;
constexpr int kSumRows = kSumThreads / 4;   // most rows whose LSE are found at once, by four lanes each or more
template <class T, int D, int kWarps>
__global__ void __launch_bounds__(kSumThreads, 6) attend_stored_join_kernel(const AttendParams p, int row_ctas, int together) {
  constexpr int kOwn = D / 32;
  __shared__ float part[kSumWarps][D];
  __shared__ float2 ends[kSumWarps];
  __shared__ float lse[kSumRows];
  pdl_wait();
  pdl_launch_dependents();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int share = kWarps != 0 ? __ldcg(p.share) : 0;
  if (static_cast<int>(blockIdx.x) < row_ctas) {
    const int row = together ? static_cast<int>(blockIdx.x) * kSumWarps + warp : static_cast<int>(blockIdx.x);
    const int unit = row / p.M, m = row - unit * p.M;
    if (unit >= p.B * p.Hk) return;
    const int b = unit / p.Hk, hk = unit - b * p.Hk;
    const ListOf l = list_of(p, b, hk / (p.Hk / p.G));
    if (m >= l.rows * p.R) return;
    const auto ps = parts_of<kWarps>(p, unit, l.n, share);
    float ref = -INFINITY, total = 0.f, o[kOwn] = {};
    // eight parts a warp at a time
    for (int s0 = together ? 0 : warp * 8; s0 < ps.count; s0 += together ? 8 : kSumWarps * 8) {
      const int s = s0 + (lane & 7);
      const float2 ml = s < ps.count ? p.ml[ps.at(s) * p.M + m] : make_float2(-INFINITY, 0.f);
      const bool some = ml.x != -INFINITY || ml.y != 0.f;   // (nothing but NaN: the sum is one)
      // (asked for before it is known which are empty: theirs hold anything)
      float2 f[8][kOwn / 2];
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int i = 0; i < kOwn; i += 2)
          f[u][i / 2] = s0 + u < ps.count ? *reinterpret_cast<const float2*>(p.part + (ps.at(s0 + u) * p.M + m) * D + lane * kOwn + i)
                                          : make_float2(0.f, 0.f);
      const unsigned have = __ballot_sync(0xffffffffu, some) & 0xffu;
      float top = fmaxf(ref, ml.x);
#pragma unroll
      for (int i = 4; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, i));
      const float w = !some ? 0.f : ml.x == top ? 1.f : ex2(ml.x - top);
      const float keep = ref == top ? 1.f : ex2(ref - top);
      ref = top;
      total = total * keep + (some ? w * ml.y : 0.f);   // of the parts lane & 7, + 8 ..
#pragma unroll
      for (int i = 0; i < kOwn; ++i) o[i] *= keep;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const float wu = __shfl_sync(0xffffffffu, w, u);
        if (!(have >> u & 1u)) continue;
#pragma unroll
        for (int i = 0; i < kOwn; i += 2) {
          o[i] += wu * f[u][i / 2].x;
          o[i + 1] += wu * f[u][i / 2].y;
        }
      }
    }
#pragma unroll
    for (int i = 4; i > 0; i >>= 1) total += __shfl_xor_sync(0xffffffffu, total, i);
    uint16_t* out = p.o + (static_cast<long long>(b) * p.T + m / p.R) * p.ldo + static_cast<long long>(hk * p.R + m % p.R) * D;
    if (together) {
      const float inv = ref == -INFINITY && total == 0.f ? 0.f : 1.f / total;
#pragma unroll
      for (int i = 0; i < kOwn; i += 2) reinterpret_cast<uint32_t*>(out)[(lane * kOwn + i) / 2] = T::pack(o[i] * inv, o[i + 1] * inv);
      return;
    }
    if (lane == 0) ends[warp] = make_float2(ref, total);
#pragma unroll
    for (int i = 0; i < kOwn; ++i) part[warp][lane * kOwn + i] = o[i];
    __syncthreads();
    if (static_cast<int>(threadIdx.x) >= D / 2) return;
    float top = -INFINITY, sum = 0.f, v[2] = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kSumWarps; ++w) top = fmaxf(top, ends[w].x);
#pragma unroll
    for (int w = 0; w < kSumWarps; ++w) {
      const float2 end = ends[w];
      const float k = end.x == top ? 1.f : end.x == -INFINITY && end.y == 0.f ? 0.f : ex2(end.x - top);
      sum += k * end.y;
      v[0] += k * part[w][2 * threadIdx.x];
      v[1] += k * part[w][2 * threadIdx.x + 1];
    }
    const float inv = top == -INFINITY && sum == 0.f ? 0.f : 1.f / sum;
    reinterpret_cast<uint32_t*>(out)[threadIdx.x] = T::pack(v[0] * inv, v[1] * inv);
    return;
  }
  const int chunks = (p.C + kSumSlots - 1) / kSumSlots, id = blockIdx.x - row_ctas;
  const int list = id / chunks, b = list / p.G, g = list - b * p.G, of = p.Hk / p.G, unit0 = b * p.Hk + g * of;
  const ListOf l = list_of(p, b, g);
  const int j0 = (id - list * chunks) * kSumSlots, j = j0 + static_cast<int>(threadIdx.x) * 4;
  if (j0 >= l.n) return;
  const int rows_m = l.rows * p.R, rows = of * rows_m;
  const long long at = static_cast<long long>(list) * p.C + j;
  float old[4] = {}, sum[4] = {};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (j + i < l.n) old[i] = p.acc[at + i];
  const int lanes = rows <= kSumThreads / 16 ? 16 : rows <= kSumThreads / 8 ? 8 : 4;   // of a row's LSE
  for (int r0 = 0; r0 < rows; r0 += kSumRows) {
    const int here = min(kSumRows, rows - r0), i = threadIdx.x / lanes;
    const int h = r0 / rows_m, m0 = r0 - h * rows_m;
    // the first rows' scores are asked for before the LSE are known
    const float* row = p.scores + (static_cast<long long>(unit0 + h) * p.M + m0) * p.pitch + j;
    int m = m0;
    auto next = [&]() {
      const float4 t = *reinterpret_cast<const float4*>(row);
      const bool end = ++m == rows_m;   // of the head's rows in use
      row += static_cast<long long>(end ? p.M - rows_m + 1 : 1) * p.pitch;
      m = end ? 0 : m;
      return t;
    };
    float4 ahead[kSumAhead];
#pragma unroll
    for (int k = 0; k < kSumAhead; ++k)
      if (k < here && j < l.n) ahead[k] = next();
    __syncthreads();
    // (whole warps: several rows each)
    const int mine = m0 + min(i, here - 1), hi = mine / rows_m, unit = unit0 + h + hi;
    const auto ps = parts_of<kWarps>(p, unit, l.n, share);
    float ref = -INFINITY, total = 0.f;
    for (int s0 = lane & (lanes - 1); s0 < ps.count; s0 += 4 * lanes) {
      float2 ml[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        ml[u] = s0 + lanes * u < ps.count ? p.ml[ps.at(s0 + lanes * u) * p.M + mine - hi * rows_m] : make_float2(-INFINITY, 0.f);
      const float top = fmaxf(fmaxf(fmaxf(ref, ml[0].x), fmaxf(ml[1].x, ml[2].x)), ml[3].x);
      total *= ref == top ? 1.f : ex2(ref - top);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (ml[u].x != -INFINITY || ml[u].y != 0.f) total += ml[u].y * (ml[u].x == top ? 1.f : ex2(ml[u].x - top));
      ref = top;
    }
    float top = ref;
    for (int k = lanes / 2; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, k));
    if (ref != top && (ref != -INFINITY || total != 0.f)) total *= ex2(ref - top);
    for (int k = lanes / 2; k > 0; k >>= 1) total += __shfl_xor_sync(0xffffffffu, total, k);
    if ((lane & (lanes - 1)) == 0 && i < here) lse[i] = top == -INFINITY && total == 0.f ? INFINITY : top + log2f(total);
    __syncthreads();
    if (j >= l.n) continue;
#pragma unroll
    for (int k = 0; k < kSumAhead; ++k)
      if (k < here) {
        sum[0] += ex2(ahead[k].x - lse[k]);
        sum[1] += ex2(ahead[k].y - lse[k]);
        sum[2] += ex2(ahead[k].z - lse[k]);
        sum[3] += ex2(ahead[k].w - lse[k]);
      }
#pragma unroll 4
    for (int k = kSumAhead; k < here; ++k) {
      const float4 t = next();
      sum[0] += ex2(t.x - lse[k]);
      sum[1] += ex2(t.y - lse[k]);
      sum[2] += ex2(t.z - lse[k]);
      sum[3] += ex2(t.w - lse[k]);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (j + i < l.n) p.acc_out[at + i] = l.rows > 0 ? p.decay * old[i] + sum[i] / static_cast<float>(p.H / p.G) : old[i];
}

namespace {

// launch_chained with the kernel's dynamic shared memory allowed
template <auto kKernel, typename... Args>
cudaError_t launch_with(dim3 grid, int threads, size_t bytes, cudaStream_t st, const Args&... args) {
  const cudaError_t e = allow_shared<kKernel>(bytes);
  return e == cudaSuccess ? launch_chained(kKernel, grid, dim3(threads), bytes, st, args...) : e;
}

template <class T, int D>
cudaError_t launch_of(const AttendParams& p, cudaStream_t st) {
  const long long units = static_cast<long long>(p.B) * p.Hk;
  const int tiles_m = (p.M + kRowTile - 1) / kRowTile;
  const dim3 rows(static_cast<unsigned>(units * tiles_m * p.splits));
  const size_t rows_bytes = sizeof(RowsSmem<D>) + 128;
  if (p.M <= kJoinedRows) {   // scores kept, rows and weights in one launch
    constexpr int kWarps = FewShape<D>::kWarps;
    const bool few = p.M <= kFewRows;
    cudaError_t e = few ? launch_with<attend_few_kernel<T, D>>(dim3(p.warps / kWarps), FewShape<D>::kThreads, FewShape<D>::kBytes, st, p)
                        : launch_with<attend_rows_kernel<T, D, 2>>(rows, kAttendThreads, rows_bytes, st, p);
    if (e != cudaSuccess) return e;
    const long long all_rows = units * p.M;
    const int together = all_rows > 2 * kCacheSms;
    const int row_ctas = static_cast<int>(together ? (all_rows + kSumWarps - 1) / kSumWarps : all_rows);
    const long long sums = static_cast<long long>(p.B) * p.G * ((p.C + kSumSlots - 1) / kSumSlots);
    const dim3 grid(static_cast<unsigned>(row_ctas + sums));
    return few ? launch_chained(attend_stored_join_kernel<T, D, kWarps>, grid, dim3(kSumThreads), 0, st, p, row_ctas, together)
               : launch_chained(attend_stored_join_kernel<T, D, 0>, grid, dim3(kSumThreads), 0, st, p, row_ctas, together);
  }
  cudaError_t e = launch_with<attend_rows_kernel<T, D, 1>>(rows, kAttendThreads, rows_bytes, st, p);
  if (e != cudaSuccess) return e;
  e = launch_chained(attend_join_kernel<T, D>, dim3(static_cast<unsigned>((units * p.M + kJoinWarps - 1) / kJoinWarps)),
                     dim3(kJoinWarps * 32), 0, st, p);
  if (e != cudaSuccess) return e;
  const long long lists = static_cast<long long>(p.B) * p.G;
  if (p.stored)
    return launch_chained(attend_stored_sums_kernel, dim3(static_cast<unsigned>(lists * ((p.C + kStoredSlots - 1) / kStoredSlots))),
                          dim3(256), 0, st, p);
  const long long pieces = (p.C + SumsSmem<D>::kSlots - 1) / SumsSmem<D>::kSlots;
  e = launch_with<attend_sums_kernel<T, D>>(dim3(static_cast<unsigned>(pieces * units * p.row_parts)), kAttendThreads,
                                            sizeof(SumsSmem<D>) + 128, st, p);
  if (e != cudaSuccess) return e;
  return launch_chained(attend_heads_kernel, dim3(static_cast<unsigned>(lists * ((p.C + 255) / 256))), dim3(256), 0, st, p);
}

}  // namespace

cudaError_t launch_attend(const AttendParams& p, int d, int dtype, cudaStream_t st) {
  if (dtype == SC_FP16) return d == 64 ? launch_of<Fp16, 64>(p, st) : launch_of<Fp16, 128>(p, st);
  return d == 64 ? launch_of<Bf16, 64>(p, st) : launch_of<Bf16, 128>(p, st);
}

}  // namespace sc
