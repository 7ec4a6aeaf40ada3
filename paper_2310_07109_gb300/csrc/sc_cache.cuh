// sc_cache.cuh -- parameter blocks and launchers of the pruned key-value cache (norm
// and rotation of heads, append, attention with accumulated weights, eviction), and
// the 16-bit types that its kernels take.
#pragma once

#include <atomic>
#include <cstddef>
#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/sparsecoder.h"
#include "sm103_primitives.cuh"

namespace sc {

constexpr int kCacheSms = 152;   // what splits and workspaces are sized for

// Every kernel of the cache is launched while the one before it still runs, and waits for it.  What that one may write
// (len, seen, pos, rows, queries) is therefore read by ordinary loads: the read-only path wants data that
// nobody writes while the kernel lives, from before its wait on.

// The two 16-bit types: eight values <-> fp32, and the warp product of their fragments.
struct Bf16 {
  static __device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi) {
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return pack_bf16x2(lo, hi); }
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    mma_bf16(c, a, b0, b1);
  }
  // The weights' reference lies this far (a power of two) below the largest score.
  static constexpr float kHeadroom = 0.f;
  // A pair of weights x, y >= 0 as sums of two values each.
  static __device__ __forceinline__ void split(float x, float y, uint32_t& first, uint32_t& second) {
    const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
    first = __byte_perm(a, b, 0x7632);   // (cut off, not rounded)
    second = pack(fmaf(x, 1.f + 0x1p-20f, -__uint_as_float(a & 0xffff0000u)), fmaf(y, 1.f + 0x1p-20f, -__uint_as_float(b & 0xffff0000u)));
  }
};

struct Fp16 {
  static __device__ __forceinline__ void unpack(uint32_t w, float& lo, float& hi) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
  }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
  // A weight of 2^-24 is fp16's smallest: up to 2^12 instead of 1, so that the many small
  // weights of a long list keep eleven bits down to 2^-26 of the largest.
  static constexpr float kHeadroom = 12.f;
  static __device__ __forceinline__ void split(float x, float y, uint32_t& first, uint32_t& second) {
    first = pack((1.f - 0x1p-10f) * x, (1.f - 0x1p-10f) * y);
    float a, b;
    unpack(first, a, b);
    second = pack(x - a, y - b);
  }
};

// The softmax's weights meet V as two 16-bit values each, one product after the other: one value's half step (2^-8 of
// a bf16 weight) is about what the one rounding of O may change, the sum's (2^-15; fp16: 2^-20) is not seen.  The second value is
// positive where the first is, so that infinities in V stay what they are (but for weights whose second value the type cannot
// hold: of fp16 those below 2^-26 of the largest, whose product with an infinity may be a NaN).

// One side of a rotation: heads of all tokens, `ld` elements a token.
struct HeadsIn {
  const uint16_t* p;
  long long ld;
};
struct HeadsOut {
  uint16_t* p;
  long long ld;
};

struct RotateParams {
  int B, L, Hq, Hk, d;
  long long T;               // B L
  float over_d;              // 1 / d
  unsigned long long per_row;   // 2^63 / L, rounded up: t / L is the high half of 2 t times it (t < 2^31)
  HeadsIn q, k;              // forward: the heads; backward: the forward call's heads
  HeadsIn dq, dk;            // backward: gradients of the outputs
  HeadsOut q_out, k_out;     // the outputs, or the gradients of the inputs
  const int32_t* rows;       // [B] or nullptr
  const int32_t* pos;        // [T] or nullptr (the row)
  const float* gamma_q;      // [d] or nullptr
  const float* gamma_k;
  float eps;
  int rot, interleaved;
  const double* freq;        // [rot / 2]
  float mscale;
  float* dgamma_q;           // [d] or nullptr
  float* dgamma_k;
  float* part;               // workspace: [CTAs][2][d]
  // append: where keys and values go instead of k_out
  HeadsIn v;
  uint16_t* cache_k;         // nullptr: not an append
  uint16_t* cache_v;
  long long stride_b, stride_h, stride_c;
  int C, G;
  float* acc;
  int32_t* slot_pos;
  const int32_t* len;
  const int32_t* seen;
  int32_t* len_out;
  int32_t* seen_out;
  int* status;
  unsigned* done;            // workspace: CTAs that have read len and seen
};

constexpr int kRotateMaxParts = 152 * 5;   // CTAs of the gradient

struct AttendParams {
  int B, C, H, Hk, G, T;
  int R, M;                  // query heads a key head; rows a key head (T R)
  const uint16_t* k;
  const uint16_t* v;
  long long stride_b, stride_h, stride_c;
  const float* acc;
  const int32_t* pos;
  const int32_t* len;
  const int32_t* seen;
  const uint16_t* q;
  long long ldq;
  const int32_t* rows;       // [B] or nullptr
  float scale2;              // scale log2(e)
  float decay;
  uint16_t* o;
  long long ldo;
  float* acc_out;
  // workspace, many rows
  int splits;                // parts of a list that CTAs take
  float* lse;                // [B][Hk][M], base 2; +inf: the row adds nothing
  // workspace, few rows
  int warps;                 // at work on the tiles of all lists
  int* share;                // tiles a warp, then [B][Hk] the first tile of each unit
  int stored;                // the scores are kept
  int row_parts;             // where they are not: parts that CTAs take a key head's rows in,
  float* sums;               // [B][Hk][row_parts][pitch] and the weights' sums over each
  float* scores;             // [B][Hk][M][pitch] scale log2(e) q . k; -inf: not seen
  int pitch;
  // both: parts (many rows: [B][Hk][splits]; few: a warp's number + a unit's)
  float2* ml;                // [part][M] reference, sum of weights
  float* part;               // [part][M][d]
};

constexpr int kFewRows = 16;                 // most rows a key head that the kernel for few rows takes
// Slots of a CTA that computes scores again: four tiles of 64, or two of wider heads.
constexpr int sum_tiles(int d) { return d == 64 ? 4 : 2; }
// Most rows that one launch joins and adds the weights of, from scores that are kept whatever they take (4 bytes a row and slot, in the
// workspace too: for 32 rows half of the bytes of K and V of 64 features).  32 rows, 65536 slots: 8 x 8 heads of 64 434 us, and
// 548 by the launches for more rows, which compute them again; 2 x 8 of 64 162 and 155; 2 x 8 of 128 203 and 301.  (16384
// slots, 2 x 8 heads of 64: 67 and 44, as few units make many parts, whose rows' LSE every CTA of sums finds for itself.)
constexpr int kJoinedRows = 32;
constexpr size_t kStoredBytes = 32u << 20;   // most bytes of the scores of more rows, else they are computed again
constexpr int kFewTile = 16;                 // slots a warp takes at a time
constexpr int kFewMinTiles = 2;              // fewest tiles of a warp
constexpr int few_warps_sm(int d) { return d == 64 ? 12 : 8; }

struct EvictParams {
  int B, C, Hk, G, d;
  uint16_t* k;
  uint16_t* v;
  long long stride_b, stride_h, stride_c;
  const float* acc;
  const int32_t* pos;
  const int32_t* len;
  const int32_t* seen;
  int budget, slack, sinks, recent;
  float* acc_out;
  int32_t* pos_out;
  int32_t* len_out;
  int32_t* moved;            // workspace: [B][G] rows that move
  int2* pairs;               // workspace: [B][G][pair_pitch] (to, from)
  long long pair_pitch;
  uint8_t* free_places;      // workspace: [B][G][free_pitch] a bit for each slot below budget
  long long free_pitch;
};

// A kernel's most dynamic shared memory, set before its first launch on a device (and not at set-up: who does not use
// the cache need not load its kernels).
template <auto kKernel>
cudaError_t allow_shared(size_t bytes) {
  static std::atomic<bool> ready[256];
  int dev = 0;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev >= 0 && dev < 256 && ready[dev].load(std::memory_order_acquire)) return cudaSuccess;
  const cudaError_t set = cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (set == cudaSuccess && dev >= 0 && dev < 256) ready[dev].store(true, std::memory_order_release);
  return set;
}

cudaError_t launch_rotate(const RotateParams& p, int dtype, cudaStream_t st);
cudaError_t launch_rotate_back(const RotateParams& p, int dtype, cudaStream_t st);
cudaError_t launch_attend(const AttendParams& p, int d, int dtype, cudaStream_t st);
cudaError_t launch_evict(const EvictParams& p, cudaStream_t st);

}  // namespace sc
