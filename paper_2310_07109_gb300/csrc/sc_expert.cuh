// sc_expert.cuh -- parameter blocks and launchers of the expert feed-forward
// operators (routing, products grouped by expert, gated sum with layer norm),
// shared by their kernels and the C entry points.
#pragma once

#include <cstddef>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/sparsecoder.h"

namespace sc {

constexpr int kMaxExperts = SC_MAX_EXPERTS;
constexpr int kMaxChoices = SC_MAX_CHOICES;
constexpr int kMaxExpertDim = SC_MAX_EXPERT_DIM;

// Tokens that a routing CTA chooses for at a time, and the most CTAs: each
// placing CTA adds up the counts of all CTAs before it, so their number is bounded.
constexpr int kRouteTokens = 128;
constexpr int kRouteMaxCtas = 256;

struct RouteParams {
  int B, L, E, k;
  long long T;               // B L
  const float* logits;       // [T][ld]
  long long ld;
  const int32_t* rows;       // [B] or nullptr
  int renormalize;
  int32_t* expert;           // [T][k]
  float* gate;               // [T][k]
  int32_t* offsets;          // [E + 1]
  int32_t* slot;             // [T][k]
  int32_t* token;            // [T k]
  int32_t* counts;           // workspace: [CTAs][E] slots that each CTA's tokens take
  int per_cta;               // tokens per CTA, a multiple of kRouteTokens
};

struct RouteBackParams {
  int B, L, E, k;
  long long T;
  const float* logits;
  long long ld;
  const int32_t* rows;
  int renormalize;
  const int32_t* expert;     // [T][k]
  const float* gate;         // [T][k]
  const float* dgate;        // [T][k]
  float* dlogits;            // [T][E]
};

constexpr int kExpertTimeout = 1;   // status word: a bounded wait expired

// One product grouped by expert.  Expert e has the slots offsets[e] .. offsets[e + 1].
enum class ExpertProduct { kForward, kBackInput, kBackWeight };
struct ExpertLinearParams {
  int M, E, N, K;
  const uint16_t* x;         // kForward, kBackWeight: rows [x_rows][ldx]
  long long ldx;
  int x_rows;
  const uint16_t* dy;        // kBackInput, kBackWeight: rows [M][ldy]
  long long ldy;
  const int32_t* token;      // [M] row of x per slot, or nullptr (the slot's own)
  const int32_t* offsets;    // [E + 1]
  const uint16_t* w;         // [E][N][K]
  const float* bias;         // [E][N] or nullptr
  int gelu;                  // kForward: out = GELU(y)
  const uint16_t* pre_in;    // kBackInput: [M][K] or nullptr; out = dx GELU'(pre)
  uint16_t* pre;             // kForward: [M][N] y itself, or nullptr
  void* out;                 // [M][N], [M][K] or [E][N][K]: bf16, or fp32 with out_f32
  int out_f32;
  float* dbias;              // kBackWeight: [E][N] or nullptr
  int* status;
  unsigned long long stall_ns;   // test hook (0: off): a wait of the products that nothing ends
};

// Slots of expert e: the caller's offsets, held within [0, M].
__device__ __forceinline__ void expert_range(const ExpertLinearParams& p, int e, int& lo, int& hi) {
  lo = min(max(__ldg(p.offsets + e), 0), p.M);
  hi = min(max(__ldg(p.offsets + e + 1), lo), p.M);
}

// The row of x that slot s reads, held within x.
__device__ __forceinline__ int expert_row(const ExpertLinearParams& p, int s) {
  return p.token == nullptr ? s : min(max(__ldg(p.token + s), 0), p.x_rows - 1);
}

constexpr int kCombineMaxParts = 256;   // CTAs of the gradient: partial sums per feature

struct CombineParams {
  int B, L, D, k, M;
  long long T;
  const int32_t* rows;       // [B] or nullptr
  const uint16_t* y;         // [M][D]
  const int32_t* slot;       // [T][k]
  const float* gate;         // [T][k] or nullptr (1)
  const uint16_t* res;       // [T][D] or nullptr
  float res_scale;
  const float* gamma;        // [D] or nullptr (no norm)
  const float* beta;
  float eps;
  uint16_t* sum;             // forward: [T][D] or nullptr
  uint16_t* out;             // forward: [T][D] or nullptr
  const uint16_t* dout;      // backward: [T][D] or nullptr
  const uint16_t* dsum;      // backward: [T][D] or nullptr
  uint16_t* dy;              // backward: [M][D]
  float* dgate;              // backward: [T][k] or nullptr
  uint16_t* dres;            // backward: [T][D] or nullptr
  float* dgamma;             // backward: [D] or nullptr
  float* dbeta;
  float* part;               // workspace: [CTAs][2][D]
};

int api_device_sms();   // multiprocessors of the current device (0 if unknown)
cudaError_t configure_expert();
cudaError_t configure_combine();
cudaError_t launch_route(const RouteParams& p, cudaStream_t st);
cudaError_t launch_route_back(const RouteBackParams& p, cudaStream_t st);
cudaError_t launch_expert_linear(ExpertProduct what, const ExpertLinearParams& p, cudaStream_t st);
cudaError_t launch_combine(const CombineParams& p, cudaStream_t st);
cudaError_t launch_combine_back(const CombineParams& p, cudaStream_t st);

template <typename... KArgs>
inline cudaError_t launch_chained(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                                  cudaStream_t st, const KArgs&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace sc
