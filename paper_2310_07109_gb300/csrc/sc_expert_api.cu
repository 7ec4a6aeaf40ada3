// sc_expert_api.cu -- C entry points of the expert feed-forward operators: checks
// of the arguments, parameter blocks, launches.
#include <cstdio>

#include <cuda.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include "sc_expert.cuh"

namespace sc {
int api_fail_cuda(const char* what, cudaError_t e);
int api_ensure_configured();
unsigned long long api_stall_ns();
}  // namespace sc

namespace {

using namespace sc;

constexpr size_t kAlign = 256;
// (tiles and strides of threads may pass the last slot without passing 32 bits)
constexpr long long kMaxSlots = (1ll << 31) - 4096;

size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }
bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
// int32 and fp32 arrays (null ones too)
template <typename... T>
bool words(const T*... p) {
  return (aligned(p, 4) && ...);
}

struct ExpertLayout {
  size_t counts, part, total;
};

// The status word, then what the calls keep between their kernels.
ExpertLayout expert_layout(int E, int D) {
  ExpertLayout w;
  w.counts = kAlign;
  w.part = align_up(w.counts + sizeof(int32_t) * kRouteMaxCtas * static_cast<size_t>(E));
  w.total = align_up(w.part + sizeof(float) * kCombineMaxParts * 2 * static_cast<size_t>(D));
  return w;
}

bool good_tokens(int B, int L, int k) {
  return B >= 1 && L >= 1 && k >= 1 && k <= kMaxChoices &&
         static_cast<long long>(B) * L <= kMaxSlots / k;
}
bool good_width(int D) { return D >= 8 && D % 8 == 0 && D <= kMaxExpertDim; }

int check_workspace(const void* ws, size_t bytes, size_t need) {
  return !ws || bytes < need || !aligned(ws, kAlign) ? SC_ERR_WORKSPACE : SC_OK;
}

int check_product(int M, int E, int N, int K, const int32_t* offsets) {
  if (M < 1 || E < 1 || N < 8 || K < 8 || N % 8 || K % 8 || !offsets || !aligned(offsets, 4))
    return SC_ERR_INVALID_ARG;
  if (E > kMaxExperts || N > kMaxExpertDim || K > kMaxExpertDim || M > kMaxSlots) return SC_ERR_UNSUPPORTED;
  return SC_OK;
}

bool good_matrix(const void* p, long long ld, int width) {
  return p && aligned(p, 16) && ld >= width && ld % 8 == 0 && ld < (1ll << 30);
}

int launch_product(ExpertProduct what, ExpertLinearParams& p, void* stream) {
  const int rc = api_ensure_configured();
  if (rc != SC_OK) return rc;
  p.stall_ns = api_stall_ns();
  const cudaError_t e = launch_expert_linear(what, p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch expert product", e);
}

int check_combine(int B, int L, int D, int k, int M, const uint16_t* Y, const int32_t* slot,
                  const uint16_t* res, const float* gamma, float eps) {
  if (!good_tokens(B, L, k) || M < 1 || D < 8 || D % 8) return SC_ERR_INVALID_ARG;
  if (D > kMaxExpertDim) return SC_ERR_UNSUPPORTED;
  if (!Y || !aligned(Y, 16) || !slot || !aligned(res, 16) || (gamma && !(eps > 0.f)))
    return SC_ERR_INVALID_ARG;
  return SC_OK;
}

}  // namespace

extern "C" size_t sc_expert_workspace_size(int B, int L, int E, int k, int D) {
  if (!good_tokens(B, L, k) || E < 1 || E > kMaxExperts || k > E || !good_width(D)) return 0;
  return expert_layout(E, D).total;
}

extern "C" int sc_expert_route_forward(const sc_expert_route_args* a, void* workspace,
                                       size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  if (a->B < 1 || a->L < 1 || a->E < 1 || a->k < 1 || a->k > a->E) return SC_ERR_INVALID_ARG;
  if (a->E > kMaxExperts || a->k > kMaxChoices) return SC_ERR_UNSUPPORTED;
  if (!good_tokens(a->B, a->L, a->k)) return SC_ERR_INVALID_ARG;
  if (!a->logits || a->ld < a->E || !a->expert || !a->gate || !a->offsets || !a->slot || !a->token ||
      !words(a->logits, a->rows, a->expert, a->gate, a->offsets, a->slot, a->token))
    return SC_ERR_INVALID_ARG;
  const ExpertLayout lay = expert_layout(a->E, 8);
  int rc = check_workspace(workspace, ws_bytes, lay.part);
  if (rc != SC_OK || (rc = api_ensure_configured()) != SC_OK) return rc;
  RouteParams p{};
  p.B = a->B; p.L = a->L; p.E = a->E; p.k = a->k;
  p.T = static_cast<long long>(a->B) * a->L;
  p.logits = a->logits; p.ld = a->ld; p.rows = a->rows; p.renormalize = a->renormalize;
  p.expert = a->expert; p.gate = a->gate; p.offsets = a->offsets; p.slot = a->slot;
  p.token = a->token;
  p.counts = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + lay.counts);
  const cudaError_t e = launch_route(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch routing kernels", e);
}

extern "C" int sc_expert_route_backward(const sc_expert_route_backward_args* a, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  if (a->B < 1 || a->L < 1 || a->E < 1 || a->k < 1 || a->k > a->E) return SC_ERR_INVALID_ARG;
  if (a->E > kMaxExperts || a->k > kMaxChoices) return SC_ERR_UNSUPPORTED;
  if (!good_tokens(a->B, a->L, a->k)) return SC_ERR_INVALID_ARG;
  if (!a->logits || a->ld < a->E || !a->expert || !a->gate || !a->dgate || !a->dlogits ||
      !words(a->logits, a->rows, a->expert, a->gate, a->dgate, a->dlogits))
    return SC_ERR_INVALID_ARG;
  const int rc = api_ensure_configured();
  if (rc != SC_OK) return rc;
  RouteBackParams p{};
  p.B = a->B; p.L = a->L; p.E = a->E; p.k = a->k;
  p.T = static_cast<long long>(a->B) * a->L;
  p.logits = a->logits; p.ld = a->ld; p.rows = a->rows; p.renormalize = a->renormalize;
  p.expert = a->expert; p.gate = a->gate; p.dgate = a->dgate; p.dlogits = a->dlogits;
  const cudaError_t e = launch_route_back(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch routing gradient", e);
}

extern "C" int sc_expert_linear_forward(const sc_expert_linear_args* a, void* workspace,
                                        size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_product(a->M, a->E, a->N, a->K, a->offsets);
  if (rc != SC_OK) return rc;
  if (!good_matrix(a->X, a->ldx, a->K) || a->x_rows < 1 || (!a->token && a->x_rows < a->M) ||
      !a->W || !aligned(a->W, 16) || !a->out || !aligned(a->out, 16) || !aligned(a->pre, 16) ||
      !words(a->token, a->bias))
    return SC_ERR_INVALID_ARG;
  if ((rc = check_workspace(workspace, ws_bytes, kAlign)) != SC_OK) return rc;
  ExpertLinearParams p{};
  p.M = a->M; p.E = a->E; p.N = a->N; p.K = a->K;
  p.x = a->X; p.ldx = a->ldx; p.x_rows = a->x_rows; p.token = a->token; p.offsets = a->offsets;
  p.w = a->W; p.bias = a->bias; p.gelu = a->gelu; p.pre = a->pre;
  p.out = a->out; p.out_f32 = a->out_f32;
  p.status = static_cast<int*>(workspace);
  return launch_product(ExpertProduct::kForward, p, stream);
}

extern "C" int sc_expert_linear_backward_input(const sc_expert_linear_backward_input_args* a,
                                               void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_product(a->M, a->E, a->N, a->K, a->offsets);
  if (rc != SC_OK) return rc;
  if (!good_matrix(a->dY, a->ldy, a->N) || !a->W || !aligned(a->W, 16) || !a->dX ||
      !aligned(a->dX, 16) || !aligned(a->pre, 16))
    return SC_ERR_INVALID_ARG;
  if ((rc = check_workspace(workspace, ws_bytes, kAlign)) != SC_OK) return rc;
  ExpertLinearParams p{};
  p.M = a->M; p.E = a->E; p.N = a->N; p.K = a->K;
  p.dy = a->dY; p.ldy = a->ldy; p.offsets = a->offsets; p.w = a->W; p.pre_in = a->pre;
  p.out = a->dX; p.out_f32 = a->out_f32;
  p.status = static_cast<int*>(workspace);
  return launch_product(ExpertProduct::kBackInput, p, stream);
}

extern "C" int sc_expert_linear_backward_weight(const sc_expert_linear_backward_weight_args* a,
                                                void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_product(a->M, a->E, a->N, a->K, a->offsets);
  if (rc != SC_OK) return rc;
  if (!good_matrix(a->dY, a->ldy, a->N) || !good_matrix(a->X, a->ldx, a->K) || a->x_rows < 1 ||
      (!a->token && a->x_rows < a->M) || !a->dW || !aligned(a->dW, 16) || !words(a->token, a->dbias))
    return SC_ERR_INVALID_ARG;
  if ((rc = check_workspace(workspace, ws_bytes, kAlign)) != SC_OK) return rc;
  ExpertLinearParams p{};
  p.M = a->M; p.E = a->E; p.N = a->N; p.K = a->K;
  p.dy = a->dY; p.ldy = a->ldy; p.x = a->X; p.ldx = a->ldx; p.x_rows = a->x_rows;
  p.token = a->token; p.offsets = a->offsets;
  p.out = a->dW; p.out_f32 = a->out_f32; p.dbias = a->dbias;
  p.status = static_cast<int*>(workspace);
  return launch_product(ExpertProduct::kBackWeight, p, stream);
}

extern "C" int sc_expert_combine_forward(const sc_expert_combine_args* a, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_combine(a->B, a->L, a->D, a->k, a->M, a->Y, a->slot, a->res, a->gamma, a->eps);
  if (rc != SC_OK) return rc;
  if ((a->gamma == nullptr) != (a->beta == nullptr) || (a->gamma != nullptr && !a->out) ||
      (!a->sum && !a->gamma) || !aligned(a->sum, 16) || !aligned(a->out, 16) ||
      !words(a->rows, a->slot, a->gate, a->gamma, a->beta))
    return SC_ERR_INVALID_ARG;
  if ((rc = api_ensure_configured()) != SC_OK) return rc;
  CombineParams p{};
  p.B = a->B; p.L = a->L; p.D = a->D; p.k = a->k; p.M = a->M;
  p.T = static_cast<long long>(a->B) * a->L;
  p.rows = a->rows; p.y = a->Y; p.slot = a->slot; p.gate = a->gate; p.res = a->res;
  p.res_scale = a->res_scale; p.gamma = a->gamma; p.beta = a->beta; p.eps = a->eps;
  p.sum = a->sum; p.out = a->out;
  const cudaError_t e = launch_combine(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch combine kernel", e);
}

extern "C" int sc_expert_combine_backward(const sc_expert_combine_backward_args* a, void* workspace,
                                          size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_combine(a->B, a->L, a->D, a->k, a->M, a->Y, a->slot, a->res, a->gamma, a->eps);
  if (rc != SC_OK) return rc;
  const bool norm = a->gamma != nullptr;
  if (norm != (a->dout != nullptr) || norm != (a->dgamma != nullptr) ||
      norm != (a->dbeta != nullptr) || (!a->dout && !a->dsum) || !a->dY || !aligned(a->dY, 16) ||
      !aligned(a->dout, 16) || !aligned(a->dsum, 16) || !aligned(a->dres, 16) ||
      !words(a->rows, a->slot, a->gate, a->gamma, a->dgate, a->dgamma, a->dbeta))
    return SC_ERR_INVALID_ARG;
  const ExpertLayout lay = expert_layout(1, a->D);
  if ((rc = check_workspace(workspace, ws_bytes, norm ? lay.total - lay.part + kAlign : kAlign)) != SC_OK)
    return rc;
  if ((rc = api_ensure_configured()) != SC_OK) return rc;
  CombineParams p{};
  p.B = a->B; p.L = a->L; p.D = a->D; p.k = a->k; p.M = a->M;
  p.T = static_cast<long long>(a->B) * a->L;
  p.rows = a->rows; p.y = a->Y; p.slot = a->slot; p.gate = a->gate; p.res = a->res;
  p.res_scale = a->res_scale; p.gamma = a->gamma; p.eps = a->eps;
  p.dout = a->dout; p.dsum = a->dsum; p.dy = a->dY; p.dgate = a->dgate; p.dres = a->dres;
  p.dgamma = a->dgamma; p.dbeta = a->dbeta;
  // the parts share the space after the status word with the routing's counts: each
  // call is done with it when the next one of its stream starts
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kAlign);
  const cudaError_t e = launch_combine_back(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch combine gradient", e);
}
