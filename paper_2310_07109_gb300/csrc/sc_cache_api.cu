// sc_cache_api.cu -- C entry points of the rotation of heads and of the pruned key-value
// cache: checks of the arguments, parameter blocks, launches.
#include <algorithm>
#include <cmath>
#include <cuda_runtime.h>

#include "sc_cache.cuh"

namespace sc {
int api_fail_cuda(const char* what, cudaError_t e);
int api_ensure_configured();
}  // namespace sc

namespace {

using namespace sc;

constexpr size_t kAlign = 256;
constexpr long long kMaxTokens = (1ll << 31) - 4096;
constexpr int kRowsTile = 64;   // of the attention kernels

size_t align_up(size_t x) { return (x + kAlign - 1) & ~(kAlign - 1); }
bool aligned(const void* p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }
template <typename... T>
bool words(const T*... p) {
  return (aligned(p, 4) && ...);
}

int check_workspace(const void* ws, size_t bytes, size_t need) {
  return !ws || bytes < need || !aligned(ws, kAlign) ? SC_ERR_WORKSPACE : SC_OK;
}

bool good_dtype(int dtype) { return dtype == SC_BF16 || dtype == SC_FP16; }
// heads of all tokens, one token `ld` elements after the other
bool good_heads(const void* p, long long ld, int heads, int d) {
  return p && aligned(p, 16) && ld >= static_cast<long long>(heads) * d && ld % 8 == 0 && ld < (1ll << 30);
}

// Whether outputs lie apart from the inputs or, in their place, with their distances (one token has none).
bool good_place(const void* in, long long ld_in, const void* out, long long ld_out, int B, int L) {
  return in != out || ld_in == ld_out || static_cast<long long>(B) * L == 1;
}

int check_rotate(int B, int L, int Hq, int Hk, int d, int dtype, const int32_t* rows, const float* gamma_q,
                 const float* gamma_k, float eps, int rot, const double* freq, float mscale) {
  if (B < 1 || L < 1 || Hq < 0 || Hk < 0 || Hq + static_cast<long long>(Hk) < 1 || d < 16 || d % 16 || !good_dtype(dtype) ||
      rot < 0 || rot > d || rot % 16)
    return SC_ERR_INVALID_ARG;
  if (d > SC_MAX_HEAD_WIDTH || Hq + static_cast<long long>(Hk) > SC_MAX_HEADS ||
      static_cast<long long>(B) * L > kMaxTokens)
    return SC_ERR_UNSUPPORTED;
  if ((rot > 0 && (!freq || !aligned(freq, 8) || !std::isfinite(mscale))) || ((gamma_q || gamma_k) && !(eps > 0.f)) ||
      !words(rows, gamma_q, gamma_k))
    return SC_ERR_INVALID_ARG;
  return SC_OK;
}

struct CacheLayout {
  size_t lse, share, scores, sums, ml, part, moved, pairs, free_places, evict, total;
  int splits, warps, pitch, row_parts;
  bool stored;
  long long pair_pitch, free_pitch;
};

// Parts that the attention takes a list in: as many CTAs as SMs have room for (three, two of wide heads), parts of 256
// slots at least.
int splits_of(int B, int C, int Hk, int M, int d) {
  const long long ctas = static_cast<long long>(B) * Hk * ((M + kRowsTile - 1) / kRowsTile);
  const long long want = std::max<long long>(1, (d == 64 ? 3 : 2) * kCacheSms / ctas);
  return static_cast<int>(std::min<long long>(want, (C + 255) / 256));
}

// The status word and a counter, then what the calls keep between their kernels (each is done with it when
// the next one of its stream starts, so they share the space).
CacheLayout cache_layout(int B, int C, int H, int Hk, int G, int d, int T) {
  CacheLayout w;
  const size_t units = static_cast<size_t>(B) * Hk, lists = static_cast<size_t>(B) * G;
  const size_t M = static_cast<size_t>(T) * (H / Hk);
  const bool few = M <= kFewRows;
  // no more warps than the most tiles give work to
  w.splits = few ? 1 : splits_of(B, C, Hk, static_cast<int>(M), d);
  const size_t tiles = units * ((C + kFewTile - 1) / kFewTile);
  const size_t cta = kFewMinTiles * few_warps_sm(d);   // fewest tiles of a CTA
  w.warps = static_cast<int>(std::min<size_t>(kCacheSms, (tiles + cta - 1) / cta)) * few_warps_sm(d);
  w.pitch = (C + 3) & ~3;
  const size_t parts = few ? w.warps + units : units * w.splits;
  const size_t scores = sizeof(float) * units * M * w.pitch;
  w.stored = M <= kJoinedRows || scores <= kStoredBytes;
  // parts of the rows, until the SMs have three CTAs each
  const size_t ctas = units * ((C + 64 * sum_tiles(d) - 1) / (64 * sum_tiles(d)));
  w.row_parts = static_cast<int>(std::max<size_t>(1, std::min<size_t>(3 * kCacheSms / ctas, (M + kRowsTile - 1) / kRowsTile)));
  w.share = w.lse = kAlign;
  w.scores = align_up(kAlign + std::max(sizeof(int) * (1 + units), sizeof(float) * units * M));
  w.sums = w.scores;
  w.ml = align_up(w.scores + (w.stored ? scores : sizeof(float) * units * w.row_parts * w.pitch));
  w.part = align_up(w.ml + sizeof(float2) * parts * M);
  const size_t attend = align_up(w.part + sizeof(float) * parts * M * d);
  w.pair_pitch = C / 2 + 1;
  w.moved = kAlign;
  w.pairs = align_up(w.moved + sizeof(int32_t) * lists);
  w.free_places = align_up(w.pairs + sizeof(int2) * lists * w.pair_pitch);
  w.free_pitch = (C + 7) / 8;
  w.evict = align_up(w.free_places + lists * w.free_pitch);
  w.total = std::max(attend, w.evict);
  return w;
}

// The most that a call of 1 to T tokens a sequence needs.  Its bytes grow with the tokens but where few rows become more, scores are no
// longer kept, or one more tile of rows leaves a list fewer parts: the last sizes before these, and T itself.
size_t most_bytes(int B, int C, int H, int Hk, int G, int d, int T) {
  const long long R = H / Hk, M = T * R, units = static_cast<long long>(B) * Hk, pitch = (C + 3) & ~3;
  size_t most = 0;
  const auto up_to = [&](long long rows) {   // the most tokens of no more than these rows
    if (rows >= R) most = std::max(most, cache_layout(B, C, H, Hk, G, d, static_cast<int>(std::min(rows, M) / R)).total);
  };
  up_to(kFewRows);
  up_to(kJoinedRows);
  up_to(static_cast<long long>(kStoredBytes) / (static_cast<long long>(sizeof(float)) * units * pitch));
  for (long long rows = kRowsTile; rows < M && splits_of(B, C, Hk, static_cast<int>(rows), d) > 1; rows += kRowsTile) up_to(rows);
  up_to(M);
  return most;
}

// SC_OK for sizes of a cache that the calls take (H: 0 where there are no queries).
int check_cache_sizes(int B, int C, int H, int Hk, int G, int d) {
  if (B < 1 || C < 1 || H < 0 || Hk < 1 || G < 1 || Hk % G || H % Hk || d < 16 || d % 16) return SC_ERR_INVALID_ARG;
  if (C > SC_MAX_CACHE || d > SC_MAX_HEAD_WIDTH || static_cast<long long>(H) + Hk > SC_MAX_HEADS ||
      static_cast<long long>(B) * Hk * ((C + kFewTile - 1) / kFewTile) > kMaxTokens)
    return SC_ERR_UNSUPPORTED;
  return SC_OK;
}

int check_cache(int B, int C, int H, int Hk, int G, int d, int dtype, const void* K, const void* V, long long sb,
                long long sh, long long sc_, const float* acc, const int32_t* pos, const int32_t* len, const int32_t* seen) {
  const int rc = check_cache_sizes(B, C, H, Hk, G, d);
  if (rc != SC_OK) return rc;
  if (!good_dtype(dtype) || !K || !V || !aligned(K, 16) || !aligned(V, 16) || sb % 8 || sh % 8 || sc_ % 8 || sc_ < d ||
      (B > 1 && sb < d) || (Hk > 1 && sh < d) || !acc || !pos || !len || !seen || !words(acc, pos, len, seen))
    return SC_ERR_INVALID_ARG;
  return SC_OK;
}

int check_attend_sizes(int B, int H, int Hk, int d, int T) {
  if (H < 1 || T < 1) return SC_ERR_INVALID_ARG;
  if (T > SC_MAX_STEP || (d != 64 && d != 128) || static_cast<long long>(B) * H > kMaxTokens / T)
    return SC_ERR_UNSUPPORTED;
  return SC_OK;
}

}  // namespace

extern "C" size_t sc_rotate_workspace_size(int d) {
  if (d < 16 || d % 16 || d > SC_MAX_HEAD_WIDTH) return 0;
  return align_up(kAlign + sizeof(float) * 2 * static_cast<size_t>(d) * kRotateMaxParts);
}

extern "C" int sc_rotate_forward(const sc_rotate_args* a, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_rotate(a->B, a->L, a->Hq, a->Hk, a->d, a->dtype, a->rows, a->gamma_q, a->gamma_k, a->eps, a->rot,
                        a->freq, a->mscale);
  if (rc != SC_OK) return rc;
  if (!words(a->pos) || (a->Hq > 0 && (!good_heads(a->Q, a->ldq, a->Hq, a->d) || !good_heads(a->Q_out, a->ldq_out, a->Hq, a->d))) ||
      (a->Hk > 0 && (!good_heads(a->K, a->ldk, a->Hk, a->d) || !good_heads(a->K_out, a->ldk_out, a->Hk, a->d))) ||
      (a->Hq > 0 && !good_place(a->Q, a->ldq, a->Q_out, a->ldq_out, a->B, a->L)) ||
      (a->Hk > 0 && !good_place(a->K, a->ldk, a->K_out, a->ldk_out, a->B, a->L)))
    return SC_ERR_INVALID_ARG;
  if ((rc = api_ensure_configured()) != SC_OK) return rc;
  RotateParams p{};
  p.B = a->B; p.L = a->L; p.Hq = a->Hq; p.Hk = a->Hk; p.d = a->d;
  p.T = static_cast<long long>(a->B) * a->L;
  p.over_d = 1.f / static_cast<float>(a->d);
  p.per_row = (1ull << 63) / static_cast<unsigned>(a->L) + 1;
  p.q = {static_cast<const uint16_t*>(a->Q), a->ldq};
  p.k = {static_cast<const uint16_t*>(a->K), a->ldk};
  p.q_out = {static_cast<uint16_t*>(a->Q_out), a->ldq_out};
  p.k_out = {static_cast<uint16_t*>(a->K_out), a->ldk_out};
  p.rows = a->rows; p.pos = a->pos; p.gamma_q = a->gamma_q; p.gamma_k = a->gamma_k; p.eps = a->eps;
  p.rot = a->rot; p.interleaved = a->interleaved; p.freq = a->freq; p.mscale = a->mscale;
  const cudaError_t e = launch_rotate(p, a->dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch rotation", e);
}

extern "C" int sc_rotate_backward(const sc_rotate_backward_args* a, void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_rotate(a->B, a->L, a->Hq, a->Hk, a->d, a->dtype, a->rows, a->gamma_q, a->gamma_k, a->eps, a->rot,
                        a->freq, a->mscale);
  if (rc != SC_OK) return rc;
  if (!words(a->pos, a->dgamma_q, a->dgamma_k) || (a->gamma_q == nullptr) != (a->dgamma_q == nullptr) ||
      (a->gamma_k == nullptr) != (a->dgamma_k == nullptr) ||
      (a->Hq > 0 && (!good_heads(a->dQ_out, a->ldq_out, a->Hq, a->d) || !good_heads(a->dQ, a->ldq_grad, a->Hq, a->d) ||
                     (a->gamma_q && !good_heads(a->Q, a->ldq, a->Hq, a->d)))) ||
      (a->Hk > 0 && (!good_heads(a->dK_out, a->ldk_out, a->Hk, a->d) || !good_heads(a->dK, a->ldk_grad, a->Hk, a->d) ||
                     (a->gamma_k && !good_heads(a->K, a->ldk, a->Hk, a->d)))) ||
      (a->Hq > 0 && !good_place(a->dQ_out, a->ldq_out, a->dQ, a->ldq_grad, a->B, a->L)) ||
      (a->Hk > 0 && !good_place(a->dK_out, a->ldk_out, a->dK, a->ldk_grad, a->B, a->L)))
    return SC_ERR_INVALID_ARG;
  if ((rc = check_workspace(workspace, ws_bytes, sc_rotate_workspace_size(a->d))) != SC_OK) return rc;
  if ((rc = api_ensure_configured()) != SC_OK) return rc;
  RotateParams p{};
  p.B = a->B; p.L = a->L; p.Hq = a->Hq; p.Hk = a->Hk; p.d = a->d;
  p.T = static_cast<long long>(a->B) * a->L;
  p.over_d = 1.f / static_cast<float>(a->d);
  p.per_row = (1ull << 63) / static_cast<unsigned>(a->L) + 1;
  p.dq = {static_cast<const uint16_t*>(a->dQ_out), a->ldq_out};
  p.dk = {static_cast<const uint16_t*>(a->dK_out), a->ldk_out};
  // without a norm Q and K are not read, and nothing was checked of them: no address is made from them
  p.q = a->gamma_q ? HeadsIn{static_cast<const uint16_t*>(a->Q), a->ldq} : p.dq;
  p.k = a->gamma_k ? HeadsIn{static_cast<const uint16_t*>(a->K), a->ldk} : p.dk;
  p.q_out = {static_cast<uint16_t*>(a->dQ), a->ldq_grad};
  p.k_out = {static_cast<uint16_t*>(a->dK), a->ldk_grad};
  p.rows = a->rows; p.pos = a->pos; p.gamma_q = a->gamma_q; p.gamma_k = a->gamma_k; p.eps = a->eps;
  p.rot = a->rot; p.interleaved = a->interleaved; p.freq = a->freq; p.mscale = a->mscale;
  p.dgamma_q = a->dgamma_q; p.dgamma_k = a->dgamma_k;
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + kAlign);
  const cudaError_t e = launch_rotate_back(p, a->dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch rotation gradient", e);
}

extern "C" size_t sc_cache_workspace_size(int B, int C, int H, int Hk, int G, int d, int T) {
  if (check_cache_sizes(B, C, H, Hk, G, d) != SC_OK) return 0;
  if (T < 1 || (d == 64 || d == 128 ? check_attend_sizes(B, std::max(H, Hk), Hk, d, T) != SC_OK : T > 1)) return 0;
  return most_bytes(B, C, std::max(H, Hk), Hk, G, d, T);
}

extern "C" int sc_cache_append(const sc_cache_append_args* a, void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_cache(a->B, a->C, a->H, a->Hk, a->G, a->d, a->dtype, a->K, a->V, a->stride_b, a->stride_h, a->stride_c,
                       a->acc, a->pos, a->len, a->seen);
  if (rc == SC_OK)
    rc = check_rotate(a->B, a->L, a->H, a->Hk, a->d, a->dtype, a->rows, a->gamma_q, a->gamma_k, a->eps, a->rot, a->freq, a->mscale);
  if (rc != SC_OK) return rc;
  if ((a->H > 0 && (!good_heads(a->Q, a->ldq, a->H, a->d) || !good_heads(a->Q_out, a->ldq_out, a->H, a->d) ||
                    !good_place(a->Q, a->ldq, a->Q_out, a->ldq_out, a->B, a->L))) ||
      !good_heads(a->K_in, a->ldk, a->Hk, a->d) || !good_heads(a->V_in, a->ldv, a->Hk, a->d) || !a->len_out ||
      !a->seen_out || !words(a->len_out, a->seen_out))
    return SC_ERR_INVALID_ARG;
  if ((rc = check_workspace(workspace, ws_bytes, kAlign)) != SC_OK || (rc = api_ensure_configured()) != SC_OK) return rc;
  RotateParams p{};
  p.B = a->B; p.L = a->L; p.Hq = a->H; p.Hk = a->Hk; p.d = a->d;
  p.T = static_cast<long long>(a->B) * a->L;
  p.over_d = 1.f / static_cast<float>(a->d);
  p.per_row = (1ull << 63) / static_cast<unsigned>(a->L) + 1;
  p.q = {static_cast<const uint16_t*>(a->Q), a->ldq};
  p.k = {static_cast<const uint16_t*>(a->K_in), a->ldk};
  p.v = {static_cast<const uint16_t*>(a->V_in), a->ldv};
  p.q_out = {static_cast<uint16_t*>(a->Q_out), a->ldq_out};
  p.rows = a->rows; p.gamma_q = a->gamma_q; p.gamma_k = a->gamma_k; p.eps = a->eps;
  p.rot = a->rot; p.interleaved = a->interleaved; p.freq = a->freq; p.mscale = a->mscale;
  p.cache_k = static_cast<uint16_t*>(a->K); p.cache_v = static_cast<uint16_t*>(a->V);
  p.stride_b = a->stride_b; p.stride_h = a->stride_h; p.stride_c = a->stride_c;
  p.C = a->C; p.G = a->G; p.acc = a->acc; p.slot_pos = a->pos; p.len = a->len; p.seen = a->seen;
  p.len_out = a->len_out; p.seen_out = a->seen_out;
  p.status = static_cast<int*>(workspace);
  p.done = static_cast<unsigned*>(workspace) + 16;
  const cudaError_t e = launch_rotate(p, a->dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch cache append", e);
}

extern "C" int sc_cache_attend(const sc_cache_attend_args* a, void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_cache(a->B, a->C, a->H, a->Hk, a->G, a->d, a->dtype, a->K, a->V, a->stride_b, a->stride_h, a->stride_c,
                       a->acc, a->pos, a->len, a->seen);
  if (rc == SC_OK) rc = check_attend_sizes(a->B, a->H, a->Hk, a->d, a->T);
  if (rc != SC_OK) return rc;
  if (!good_heads(a->Q, a->ldq, a->H, a->d) || !good_heads(a->O, a->ldo, a->H, a->d) || !a->acc_out ||
      a->O == a->Q || !words(a->acc_out, a->rows) || !std::isfinite(a->scale) || !std::isfinite(a->decay))
    return SC_ERR_INVALID_ARG;
  const CacheLayout w = cache_layout(a->B, a->C, a->H, a->Hk, a->G, a->d, a->T);
  if ((rc = check_workspace(workspace, ws_bytes, w.total)) != SC_OK || (rc = api_ensure_configured()) != SC_OK) return rc;
  AttendParams p{};
  p.B = a->B; p.C = a->C; p.H = a->H; p.Hk = a->Hk; p.G = a->G; p.T = a->T;
  p.R = a->H / a->Hk; p.M = a->T * p.R;
  p.k = static_cast<const uint16_t*>(a->K); p.v = static_cast<const uint16_t*>(a->V);
  p.stride_b = a->stride_b; p.stride_h = a->stride_h; p.stride_c = a->stride_c;
  p.acc = a->acc; p.pos = a->pos; p.len = a->len; p.seen = a->seen;
  p.q = static_cast<const uint16_t*>(a->Q); p.ldq = a->ldq; p.rows = a->rows;
  p.scale2 = static_cast<float>(static_cast<double>(a->scale) * 1.4426950408889634);   // log2(e)
  p.decay = a->decay;
  p.o = static_cast<uint16_t*>(a->O); p.ldo = a->ldo; p.acc_out = a->acc_out;
  p.splits = w.splits; p.warps = w.warps; p.pitch = w.pitch; p.stored = w.stored;
  p.row_parts = w.row_parts;
  char* ws = static_cast<char*>(workspace);
  p.lse = reinterpret_cast<float*>(ws + w.lse);
  p.share = reinterpret_cast<int*>(ws + w.share);
  p.scores = reinterpret_cast<float*>(ws + w.scores);
  p.sums = reinterpret_cast<float*>(ws + w.sums);
  p.ml = reinterpret_cast<float2*>(ws + w.ml);
  p.part = reinterpret_cast<float*>(ws + w.part);
  const cudaError_t e = launch_attend(p, a->d, a->dtype, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch cache attention", e);
}

extern "C" int sc_cache_evict(const sc_cache_evict_args* a, void* workspace, size_t ws_bytes, void* stream) {
  if (!a) return SC_ERR_INVALID_ARG;
  int rc = check_cache(a->B, a->C, 0, a->Hk, a->G, a->d, a->dtype, a->K, a->V, a->stride_b, a->stride_h, a->stride_c,
                       a->acc, a->pos, a->len, a->seen);
  if (rc != SC_OK) return rc;
  if (a->budget < 1 || a->slack < 0 || a->sinks < 0 || a->recent < 0 ||
      static_cast<long long>(a->sinks) + a->recent > a->budget || !a->acc_out || !a->pos_out || !a->len_out ||
      !words(a->acc_out, a->pos_out, a->len_out))
    return SC_ERR_INVALID_ARG;
  const CacheLayout w = cache_layout(a->B, a->C, a->Hk, a->Hk, a->G, a->d, 1);
  if ((rc = check_workspace(workspace, ws_bytes, w.evict)) != SC_OK || (rc = api_ensure_configured()) != SC_OK) return rc;
  EvictParams p{};
  p.B = a->B; p.C = a->C; p.Hk = a->Hk; p.G = a->G; p.d = a->d;
  p.k = static_cast<uint16_t*>(a->K); p.v = static_cast<uint16_t*>(a->V);
  p.stride_b = a->stride_b; p.stride_h = a->stride_h; p.stride_c = a->stride_c;
  p.acc = a->acc; p.pos = a->pos; p.len = a->len; p.seen = a->seen;
  p.budget = a->budget; p.slack = a->slack; p.sinks = a->sinks; p.recent = a->recent;
  p.acc_out = a->acc_out; p.pos_out = a->pos_out; p.len_out = a->len_out;
  char* ws = static_cast<char*>(workspace);
  p.moved = reinterpret_cast<int32_t*>(ws + w.moved);
  p.pairs = reinterpret_cast<int2*>(ws + w.pairs);
  p.pair_pitch = w.pair_pitch;
  p.free_places = reinterpret_cast<uint8_t*>(ws + w.free_places);
  p.free_pitch = w.free_pitch;
  const cudaError_t e = launch_evict(p, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? SC_OK : api_fail_cuda("launch cache eviction", e);
}
