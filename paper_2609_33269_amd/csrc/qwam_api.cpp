// C ABI of libqwam: argument validation and dispatch to the HIP kernels.
// Every check runs on the host before any HIP call; device memory is never
// dereferenced here.
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstdarg>
#include <cstdint>
#include <cstdio>

#include "../../include/qwam.h"
#include "../../include/qwam_probe.h"
#include "qwam_internal.h"

namespace {

thread_local char g_err[512] = "";

qwam_status fail(qwam_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_err, sizeof(g_err), fmt, ap);
  va_end(ap);
  return s;
}

qwam_status ok() {
  g_err[0] = '\0';
  return QWAM_OK;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

#define QWAM_REQUIRE_PTR(p)                                                              \
  do {                                                                                   \
    if ((p) == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: %s is NULL", fn, #p);     \
    if (!aligned16(p)) return fail(QWAM_ERR_MISALIGNED, "%s: %s is not 16-byte aligned", fn, #p); \
  } while (0)

constexpr int32_t kMaxK = 65536;
constexpr int32_t kMaxN = 1 << 20;
constexpr int32_t kMaxM = 1 << 20;

// N is checked unless need_n is false (a call that does not read it)
qwam_status check_kn(const char* fn, int32_t K, int32_t N, int32_t group, bool need_n = true) {
  if (group != QWAM_GROUP && group != 32)
    return fail(QWAM_ERR_INVALID_ARG, "%s: group must be 64 or 32 (got %d)", fn, group);
  if (K <= 0 || K % QWAM_GROUP != 0) return fail(QWAM_ERR_INVALID_ARG, "%s: K must be a positive multiple of 64 (got %d)", fn, K);
  if (need_n && (N <= 0 || N % 16 != 0))
    return fail(QWAM_ERR_INVALID_ARG, "%s: N must be a positive multiple of 16 (got %d)", fn, N);
  if (K > kMaxK) return fail(QWAM_ERR_UNSUPPORTED, "%s: K = %d exceeds %d", fn, K, kMaxK);
  if (need_n && N > kMaxN) return fail(QWAM_ERR_UNSUPPORTED, "%s: N = %d exceeds %d", fn, N, kMaxN);
  return QWAM_OK;
}

qwam_status check_layer(const char* fn, const qwam_layer* L, bool need_branch, bool need_n = true) {
  if (L == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: layer is NULL", fn);
  qwam_status s = check_kn(fn, L->K, L->N, L->group, need_n);
  if (s != QWAM_OK) return s;
  if (need_branch && !(L->r == 16 || L->r == 32 || L->r == 48 || L->r == 64))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: rank r must be 16, 32, 48 or 64 (got %d)", fn, L->r);
  const int32_t B = L->hadamard;
  if (B != 0 && (B < 16 || B > 1024 || (B & (B - 1)) != 0 || L->K % B != 0))
    return fail(QWAM_ERR_INVALID_ARG, "%s: hadamard must be 0 or a power of two in [16, 1024] dividing K (got %d)",
                fn, B);
  return QWAM_OK;
}

qwam_status check_m(const char* fn, int32_t M) {
  if (M <= 0) return fail(QWAM_ERR_INVALID_ARG, "%s: M must be >= 1 (got %d)", fn, M);
  if (M > kMaxM) return fail(QWAM_ERR_UNSUPPORTED, "%s: M = %d exceeds %d", fn, M, kMaxM);
  return QWAM_OK;
}

// The device count is queried once per process (a query per call would add
// host time to every launch, which small layers notice).
qwam_status check_device(const char* fn) {
  static std::atomic<int> visible{-1};
  int n = visible.load(std::memory_order_relaxed);
  if (n < 0) {
    int c = 0;
    if (hipGetDeviceCount(&c) != hipSuccess) {
      (void)hipGetLastError();
      c = 0;
    }
    visible.store(c, std::memory_order_relaxed);
    n = c;
  }
  if (n <= 0) return fail(QWAM_ERR_NO_DEVICE, "%s: no HIP device visible", fn);
  return QWAM_OK;
}

qwam_status launched(const char* fn, hipError_t e) {
  if (e != hipSuccess) return fail(QWAM_ERR_HIP, "%s: kernel launch failed: %s", fn, hipGetErrorString(e));
  return ok();
}

}  // namespace

extern "C" {

qwam_status qwam_pack_weights(int32_t K, int32_t N, int32_t group, const float* R, const float* smooth,
                              uint8_t* wq, float* ws, uint32_t* wsp, float* inv_smooth, void* stream) {
  const char* fn = "qwam_pack_weights";
  qwam_status s = check_kn(fn, K, N, group);
  if (s != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(R);
  QWAM_REQUIRE_PTR(smooth);
  QWAM_REQUIRE_PTR(wq);
  QWAM_REQUIRE_PTR(ws);
  QWAM_REQUIRE_PTR(wsp);
  QWAM_REQUIRE_PTR(inv_smooth);
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_pack_weights(K, N, group, R, smooth, wq, ws, wsp, inv_smooth,
                                                static_cast<hipStream_t>(stream)));
}

}  // extern "C"

namespace {

qwam_status quantize_act_common(const char* fn, bool deflate, const qwam_layer* L, int32_t M,
                                const uint16_t* x, uint8_t* xq, float* xs, uint16_t* t, void* workspace,
                                int64_t workspace_bytes, void* stream) {
  qwam_status s = check_layer(fn, L, true);
  if (s != QWAM_OK) return s;
  if ((s = check_m(fn, M)) != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(L->inv_smooth);
  QWAM_REQUIRE_PTR(L->L1t);
  QWAM_REQUIRE_PTR(L->L1f);
  if (deflate) QWAM_REQUIRE_PTR(L->L1);
  QWAM_REQUIRE_PTR(x);
  QWAM_REQUIRE_PTR(xq);
  QWAM_REQUIRE_PTR(xs);
  QWAM_REQUIRE_PTR(t);
  if (workspace != nullptr) {
    if (!aligned16(workspace)) return fail(QWAM_ERR_MISALIGNED, "%s: workspace is not 16-byte aligned", fn);
    const int64_t need = qwam::act_workspace_bytes(M, L->K, L->r, L->hadamard, deflate);
    if (workspace_bytes < need)
      return fail(QWAM_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed", fn,
                  static_cast<long long>(workspace_bytes), static_cast<long long>(need));
  }
  if ((s = check_device(fn)) != QWAM_OK) return s;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  if (L->hadamard != 0)
    return launched(fn, qwam::launch_quantize_act_rotated(M, L->K, L->r, L->group, L->hadamard, deflate, x,
                                                          L->inv_smooth, L->L1t, L->L1f, deflate ? L->L1 : nullptr,
                                                          xq, xs, t, workspace, st));
  if (deflate)
    return launched(fn, qwam::launch_quantize_act_deflated(M, L->K, L->r, L->group, x, L->inv_smooth, L->L1f, L->L1,
                                                           xq, xs, t, workspace, st));
  return launched(fn, qwam::launch_quantize_act(M, L->K, L->r, L->group, x, L->inv_smooth, L->L1f, xq, xs, t, workspace,
                                                st));
}

}  // namespace

extern "C" {

qwam_status qwam_quantize_act(const qwam_layer* L, int32_t M, const uint16_t* x, uint8_t* xq, float* xs,
                              uint16_t* t, void* stream) {
  return quantize_act_common("qwam_quantize_act", false, L, M, x, xq, xs, t, nullptr, 0, stream);
}

qwam_status qwam_quantize_act_deflated(const qwam_layer* L, int32_t M, const uint16_t* x, uint8_t* xq,
                                       float* xs, uint16_t* t, void* stream) {
  return quantize_act_common("qwam_quantize_act_deflated", true, L, M, x, xq, xs, t, nullptr, 0, stream);
}

int64_t qwam_quantize_act_workspace(const qwam_layer* L, int32_t M, int32_t deflated) {
  const char* fn = "qwam_quantize_act_workspace";
  if (check_layer(fn, L, true, false) != QWAM_OK || check_m(fn, M) != QWAM_OK) return -1;
  return qwam::act_workspace_bytes(M, L->K, L->r, L->hadamard, deflated != 0);
}

qwam_status qwam_quantize_act_ws(const qwam_layer* L, int32_t M, int32_t deflated, const uint16_t* x, uint8_t* xq,
                                 float* xs, uint16_t* t, void* workspace, int64_t workspace_bytes, void* stream) {
  return quantize_act_common(deflated != 0 ? "qwam_quantize_act_deflated" : "qwam_quantize_act", deflated != 0, L, M, x,
                             xq, xs, t, workspace, workspace_bytes, stream);
}

qwam_status qwam_asp_linear(const qwam_layer* L, int32_t M, const uint8_t* xq, const float* xs,
                            const uint16_t* t, uint16_t* y, void* stream) {
  const char* fn = "qwam_asp_linear";
  qwam_status s = check_layer(fn, L, true);
  if (s != QWAM_OK) return s;
  if ((s = check_m(fn, M)) != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(L->wq);
  QWAM_REQUIRE_PTR(L->ws);
  QWAM_REQUIRE_PTR(L->wsp);
  QWAM_REQUIRE_PTR(L->L2t);
  if (L->bias != nullptr && !aligned16(L->bias))
    return fail(QWAM_ERR_MISALIGNED, "%s: bias is not 16-byte aligned", fn);
  QWAM_REQUIRE_PTR(xq);
  QWAM_REQUIRE_PTR(xs);
  QWAM_REQUIRE_PTR(t);
  QWAM_REQUIRE_PTR(y);
  // the kernel addresses each scale array with 32-bit byte offsets
  if (static_cast<int64_t>(M) * (L->K / L->group) >= (int64_t(1) << 29) ||
      static_cast<int64_t>(L->N) * (L->K / L->group) >= (int64_t(1) << 29))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: M*K/group and N*K/group must be below 2^29", fn);
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_asp_gemm(M, L->N, L->K, L->r, L->group, xq, xs, t, L->wq, L->ws, L->wsp, L->L2t,
                                            L->bias, y, static_cast<hipStream_t>(stream)));
}

int32_t qwam_probe_gemm_form(int32_t M, int32_t N, int32_t K, int32_t group) {
  const char* fn = "qwam_probe_gemm_form";
  if (check_kn(fn, K, N, group) != QWAM_OK || check_m(fn, M) != QWAM_OK) return -1;
  if (M <= qwam::kSmallM) return qwam::small_staged(K) ? QWAM_PROBE_GEMM_FEW_STAGED : QWAM_PROBE_GEMM_FEW_DIRECT;
  switch (qwam::gemm_form(M, N, K, group)) {
    case qwam::GemmForm::kLarge: return QWAM_PROBE_GEMM_LARGE;
    case qwam::GemmForm::kLargeSplit: return QWAM_PROBE_GEMM_LARGE_HALVES;
    case qwam::GemmForm::k32x64Waves8: return QWAM_PROBE_GEMM_32X64_W8;
    case qwam::GemmForm::k32x64Waves4: return QWAM_PROBE_GEMM_32X64_W4;
    case qwam::GemmForm::k64x64Waves4: return QWAM_PROBE_GEMM_64X64_W4;
  }
  return -1;
}

qwam_status qwam_debug_group_partials(const qwam_layer* L, int32_t M, const uint8_t* xq, int32_t* P,
                                      void* stream) {
  const char* fn = "qwam_debug_group_partials";
  qwam_status s = check_layer(fn, L, false);
  if (s != QWAM_OK) return s;
  if ((s = check_m(fn, M)) != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(L->wq);
  QWAM_REQUIRE_PTR(xq);
  QWAM_REQUIRE_PTR(P);
  if (static_cast<int64_t>(M) * L->N * (L->K / L->group) > (int64_t(1) << 34))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: M*N*K/group too large for a partials dump", fn);
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_group_partials(M, L->N, L->K, L->group, xq, L->wq, P,
                                                  static_cast<hipStream_t>(stream)));
}

qwam_status qwam_asp_layer(const qwam_layer* L, int32_t M, const uint16_t* x, uint16_t* y, uint8_t* xq, float* xs,
                           uint16_t* t, void* stream) {
  const char* fn = "qwam_asp_layer";
  qwam_status s = check_layer(fn, L, true);
  if (s != QWAM_OK) return s;
  if ((s = check_m(fn, M)) != QWAM_OK) return s;
  if (M > qwam::kSmallM) return fail(QWAM_ERR_UNSUPPORTED, "%s: M = %d exceeds %d", fn, M, qwam::kSmallM);
  if (L->r != 16 && L->r != 32) return fail(QWAM_ERR_UNSUPPORTED, "%s: rank r must be 16 or 32 (got %d)", fn, L->r);
  if (L->group != QWAM_GROUP || L->hadamard != 0)
    return fail(QWAM_ERR_UNSUPPORTED, "%s: group 64 without rotation only", fn);
  if (L->K > 16384) return fail(QWAM_ERR_UNSUPPORTED, "%s: K = %d exceeds 16384", fn, L->K);
  QWAM_REQUIRE_PTR(L->wq);
  QWAM_REQUIRE_PTR(L->ws);
  QWAM_REQUIRE_PTR(L->inv_smooth);
  QWAM_REQUIRE_PTR(L->L1t);
  QWAM_REQUIRE_PTR(L->L2t);
  if (L->bias != nullptr && !aligned16(L->bias))
    return fail(QWAM_ERR_MISALIGNED, "%s: bias is not 16-byte aligned", fn);
  QWAM_REQUIRE_PTR(x);
  QWAM_REQUIRE_PTR(y);
  const int given = (xq != nullptr) + (xs != nullptr) + (t != nullptr);
  if (given != 0 && given != 3) return fail(QWAM_ERR_INVALID_ARG, "%s: xq, xs and t must be all NULL or all set", fn);
  if (given == 3) {
    QWAM_REQUIRE_PTR(xq);
    QWAM_REQUIRE_PTR(xs);
    QWAM_REQUIRE_PTR(t);
  }
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_asp_layer_small(M, L->N, L->K, L->r, x, L->inv_smooth, L->L1t, L->wq, L->ws,
                                                   L->L2t, L->bias, y, xq, xs, t, static_cast<hipStream_t>(stream)));
}

qwam_status qwam_aog_accumulate(int32_t d, int32_t n, const uint16_t* gT, float* A, void* stream) {
  const char* fn = "qwam_aog_accumulate";
  if (d < 16 || d % 16 != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: d must be a positive multiple of 16 (got %d)", fn, d);
  if (n < 64 || n % 64 != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: n must be a positive multiple of 64 (got %d)", fn, n);
  if (d > 16384) return fail(QWAM_ERR_UNSUPPORTED, "%s: d = %d exceeds 16384", fn, d);
  if (static_cast<int64_t>(d) * n >= (int64_t(1) << 30))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: d * n must be below 2^30", fn);
  QWAM_REQUIRE_PTR(gT);
  QWAM_REQUIRE_PTR(A);
  qwam_status s = check_device(fn);
  if (s != QWAM_OK) return s;
  return launched(fn, qwam::launch_aog_accumulate(d, n, gT, A, static_cast<hipStream_t>(stream)));
}

}  // extern "C"

namespace {

qwam_status check_eig(const char* fn, int32_t d, int32_t r, int32_t iters, float scale, int32_t hadamard) {
  if (d < 128 || d % 64 != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: d must be a multiple of 64, at least 128 (got %d)", fn, d);
  if (d > 16384) return fail(QWAM_ERR_UNSUPPORTED, "%s: d = %d exceeds 16384", fn, d);
  if (r < 1 || r > qwam::kEigMaxRank)
    return fail(QWAM_ERR_UNSUPPORTED, "%s: r must be in [1, %d] (got %d)", fn, qwam::kEigMaxRank, r);
  if (iters < 0 || iters > 1000) return fail(QWAM_ERR_INVALID_ARG, "%s: iters must be in [0, 1000] (got %d)", fn, iters);
  if (!(scale > 0.0f) || !(scale < 3.0e38f))
    return fail(QWAM_ERR_INVALID_ARG, "%s: scale must be positive and finite", fn);
  if (hadamard != 0 && (hadamard < 16 || hadamard > 1024 || (hadamard & (hadamard - 1)) != 0 || d % hadamard != 0))
    return fail(QWAM_ERR_INVALID_ARG, "%s: hadamard must be 0 or a power of two in [16, 1024] dividing d (got %d)",
                fn, hadamard);
  return QWAM_OK;
}

}  // namespace

extern "C" {

int64_t qwam_aog_protected_basis_workspace(int32_t d, int32_t r) {
  if (check_eig("qwam_aog_protected_basis_workspace", d, r, 0, 1.0f, 0) != QWAM_OK) return -1;
  ok();
  return qwam::eig_workspace_bytes(d, r);
}

qwam_status qwam_aog_protected_basis(int32_t d, int32_t r, int32_t iters, const float* A, float scale,
                                     const float* lam, int32_t hadamard, float* V, float* evals, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
  const char* fn = "qwam_aog_protected_basis";
  qwam_status s = check_eig(fn, d, r, iters, scale, hadamard);
  if (s != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(A);
  QWAM_REQUIRE_PTR(V);
  QWAM_REQUIRE_PTR(evals);
  QWAM_REQUIRE_PTR(workspace);
  if (lam != nullptr && !aligned16(lam)) return fail(QWAM_ERR_MISALIGNED, "%s: lam is not 16-byte aligned", fn);
  const int64_t need = qwam::eig_workspace_bytes(d, r);
  if (workspace_bytes < need)
    return fail(QWAM_ERR_INVALID_ARG, "%s: workspace of %lld bytes is below the %lld needed", fn,
                static_cast<long long>(workspace_bytes), static_cast<long long>(need));
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_aog_eig(d, r, iters, A, scale, lam, hadamard, V, evals, workspace,
                                           static_cast<hipStream_t>(stream)));
}

}  // extern "C"

namespace {

qwam_status check_workspace(const char* fn, const void* workspace, int64_t bytes, int64_t need) {
  if (need <= 0) return QWAM_OK;
  if (workspace == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: workspace is NULL", fn);
  if (!aligned16(workspace)) return fail(QWAM_ERR_MISALIGNED, "%s: workspace is not 16-byte aligned", fn);
  if (bytes < need)
    return fail(QWAM_ERR_INVALID_ARG, "%s: workspace of %lld bytes, %lld needed", fn, static_cast<long long>(bytes),
                static_cast<long long>(need));
  return QWAM_OK;
}

qwam_status check_matvec(const char* fn, const qwam_layer* L, int32_t M) {
  qwam_status s = check_layer(fn, L, false);
  if (s != QWAM_OK) return s;
  if (L->r < 0 || L->r > 64 || L->r % 16 != 0)
    return fail(QWAM_ERR_UNSUPPORTED, "%s: rank r must be 0, 16, 32, 48 or 64 (got %d)", fn, L->r);
  if ((s = check_m(fn, M)) != QWAM_OK) return s;
  if (M > qwam::kMatvecMaxM) return fail(QWAM_ERR_UNSUPPORTED, "%s: M = %d exceeds %d", fn, M, qwam::kMatvecMaxM);
  if (static_cast<int64_t>(L->N) * (L->K / L->group) >= (int64_t(1) << 29))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: N*K/group must be below 2^29", fn);
  return QWAM_OK;
}

bool finite(float v) { return v - v == 0.0f; }

// elements of `bytes` bytes each lie at multiples of their size
bool aligned_to(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

#define QWAM_REQUIRE_ELEM(p, bytes)                                                                                  \
  do {                                                                                                               \
    if ((p) == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: %s is NULL", fn, #p);                                 \
    if (!aligned_to(p, bytes)) return fail(QWAM_ERR_MISALIGNED, "%s: %s is not aligned to its elements", fn, #p);    \
  } while (0)
#define QWAM_OPTIONAL_ELEM(p, bytes) \
  do {                               \
    if ((p) != nullptr) QWAM_REQUIRE_ELEM(p, bytes); \
  } while (0)

qwam_status check_norm_shape(const char* fn, const qwam_norm* p) {
  if (p == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: p is NULL", fn);
  if (p->T <= 0 || p->S <= 0 || p->T % p->S != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: T must be a positive multiple of S (got %d, %d)", fn, p->T, p->S);
  if (p->D <= 0) return fail(QWAM_ERR_INVALID_ARG, "%s: D must be >= 1 (got %d)", fn, p->D);
  if (p->D > qwam::kNormMaxD) return fail(QWAM_ERR_UNSUPPORTED, "%s: D = %d exceeds %d", fn, p->D, qwam::kNormMaxD);
  if (p->T > kMaxM) return fail(QWAM_ERR_UNSUPPORTED, "%s: T = %d exceeds %d", fn, p->T, kMaxM);
  return QWAM_OK;
}

// the gradients' sums over rows: one launch has a workgroup for each sample and 64 channels
qwam_status check_norm_samples(const char* fn, const qwam_norm* p) {
  if (static_cast<int64_t>(p->S) * ((p->D + 63) / 64) > (1 << 21))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: S * ceil(D / 64) must be at most 2^21", fn);
  return QWAM_OK;
}

qwam_status check_norm(const char* fn, const qwam_norm* p, qwam::NormParams* out) {
  qwam_status s = check_norm_shape(fn, p);
  if (s != QWAM_OK) return s;
  if (p->kind != QWAM_NORM_RMS && p->kind != QWAM_NORM_LAYER)
    return fail(QWAM_ERR_INVALID_ARG, "%s: kind must be QWAM_NORM_RMS or QWAM_NORM_LAYER (got %d)", fn, p->kind);
  if (!(p->eps >= 0.0f) || !finite(p->eps)) return fail(QWAM_ERR_INVALID_ARG, "%s: eps must be finite and >= 0", fn);
  if (!finite(p->residual_scale)) return fail(QWAM_ERR_INVALID_ARG, "%s: residual_scale must be finite", fn);
  QWAM_OPTIONAL_ELEM(p->gate, 2);
  QWAM_OPTIONAL_ELEM(p->scale, 2);
  QWAM_OPTIONAL_ELEM(p->shift, 2);
  QWAM_OPTIONAL_ELEM(p->post_weight, 2);
  QWAM_OPTIONAL_ELEM(p->weight, 2);
  *out = {p->D, p->T / p->S, p->kind == QWAM_NORM_LAYER, p->post != 0, p->x_f32 != 0, p->eps, p->residual_scale,
          p->gate, p->scale, p->shift, p->gate_stride, p->scale_stride, p->shift_stride, p->post_weight, p->weight};
  return QWAM_OK;
}

// the cache's integers
qwam_status check_cache_shape(const char* fn, const qwam_cache* c, qwam::CacheParams* out) {
  if (c == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: cache is NULL", fn);
  if (c->type != QWAM_CACHE_BF16 && c->type != QWAM_CACHE_FP8 && c->type != QWAM_CACHE_FP4)
    return fail(QWAM_ERR_INVALID_ARG, "%s: type must be QWAM_CACHE_BF16, QWAM_CACHE_FP8 or QWAM_CACHE_FP4 (got %d)", fn, c->type);
  const int32_t step = c->type == QWAM_CACHE_BF16 ? 8 : 16, width = c->type == QWAM_CACHE_FP4 ? qwam::kFp4Group : step;
  if (c->pages <= 0 || c->heads <= 0 || c->seqs <= 0 || c->table_width <= 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: pages, heads, seqs and table_width must be >= 1", fn);
  if (c->page_size < 16 || c->page_size > 4096 || (c->page_size & (c->page_size - 1)) != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: page_size must be a power of two in [16, 4096] (got %d)", fn, c->page_size);
  if (c->dim <= 0 || c->dim % width != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: dim must be a positive multiple of %d (got %d)", fn, width, c->dim);
  if (c->dim > 256) return fail(QWAM_ERR_UNSUPPORTED, "%s: dim = %d exceeds 256", fn, c->dim);
  if (c->heads > 4096 || c->seqs > 65535)
    return fail(QWAM_ERR_UNSUPPORTED, "%s: at most 4096 heads and 65535 sequences", fn);
  if (static_cast<int64_t>(c->table_width) * c->page_size > INT32_MAX)
    return fail(QWAM_ERR_UNSUPPORTED, "%s: table_width * page_size must be below 2^31", fn);
  if (c->reserved != 0) return fail(QWAM_ERR_INVALID_ARG, "%s: reserved must be 0", fn);
  if (c->page_stride % step != 0 || c->head_stride % step != 0 || c->row_stride % step != 0)
    return fail(QWAM_ERR_MISALIGNED, "%s: the cache's strides must be multiples of %d", fn, step);
  // 16 rows are addressed with 32-bit byte offsets
  if (c->row_stride <= -(1 << 26) || c->row_stride >= (1 << 26))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: row_stride must be within 2^26", fn);
  *out = {c->pages, __builtin_ctz(static_cast<unsigned>(c->page_size)), c->heads, c->dim, c->seqs, c->table_width,
          c->page_stride, c->head_stride, c->row_stride, c->k, c->v, nullptr, nullptr, c->table, nullptr, nullptr};
  if (c->type == QWAM_CACHE_FP8) {
    out->k_scale = static_cast<const float*>(c->k_scale);
    out->v_scale = static_cast<const float*>(c->v_scale);
  } else if (c->type == QWAM_CACHE_FP4) {
    out->k_exp = static_cast<uint8_t*>(const_cast<void*>(c->k_scale));
    out->v_exp = static_cast<uint8_t*>(const_cast<void*>(c->v_scale));
  }
  return QWAM_OK;
}

qwam::CacheType type_of(const qwam_cache* c) { return static_cast<qwam::CacheType>(c->type); }

qwam_status check_cache(const char* fn, const qwam_cache* c, qwam::CacheParams* out) {
  qwam_status s = check_cache_shape(fn, c, out);
  if (s != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(c->k);
  QWAM_REQUIRE_PTR(c->v);
  QWAM_REQUIRE_ELEM(c->table, 4);
  if (c->type == QWAM_CACHE_FP8) {
    QWAM_REQUIRE_ELEM(c->k_scale, 4);
    QWAM_REQUIRE_ELEM(c->v_scale, 4);
  } else if (c->type == QWAM_CACHE_FP4) {
    QWAM_REQUIRE_PTR(c->k_scale);
    QWAM_REQUIRE_PTR(c->v_scale);
  }
  return QWAM_OK;
}

// the arguments that the calls on a list of tokens share
qwam_status check_tokens(const char* fn, const qwam_cache* c, int32_t tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                         int64_t v_stride, const int32_t* seq, const int32_t* pos) {
  if (tokens <= 0) return fail(QWAM_ERR_INVALID_ARG, "%s: tokens must be >= 1 (got %d)", fn, tokens);
  if (static_cast<int64_t>(tokens) * c->heads * c->dim > (int64_t(1) << 32))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: tokens * heads * dim must be at most 2^32", fn);
  QWAM_REQUIRE_PTR(k);
  QWAM_REQUIRE_PTR(v);
  if (k_stride % 8 != 0 || v_stride % 8 != 0)
    return fail(QWAM_ERR_MISALIGNED, "%s: k_stride and v_stride must be multiples of 8", fn);
  QWAM_REQUIRE_ELEM(seq, 4);
  QWAM_REQUIRE_ELEM(pos, 4);
  return QWAM_OK;
}

// whether the rows of an output lie apart from each other
bool rows_apart(int32_t rows, int64_t stride, int64_t width) {
  return rows <= 1 || stride >= width || stride <= -width;
}

// Whether rows of `width` elements, `rows` of them s apart from p on, and as many t apart from q on, have an element in common.
// (Rows of one stride need one turn of the loop.  The places of others repeat after t / gcd(s, t) turns, and rows that fit the
// memory have no more than half a million before that.)
bool rows_meet(const uint16_t* p, int64_t s, const uint16_t* q, int64_t t, int32_t rows, int64_t width) {
  typedef __int128 wide;                // (strides are any)
  wide a = static_cast<wide>(reinterpret_cast<uintptr_t>(p) / 2), b = static_cast<wide>(reinterpret_cast<uintptr_t>(q) / 2);
  wide sp = rows > 1 ? s : width, tq = rows > 1 ? t : width;
  const wide last = rows - 1;
  if (sp < 0) a += last * sp, sp = -sp;
  if (tq < 0) b += last * tq, tq = -tq;
  const wide end = b + last * tq + width;
  wide first = -1;
  for (wide i = a + width <= b ? (b - width - a) / sp + 1 : 0; i <= last && a + i * sp < end; ++i) {
    const wide from = a + i * sp - b, place = from < 0 ? from + tq : from % tq;       // (from > -width)
    if (place < width || place > tq - width) return true;
    if (place == first) return false;
    if (first < 0) first = place;
  }
  return false;
}

qwam_status check_attention(const char* fn, const qwam_cache* c, const qwam::CacheParams& cp, int32_t q_heads, int32_t max_len) {
  if (q_heads <= 0 || q_heads % c->heads != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: q_heads must be a positive multiple of heads (got %d, %d)", fn, q_heads, c->heads);
  if (q_heads / c->heads > qwam::kMaxHeadGroup)
    return fail(QWAM_ERR_UNSUPPORTED, "%s: more than %d query heads per key head", fn, qwam::kMaxHeadGroup);
  if (static_cast<int64_t>(c->seqs) * q_heads > (1 << 22))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: seqs * q_heads must be at most 2^22", fn);
  if (max_len < 1 || max_len > static_cast<int64_t>(c->table_width) * c->page_size)
    return fail(QWAM_ERR_INVALID_ARG, "%s: max_len must be in [1, table_width * page_size] (got %d)", fn, max_len);
  // the kernels count positions in 32 bits, up to a range past the last
  if (static_cast<int64_t>(max_len) + qwam::kMaxChunk > (int64_t(1) << 31))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: max_len = %d exceeds 2^31 - %d", fn, max_len, qwam::kMaxChunk);
  if (!qwam::paged_attention_fits(cp, type_of(c), q_heads, max_len))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: too many sequences and heads of too long a max_len for one launch", fn);
  return QWAM_OK;
}

}  // namespace

extern "C" {

int64_t qwam_asp_matvec_workspace(const qwam_layer* L, int32_t M) {
  if (check_matvec("qwam_asp_matvec_workspace", L, M) != QWAM_OK) return -1;
  ok();
  return qwam::matvec_workspace_bytes(M, L->N, L->K, L->r, L->hadamard);
}

qwam_status qwam_asp_matvec(const qwam_layer* L, int32_t M, const uint16_t* x, uint16_t* y, void* workspace,
                            int64_t workspace_bytes, void* stream) {
  const char* fn = "qwam_asp_matvec";
  qwam_status s = check_matvec(fn, L, M);
  if (s != QWAM_OK) return s;
  QWAM_REQUIRE_PTR(L->wq);
  QWAM_REQUIRE_PTR(L->ws);
  if (L->r > 0) {
    QWAM_REQUIRE_PTR(L->L1f);
    QWAM_REQUIRE_PTR(L->L2t);
  }
  if (L->inv_smooth != nullptr && !aligned16(L->inv_smooth))
    return fail(QWAM_ERR_MISALIGNED, "%s: inv_smooth is not 16-byte aligned", fn);
  if (L->bias != nullptr && !aligned16(L->bias))
    return fail(QWAM_ERR_MISALIGNED, "%s: bias is not 16-byte aligned", fn);
  QWAM_REQUIRE_PTR(x);
  QWAM_REQUIRE_PTR(y);
  if ((s = check_workspace(fn, workspace, workspace_bytes, qwam::matvec_workspace_bytes(M, L->N, L->K, L->r, L->hadamard))) != QWAM_OK)
    return s;
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_asp_matvec(M, L->N, L->K, L->r, L->group, L->hadamard, x, L->inv_smooth, L->L1f, L->wq, L->ws, L->L2t,
                                              L->bias, y, workspace, static_cast<hipStream_t>(stream)));
}

qwam_status qwam_block_norm(const qwam_norm* p, const void* x, const uint16_t* branch, void* x_out, uint16_t* h, void* stream) {
  const char* fn = "qwam_block_norm";
  qwam::NormParams np;
  qwam_status s = check_norm(fn, p, &np);
  if (s != QWAM_OK) return s;
  const uintptr_t xe = np.x_f32 ? 4 : 2;
  QWAM_REQUIRE_ELEM(x, xe);
  QWAM_REQUIRE_ELEM(h, 2);
  if (branch != nullptr) {
    QWAM_REQUIRE_ELEM(branch, 2);
    QWAM_REQUIRE_ELEM(x_out, xe);
  } else if (x_out != nullptr) {
    return fail(QWAM_ERR_INVALID_ARG, "%s: x_out without a branch", fn);
  }
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_block_norm(np, p->T, x, branch, x_out, h, static_cast<hipStream_t>(stream)));
}

int64_t qwam_block_norm_backward_workspace(const qwam_norm* p) {
  const char* fn = "qwam_block_norm_backward_workspace";
  if (check_norm_shape(fn, p) != QWAM_OK || check_norm_samples(fn, p) != QWAM_OK) return -1;
  ok();
  return qwam::block_norm_bwd_workspace_bytes(p->T, p->D, p->S);
}

qwam_status qwam_block_norm_backward(const qwam_norm* p, const void* dx_out, const uint16_t* dh, const void* x_out,
                                     const uint16_t* branch, void* dx, uint16_t* dbranch, float* dgate, float* dscale,
                                     float* dshift, float* dpost_weight, float* dweight, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
  const char* fn = "qwam_block_norm_backward";
  qwam::NormParams np;
  qwam_status s = check_norm(fn, p, &np);
  if (s != QWAM_OK) return s;
  const uintptr_t xe = np.x_f32 ? 4 : 2;
  QWAM_OPTIONAL_ELEM(dx_out, xe);
  QWAM_REQUIRE_ELEM(dh, 2);
  QWAM_REQUIRE_ELEM(x_out, xe);
  QWAM_OPTIONAL_ELEM(branch, 2);
  QWAM_REQUIRE_ELEM(dx, xe);
  QWAM_OPTIONAL_ELEM(dbranch, 2);
  QWAM_OPTIONAL_ELEM(dgate, 4);
  QWAM_OPTIONAL_ELEM(dscale, 4);
  QWAM_OPTIONAL_ELEM(dshift, 4);
  QWAM_OPTIONAL_ELEM(dpost_weight, 4);
  QWAM_OPTIONAL_ELEM(dweight, 4);
  if (branch == nullptr && (dbranch != nullptr || dgate != nullptr || dpost_weight != nullptr))
    return fail(QWAM_ERR_INVALID_ARG, "%s: dbranch, dgate or dpost_weight without a branch", fn);
  if ((s = check_norm_samples(fn, p)) != QWAM_OK) return s;
  if (!np.post && dpost_weight != nullptr)
    return fail(QWAM_ERR_INVALID_ARG, "%s: dpost_weight without a post-norm", fn);
  if ((s = check_workspace(fn, workspace, workspace_bytes, qwam::block_norm_bwd_workspace_bytes(p->T, p->D, p->S))) != QWAM_OK)
    return s;
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_block_norm_bwd(np, p->T, dx_out, dh, x_out, branch, dx, dbranch, dgate, dscale, dshift,
                                                  dpost_weight, dweight, workspace, static_cast<hipStream_t>(stream)));
}

qwam_status qwam_kv_append(const qwam_cache* c, int32_t tokens, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                           int64_t v_stride, const int32_t* seq, const int32_t* pos, void* stream) {
  const char* fn = "qwam_kv_append";
  qwam::CacheParams cp;
  qwam_status s = check_cache(fn, c, &cp);
  if (s != QWAM_OK) return s;
  if ((s = check_tokens(fn, c, tokens, k, k_stride, v, v_stride, seq, pos)) != QWAM_OK) return s;
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_kv_append(cp, type_of(c), tokens, k, k_stride, v, v_stride, seq, pos,
                                             static_cast<hipStream_t>(stream)));
}

qwam_status qwam_kv_read(const qwam_cache* c, int32_t tokens, const int32_t* seq, const int32_t* pos, uint16_t* k, int64_t k_stride,
                         uint16_t* v, int64_t v_stride, void* stream) {
  const char* fn = "qwam_kv_read";
  qwam::CacheParams cp;
  qwam_status s = check_cache(fn, c, &cp);
  if (s != QWAM_OK) return s;
  if ((s = check_tokens(fn, c, tokens, k, k_stride, v, v_stride, seq, pos)) != QWAM_OK) return s;
  const int64_t width = static_cast<int64_t>(c->heads) * c->dim;
  if (!rows_apart(tokens, k_stride, width) || !rows_apart(tokens, v_stride, width))
    return fail(QWAM_ERR_INVALID_ARG, "%s: k_stride and v_stride must be at least heads * dim apart", fn);
  if (k == v) return fail(QWAM_ERR_INVALID_ARG, "%s: k and v are one output", fn);
  if (rows_meet(k, k_stride, v, v_stride, tokens, width)) return fail(QWAM_ERR_INVALID_ARG, "%s: k and v overlap", fn);
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_kv_read(cp, type_of(c), tokens, seq, pos, k, k_stride, v, v_stride,
                                           static_cast<hipStream_t>(stream)));
}

int64_t qwam_paged_attention_workspace(const qwam_cache* c, int32_t q_heads, int32_t max_len) {
  const char* fn = "qwam_paged_attention_workspace";
  qwam::CacheParams cp;
  if (check_cache_shape(fn, c, &cp) != QWAM_OK || check_attention(fn, c, cp, q_heads, max_len) != QWAM_OK) return -1;
  ok();
  return qwam::paged_attention_workspace_bytes(cp, type_of(c), q_heads, max_len);
}

qwam_status qwam_paged_attention(const qwam_cache* c, int32_t q_heads, const uint16_t* q, int64_t q_stride,
                                 const int32_t* lengths, const int32_t* starts, int32_t max_len, float scale, uint16_t* out,
                                 void* workspace, int64_t workspace_bytes, void* stream) {
  const char* fn = "qwam_paged_attention";
  qwam::CacheParams cp;
  qwam_status s = check_cache(fn, c, &cp);
  if (s != QWAM_OK) return s;
  if ((s = check_attention(fn, c, cp, q_heads, max_len)) != QWAM_OK) return s;
  if (!finite(scale)) return fail(QWAM_ERR_INVALID_ARG, "%s: scale must be finite", fn);
  QWAM_REQUIRE_PTR(q);
  if (q_stride % 8 != 0) return fail(QWAM_ERR_MISALIGNED, "%s: q_stride must be a multiple of 8", fn);
  QWAM_REQUIRE_ELEM(lengths, 4);
  QWAM_OPTIONAL_ELEM(starts, 4);
  QWAM_REQUIRE_PTR(out);
  if ((s = check_workspace(fn, workspace, workspace_bytes, qwam::paged_attention_workspace_bytes(cp, type_of(c), q_heads, max_len))) !=
      QWAM_OK)
    return s;
  if ((s = check_device(fn)) != QWAM_OK) return s;
  return launched(fn, qwam::launch_paged_attention(cp, type_of(c), q_heads, q, q_stride, lengths, starts, max_len, scale, out, workspace,
                                                   static_cast<hipStream_t>(stream)));
}

qwam_status qwam_rope(const qwam_rope_plan* p, int32_t tokens, int32_t inverse, const void* x, int64_t x_stride, void* y,
                      int64_t y_stride, void* stream) {
  const char* fn = "qwam_rope";
  if (p == nullptr) return fail(QWAM_ERR_INVALID_ARG, "%s: p is NULL", fn);
  if (p->heads <= 0 || p->dim <= 0 || p->positions <= 0 || tokens <= 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: heads, dim, positions and tokens must be >= 1 (got %d, %d, %d, %d)", fn, p->heads, p->dim,
                p->positions, tokens);
  if (p->pairs <= 0 || p->pairs > p->dim / 2)
    return fail(QWAM_ERR_INVALID_ARG, "%s: pairs must be in [1, dim / 2] (got %d for dim = %d)", fn, p->pairs, p->dim);
  if (p->axes <= 0 || p->axes > qwam::kRopeMaxAxes)
    return fail(QWAM_ERR_INVALID_ARG, "%s: axes must be in [1, %d] (got %d)", fn, qwam::kRopeMaxAxes, p->axes);
  if (tokens % p->positions != 0)
    return fail(QWAM_ERR_INVALID_ARG, "%s: tokens must be a multiple of positions (got %d, %d)", fn, tokens, p->positions);
  if (p->dim > qwam::kRopeMaxDim) return fail(QWAM_ERR_UNSUPPORTED, "%s: dim = %d exceeds %d", fn, p->dim, qwam::kRopeMaxDim);
  // (in two steps: the product of the three passes 64 bits)
  const int64_t width = static_cast<int64_t>(p->heads) * p->dim;
  if (width > (int64_t(1) << 32) || width * tokens > (int64_t(1) << 32))
    return fail(QWAM_ERR_UNSUPPORTED, "%s: tokens * heads * dim must be at most 2^32", fn);
  const uintptr_t xe = p->x_f32 ? 4 : 2;
  QWAM_REQUIRE_ELEM(p->pos, 4);
  QWAM_REQUIRE_ELEM(p->inv_freq, 4);
  QWAM_REQUIRE_ELEM(p->axis, 4);
  QWAM_REQUIRE_ELEM(x, xe);
  QWAM_REQUIRE_ELEM(y, xe);
  if (!rows_apart(tokens, y_stride, width))
    return fail(QWAM_ERR_INVALID_ARG, "%s: y_stride must be at least heads * dim apart", fn);
  if (x == y && tokens > 1 && x_stride != y_stride)
    return fail(QWAM_ERR_INVALID_ARG, "%s: y is x with another stride", fn);
  qwam_status s = check_device(fn);
  if (s != QWAM_OK) return s;
  const qwam::RopeParams rp = {p->heads, p->dim, p->pairs, p->axes, p->positions, p->interleaved != 0, p->pos_f32 != 0, p->x_f32 != 0,
                               p->pos, p->inv_freq, p->axis};
  return launched(fn, qwam::launch_rope(rp, tokens, inverse != 0, x, x_stride, y, y_stride, static_cast<hipStream_t>(stream)));
}

const char* qwam_last_error(void) { return g_err; }

const char* qwam_status_string(qwam_status s) {
  switch (s) {
    case QWAM_OK: return "QWAM_OK";
    case QWAM_ERR_INVALID_ARG: return "QWAM_ERR_INVALID_ARG";
    case QWAM_ERR_UNSUPPORTED: return "QWAM_ERR_UNSUPPORTED";
    case QWAM_ERR_MISALIGNED: return "QWAM_ERR_MISALIGNED";
    case QWAM_ERR_NO_DEVICE: return "QWAM_ERR_NO_DEVICE";
    case QWAM_ERR_HIP: return "QWAM_ERR_HIP";
  }
  return "QWAM_ERR_UNKNOWN";
}

int32_t qwam_abi_version(void) { return QWAM_ABI_VERSION; }

}  // extern "C"
