// C ABI of the operators around the layer: block norms, router, expert order, gradient
// clipping. Arguments are checked here, before any launch; the kernels are in block.hip,
// route.hip, experts.hip and gradients.hip.
#include <hip/hip_runtime.h>

#include <cmath>

#include "block.h"
#include "common.h"

using namespace sfl;

namespace {

bool dtype_ok(int32_t t) { return t == SFL_F32 || t == SFL_BF16; }

// Rows times width stays within the 64-bit byte offsets of the kernels.
bool size_ok(int64_t rows, int64_t d) { return rows >= 0 && d >= 1 && rows <= ((int64_t)1 << 60) / d; }

// A workspace of `need` bytes that holds values of `align` bytes.
sfl_status_t check_space(const void* workspace, size_t bytes, size_t need, size_t align) {
  if (need == 0) return SFL_OK;
  if (!workspace || bytes < need) return SFL_E_WORKSPACE;
  return (uintptr_t)workspace % align ? SFL_E_ARG : SFL_OK;
}

sfl_status_t status(hipError_t e) { return e == hipSuccess ? SFL_OK : SFL_E_HIP; }

sfl_status_t check_norm(sfl_dtype_t dtype, int32_t norms, int64_t T, int64_t d, float eps, const void* Y,
                        const float* w_pre, const float* w_post, const float* gate_c, const float* gate_t) {
  if (!dtype_ok(dtype) || (norms & ~(SFL_NORM_PRE | SFL_NORM_POST)) || !size_ok(T, d) || !(eps >= 0.f)) return SFL_E_ARG;
  if (w_pre && !(norms & SFL_NORM_PRE)) return SFL_E_ARG;
  if (w_post && !(norms & SFL_NORM_POST)) return SFL_E_ARG;
  if (T > 0 && !Y && ((norms & SFL_NORM_POST) || gate_c || gate_t)) return SFL_E_ARG;
  if (d > kNormMaxWidth) return SFL_E_UNSUPPORTED;
  return SFL_OK;
}

sfl_status_t check_route(const void* logits, sfl_dtype_t dtype, int64_t T, int32_t E, int32_t k, int32_t normalise) {
  if (!dtype_ok(dtype) || T < 0 || E < 1 || k < 1 || k > E || (normalise != 0 && normalise != 1)) return SFL_E_ARG;
  if (E > kRouteMaxExperts || k > kRouteMaxK || T > INT32_MAX) return SFL_E_UNSUPPORTED;
  if (T > 0 && !logits) return SFL_E_ARG;
  return SFL_OK;
}

sfl_status_t check_slots(int64_t T, int32_t k) {
  if (T < 0 || k < 1) return SFL_E_ARG;
  if (k > kRouteMaxK || T > INT32_MAX / k) return SFL_E_UNSUPPORTED;
  return SFL_OK;
}

sfl_status_t check_rows(sfl_dtype_t dtype, int64_t T, int64_t d, int32_t k, int64_t rows) {
  const sfl_status_t st = check_slots(T, k);
  if (st != SFL_OK) return st;
  if (!dtype_ok(dtype) || !size_ok(T, d) || !size_ok(rows, d)) return SFL_E_ARG;
  return d > ((int64_t)1 << 30) ? SFL_E_UNSUPPORTED : SFL_OK;
}

sfl_status_t check_grads(const sfl_grad_t* list, int32_t n) {
  if (n < 0 || (n > 0 && !list)) return SFL_E_ARG;
  for (int32_t i = 0; i < n; ++i)
    if (list[i].n < 0 || list[i].n > ((int64_t)1 << 40) || !dtype_ok(list[i].dtype) || (list[i].n > 0 && !list[i].src))
      return SFL_E_ARG;
  return SFL_OK;
}

}  // namespace

extern "C" {

sfl_status_t sfl_norm_forward(const sfl_norm_args_t* a, sfl_stream_t stream) {
  if (!a) return SFL_E_ARG;
  const sfl_status_t st =
      check_norm(a->dtype, a->norms, a->T, a->d, a->eps, a->Y, a->w_pre, a->w_post, a->gate_c, a->gate_t);
  if (st != SFL_OK) return st;
  const bool pre = a->norms & SFL_NORM_PRE;
  if (a->N && !pre) return SFL_E_ARG;
  if (a->T == 0) return SFL_OK;
  if (!a->X || (pre ? !a->N : !a->X_out)) return SFL_E_ARG;
  NormParams p{};
  p.T = a->T;
  p.d = a->d;
  p.X = a->X;
  p.Y = a->Y;
  p.w_pre = a->w_pre;
  p.w_post = a->w_post;
  p.gate_c = a->gate_c;
  p.gate_t = a->gate_t;
  p.X_out = a->X_out;
  p.N = a->N;
  p.eps = a->eps;
  p.res_scale = a->res_scale;
  p.pre = pre;
  p.post = (a->norms & SFL_NORM_POST) != 0;
  return status(launch_norm_fwd(p, a->dtype == SFL_BF16, (hipStream_t)stream));
}

sfl_status_t sfl_norm_workspace_size(int64_t T, int64_t d, sfl_dtype_t dtype, size_t* bytes) {
  if (!bytes || !dtype_ok(dtype) || !size_ok(T, d)) return SFL_E_ARG;
  if (d > kNormMaxWidth) return SFL_E_UNSUPPORTED;
  *bytes = norm_workspace_bytes(T, d, dtype == SFL_BF16);
  return SFL_OK;
}

sfl_status_t sfl_norm_backward(const sfl_norm_bwd_args_t* a, sfl_stream_t stream) {
  if (!a) return SFL_E_ARG;
  sfl_status_t st =
      check_norm(a->dtype, a->norms, a->T, a->d, a->eps, a->Y, a->w_pre, a->w_post, a->gate_c, a->gate_t);
  if (st != SFL_OK) return st;
  const bool pre = a->norms & SFL_NORM_PRE, post = a->norms & SFL_NORM_POST;
  if ((a->dN || a->dw_pre) && !pre) return SFL_E_ARG;
  if (a->dw_post && !post) return SFL_E_ARG;
  if (a->T > 0 && ((pre && !a->X_out) || (!a->Y && (a->dY || a->dgate_c || a->dgate_t)))) return SFL_E_ARG;
  const size_t need = norm_workspace_bytes(a->T, a->d, a->dtype == SFL_BF16);
  st = check_space(a->workspace, a->workspace_bytes, need, sizeof(float));
  if (st != SFL_OK) return st;
  NormBwdParams p{};
  p.T = a->T;
  p.d = a->d;
  p.X_out = a->X_out;
  p.Y = a->Y;
  p.dX_out = a->dX_out;
  p.dN = a->dN;
  p.w_pre = a->w_pre;
  p.w_post = a->w_post;
  p.gate_c = a->gate_c;
  p.gate_t = a->gate_t;
  p.dX = a->dX;
  p.dY = a->dY;
  p.dw_pre = a->dw_pre;
  p.dw_post = a->dw_post;
  p.dgate_c = a->dgate_c;
  p.dgate_t = a->dgate_t;
  p.part = (float*)a->workspace;
  p.eps = a->eps;
  p.res_scale = a->res_scale;
  p.pre = pre;
  p.post = post;
  return status(launch_norm_bwd(p, a->dtype == SFL_BF16, (hipStream_t)stream));
}

sfl_status_t sfl_route_forward(const void* logits, sfl_dtype_t dtype, int64_t T, int32_t E, int32_t k,
                               int32_t normalise, float scale, int32_t* expert, float* weight, sfl_stream_t stream) {
  const sfl_status_t st = check_route(logits, dtype, T, E, k, normalise);
  if (st != SFL_OK || T == 0) return st;
  if (!expert || !weight) return SFL_E_ARG;
  return status(launch_route_fwd(logits, dtype == SFL_BF16, T, E, k, normalise, scale, expert, weight,
                                 (hipStream_t)stream));
}

sfl_status_t sfl_route_backward(const void* logits, sfl_dtype_t dtype, int64_t T, int32_t E, int32_t k,
                                int32_t normalise, float scale, const int32_t* expert, const float* dweight,
                                void* dlogits, sfl_stream_t stream) {
  const sfl_status_t st = check_route(logits, dtype, T, E, k, normalise);
  if (st != SFL_OK || T == 0) return st;
  if (!expert || !dweight || !dlogits) return SFL_E_ARG;
  return status(launch_route_bwd(logits, dtype == SFL_BF16, T, E, k, normalise, scale, expert, dweight, dlogits,
                                 (hipStream_t)stream));
}

sfl_status_t sfl_expert_workspace_size(int64_t T, int32_t k, int32_t E, size_t* bytes) {
  const sfl_status_t st = check_slots(T, k);
  if (!bytes || E < 1) return SFL_E_ARG;
  if (st != SFL_OK) return st;
  if (E > kRouteMaxExperts) return SFL_E_UNSUPPORTED;
  *bytes = expert_workspace_bytes(T, k, E);
  return SFL_OK;
}

sfl_status_t sfl_expert_dispatch(const int32_t* expert, int64_t T, int32_t k, int32_t E, int32_t* pos,
                                 int32_t* offsets, const void* X, sfl_dtype_t dtype, int64_t d, int64_t rows, void* Xs,
                                 void* workspace, size_t workspace_bytes, sfl_stream_t stream) {
  sfl_status_t st = check_rows(dtype, T, d, k, rows);
  if (st != SFL_OK) return st;
  if (E < 1 || !offsets) return SFL_E_ARG;
  if (E > kRouteMaxExperts) return SFL_E_UNSUPPORTED;
  if (T > 0 && (!expert || !pos || (X && !Xs && rows > 0) || (Xs && !X))) return SFL_E_ARG;
  st = check_space(workspace, workspace_bytes, expert_workspace_bytes(T, k, E), sizeof(int32_t));
  if (st != SFL_OK) return st;
  return status(launch_expert_dispatch(expert, T, k, E, pos, offsets, X, dtype == SFL_BF16, d, rows, Xs, workspace,
                                       (hipStream_t)stream));
}

sfl_status_t sfl_expert_combine(const void* Ys, sfl_dtype_t dtype, int64_t T, int64_t d, int32_t k, const int32_t* pos,
                                int64_t rows, const float* weight, void* Y, sfl_stream_t stream) {
  const sfl_status_t st = check_rows(dtype, T, d, k, rows);
  if (st != SFL_OK || T == 0) return st;
  if (!pos || !Y || (rows > 0 && !Ys)) return SFL_E_ARG;
  return status(launch_expert_combine(Ys, dtype == SFL_BF16, T, d, k, pos, rows, weight, Y, (hipStream_t)stream));
}

sfl_status_t sfl_expert_combine_backward(const void* dY, const void* Ys, sfl_dtype_t dtype, int64_t T, int64_t d,
                                         int32_t k, const int32_t* pos, int64_t rows, const float* weight, void* dYs,
                                         float* dweight, sfl_stream_t stream) {
  const sfl_status_t st = check_rows(dtype, T, d, k, rows);
  if (st != SFL_OK || T == 0) return st;
  if (!pos || !dY || (dweight && rows > 0 && !Ys)) return SFL_E_ARG;
  return status(launch_expert_combine_bwd(dY, Ys, dtype == SFL_BF16, T, d, k, pos, rows, weight, dYs, dweight,
                                          (hipStream_t)stream));
}

sfl_status_t sfl_grad_workspace_size(const sfl_grad_t* list, int32_t n, size_t* bytes) {
  const sfl_status_t st = check_grads(list, n);
  if (st != SFL_OK) return st;
  if (!bytes) return SFL_E_ARG;
  *bytes = grad_workspace_bytes(list, n);
  return SFL_OK;
}

sfl_status_t sfl_grad_sumsq(const sfl_grad_t* list, int32_t n, double* sumsq, void* workspace, size_t workspace_bytes,
                            sfl_stream_t stream) {
  sfl_status_t st = check_grads(list, n);
  if (st != SFL_OK) return st;
  if (!sumsq) return SFL_E_ARG;
  st = check_space(workspace, workspace_bytes, grad_workspace_bytes(list, n), sizeof(double));
  if (st != SFL_OK) return st;
  return status(launch_grad_sumsq(list, n, sumsq, (double*)workspace, (hipStream_t)stream));
}

sfl_status_t sfl_grad_clip(const sfl_grad_t* list, int32_t n, const double* sumsq, float max_norm, float* norm,
                           sfl_stream_t stream) {
  const sfl_status_t st = check_grads(list, n);
  if (st != SFL_OK) return st;
  if (!sumsq || !(max_norm >= 0.f)) return SFL_E_ARG;
  return status(launch_grad_clip(list, n, sumsq, max_norm, norm, (hipStream_t)stream));
}

}  // extern "C"
