// Launch interfaces of the operators around the layer (block.hip, route.hip, experts.hip,
// gradients.hip); api_block.cpp checks the arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sfl.h"

namespace sfl {

// ------------------------------------------------------- norms at a block's boundary ----
constexpr int64_t kNormMaxWidth = 16384;

struct NormParams {
  int64_t T, d;
  const void* X;
  const void* Y;  // may be null: X' = res_scale X
  const float* w_pre;
  const float* w_post;
  const float* gate_c;
  const float* gate_t;
  void* X_out;
  void* N;
  float eps, res_scale;
  int pre, post;
};
struct NormBwdParams {
  int64_t T, d;
  const void* X_out;
  const void* Y;
  const void* dX_out;
  const void* dN;
  const float* w_pre;
  const float* w_post;
  const float* gate_c;
  const float* gate_t;
  void* dX;
  void* dY;
  float* dw_pre;
  float* dw_post;
  float* dgate_c;
  float* dgate_t;
  float* part;  // norm_workspace_bytes(T, d, bf16)
  float eps, res_scale;
  int pre, post;
};
size_t norm_workspace_bytes(int64_t T, int64_t d, int bf16);
hipError_t launch_norm_fwd(const NormParams& p, int bf16, hipStream_t s);
hipError_t launch_norm_bwd(const NormBwdParams& p, int bf16, hipStream_t s);

// --------------------------------------------------------------------------- router ----
constexpr int kRouteMaxExperts = 1024;
constexpr int kRouteMaxK = 64;
hipError_t launch_route_fwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            int32_t* expert, float* weight, hipStream_t s);
hipError_t launch_route_bwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            const int32_t* expert, const float* dweight, void* dlogits, hipStream_t s);

// -------------------------------------------------------------------------- experts ----
size_t expert_workspace_bytes(int64_t T, int k, int E);
// pos[t k + j] = row of slot (t, j) in expert order (stable), -1 for an expert outside
// [0, E); offsets[e] = first row of expert e, offsets[E] = number of rows; and, where X is not
// null, Xs[pos[t k + j]] = X[t].
hipError_t launch_expert_dispatch(const int32_t* expert, int64_t T, int k, int E, int32_t* pos, int32_t* offsets,
                                  const void* X, int bf16, int64_t d, int64_t rows, void* Xs, void* workspace,
                                  hipStream_t s);
// Y[t] = sum_j w[t k + j] Ys[pos[t k + j]]
hipError_t launch_expert_combine(const void* Ys, int bf16, int64_t T, int64_t d, int k, const int32_t* pos,
                                 int64_t rows, const float* weight, void* Y, hipStream_t s);
// dYs[pos] = w dY[t], dw = <dY[t], Ys[pos]>
hipError_t launch_expert_combine_bwd(const void* dY, const void* Ys, int bf16, int64_t T, int64_t d, int k,
                                     const int32_t* pos, int64_t rows, const float* weight, void* dYs, float* dweight,
                                     hipStream_t s);

// ------------------------------------------------------------------------ gradients ----
size_t grad_workspace_bytes(const sfl_grad_t* list, int n);
hipError_t launch_grad_sumsq(const sfl_grad_t* list, int n, double* sumsq, double* part, hipStream_t s);
hipError_t launch_grad_clip(const sfl_grad_t* list, int n, const double* sumsq, float max_norm, float* norm,
                            hipStream_t s);

}  // namespace sfl
