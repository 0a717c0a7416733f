// C ABI of the operators for many routed experts in 8 bits: router with groups, quantisation, expert
// products, AdamW. Arguments are checked here, before any launch; the kernels are in
// route_groups.hip, quant.hip, product8.hip and adamw.hip.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

#include "routed.h"

using namespace sfl;

namespace {

bool dtype_ok(int32_t t) { return t == SFL_F32 || t == SFL_BF16; }
bool result_ok(int32_t t) { return dtype_ok(t) || t == SFL_BF16_FAST; }  // of a product
uintptr_t result_size(int32_t t) { return t == SFL_F32 ? 4 : 2; }
bool aligned(const void* p, uintptr_t by) { return (uintptr_t)p % by == 0; }
sfl_status_t status(hipError_t e) { return e == hipSuccess ? SFL_OK : SFL_E_HIP; }

// Rows of the router and choices of a row.
sfl_status_t check_scores(int32_t dtype, int32_t score, int64_t T, int32_t E, int32_t k, int32_t normalise) {
  if (!dtype_ok(dtype) || (score != SFL_SCORE_SIGMOID && score != SFL_SCORE_SOFTMAX) || T < 0 || E < 1 || k < 1 ||
      k > E || (normalise != 0 && normalise != 1))
    return SFL_E_ARG;
  return E > kRouteGroupsExperts || k > 64 || T > INT32_MAX ? SFL_E_UNSUPPORTED : SFL_OK;
}

// Tokens of E experts in runs: their columns and units are counted in 31 bits.
sfl_status_t check_runs(int64_t T, int64_t E) {
  if (T < 0 || E < 1) return SFL_E_ARG;
  if (E > kMaxExperts8 || T > INT32_MAX - (int64_t)kBlock8 * (E + 4)) return SFL_E_UNSUPPORTED;
  // also runs that overlap, which no meaningful offsets make, are counted without overflow
  return (T / kBlock8 + 1) * E > INT32_MAX ? SFL_E_UNSUPPORTED : SFL_OK;
}

// Codes and their scales: both or neither, aligned.
bool codes_ok(const void* Q, const void* S) { return !Q == !S && aligned(Q, 16) && aligned(S, 4); }

}  // namespace

extern "C" {

sfl_status_t sfl_route_groups_forward(const sfl_route_groups_args_t* a, sfl_stream_t stream) {
  if (!a) return SFL_E_ARG;
  const sfl_status_t st = check_scores(a->dtype, a->score, a->T, a->E, a->k, a->normalise);
  if (st == SFL_E_ARG) return st;
  if (a->groups < 1 || a->E % a->groups || a->group_k < 1 || a->group_k > a->groups || a->group_top < 1 ||
      a->group_top > 2 || a->k > (int64_t)a->group_k * (a->E / a->groups))
    return SFL_E_ARG;
  if (st != SFL_OK || a->T == 0) return st;
  if (!a->logits || !a->expert || !a->weight) return SFL_E_ARG;
  return status(launch_route_groups_fwd(*a, (hipStream_t)stream));
}

sfl_status_t sfl_route_groups_backward(const sfl_route_groups_bwd_args_t* a, sfl_stream_t stream) {
  if (!a) return SFL_E_ARG;
  const sfl_status_t st = check_scores(a->dtype, a->score, a->T, a->E, a->k, a->normalise);
  if (st != SFL_OK || a->T == 0) return st;
  if (!a->logits || !a->expert || !a->dweight || !a->dlogits) return SFL_E_ARG;
  return status(launch_route_groups_bwd(*a, (hipStream_t)stream));
}

sfl_status_t sfl_quant_columns(int64_t T, int32_t E, int64_t* columns) {
  const sfl_status_t st = check_runs(T, E);
  if (!columns) return SFL_E_ARG;
  if (st == SFL_OK) *columns = columns8(T, E);
  return st;
}

sfl_status_t sfl_quant_rows(const sfl_quant_args_t* a, sfl_stream_t stream) {
  if (!a) return SFL_E_ARG;
  sfl_status_t st = check_runs(a->T, a->E);
  if (st == SFL_E_ARG || !dtype_ok(a->dtype) || a->d < 1 || (!a->offsets && a->E != 1)) return SFL_E_ARG;
  if (st != SFL_OK || a->d > kMaxWidth8) return SFL_E_UNSUPPORTED;
  if (!codes_ok(a->Q, a->S) || !codes_ok(a->Qt, a->St)) return SFL_E_ARG;
  if (a->Qt && (a->columns % 512 || a->columns < columns8(a->T, a->E) || a->columns > INT32_MAX)) return SFL_E_ARG;
  if (a->T == 0) return SFL_OK;
  if (!a->X || !(a->Q || a->Qt)) return SFL_E_ARG;
  return status(launch_quant_rows(*a, (hipStream_t)stream));
}

sfl_status_t sfl_quant_weights(const void* W, sfl_dtype_t dtype, int64_t E, int64_t R, int64_t C, uint8_t* Q,
                               uint8_t* S, uint8_t* Qt, uint8_t* St, sfl_stream_t stream) {
  if (!dtype_ok(dtype) || E < 1 || R < 1 || C < 1 || !W || !codes_ok(Q, S) || !codes_ok(Qt, St) || !(Q || Qt))
    return SFL_E_ARG;
  if (E > kMaxExperts8 || R > kMaxWidth8 || C > kMaxWidth8) return SFL_E_UNSUPPORTED;
  return status(launch_quant_weights(W, dtype == SFL_BF16, E, R, C, Q, S, Qt, St, (hipStream_t)stream));
}

sfl_status_t sfl_quant_product(const uint8_t* Q, const uint8_t* S, int64_t rows, int64_t K, const uint8_t* W,
                               const uint8_t* Ws, int32_t E, int64_t N, const int32_t* offsets, sfl_dtype_t dtype,
                               void* Y, sfl_stream_t stream) {
  sfl_status_t st = check_runs(rows, E);
  if (st == SFL_E_ARG || !result_ok(dtype) || K < kBlock8 || K % kBlock8 || N < 1 || (!offsets && E != 1))
    return SFL_E_ARG;
  if (st != SFL_OK || K > kMaxWidth8 || N > INT32_MAX - (int64_t)kBlock8 * (E + 4)) return SFL_E_UNSUPPORTED;
  if (!aligned(Q, 16) || !aligned(W, 16) || !aligned(S, 4) || !aligned(Ws, 4) || !aligned(Y, result_size(dtype)))
    return SFL_E_ARG;
  if (rows == 0) return SFL_OK;
  if (!Q || !S || !W || !Ws || !Y) return SFL_E_ARG;
  const Product8 p{Q, S, W, Ws, Y, offsets, rows, N, K, 0, E};
  return status(launch_product8(p, dtype, (hipStream_t)stream));
}

sfl_status_t sfl_quant_product_weights(const uint8_t* Yt, const uint8_t* Ys, int64_t N, const uint8_t* Xt,
                                       const uint8_t* Xs, int64_t K, int64_t rows, int64_t columns,
                                       const int32_t* offsets, int32_t E, sfl_dtype_t dtype, void* dW,
                                       sfl_stream_t stream) {
  sfl_status_t st = check_runs(rows, E);
  if (st == SFL_E_ARG || !result_ok(dtype) || K < 1 || N < 1 || (!offsets && E != 1)) return SFL_E_ARG;
  if (st != SFL_OK || K > kMaxWidth8 || N > kMaxWidth8 || columns > kMaxColumns8) return SFL_E_UNSUPPORTED;
  if (columns % 512 || columns < rows || !dW ||
      !aligned(dW, result_size(dtype)) || !aligned(Yt, 16) || !aligned(Xt, 16) || !aligned(Ys, 4) ||
      !aligned(Xs, 4) || (rows > 0 && (!Yt || !Ys || !Xt || !Xs)))
    return SFL_E_ARG;
  const Product8 p{Yt, Ys, Xt, Xs, dW, offsets, rows, N, K, columns, E};
  return status(launch_product8_weights(p, dtype, (hipStream_t)stream));
}

sfl_status_t sfl_adamw_step(const sfl_adamw_t* list, int32_t n, const sfl_adamw_cfg_t* cfg, sfl_stream_t stream) {
  if (n < 0 || (n > 0 && !list) || !cfg || !cfg->step) return SFL_E_ARG;
  auto beta_ok = [](double b) { return b >= 0.0 && b < 1.0; };
  if (!beta_ok(cfg->beta1) || !beta_ok(cfg->beta2) || !(cfg->lr >= 0.0) || !((float)cfg->eps >= FLT_MIN) ||
      (cfg->sumsq && !(cfg->max_norm >= 0.0)) || (cfg->norm && !cfg->sumsq))
    return SFL_E_ARG;
  for (int32_t i = 0; i < n; ++i) {
    const sfl_adamw_t& t = list[i];
    const bool small = t.moments == SFL_MOMENTS_8BIT;
    if (t.n < 0 || t.n > ((int64_t)1 << 40) || !dtype_ok(t.param_dtype) || !dtype_ok(t.grad_dtype) ||
        (!small && t.moments != SFL_MOMENTS_F32) || !(t.weight_decay >= 0.f) || (t.half && t.param_dtype == SFL_BF16))
      return SFL_E_ARG;
    if (!small && (t.m_scale || t.v_scale)) return SFL_E_ARG;
    if (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v || (small && (!t.m_scale || !t.v_scale)))) return SFL_E_ARG;
  }
  return status(launch_adamw(list, n, *cfg, (hipStream_t)stream));
}

}  // extern "C"
