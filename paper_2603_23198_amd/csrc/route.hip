// The router: per token the k largest of its E logits and their softmax weights, and the
// gradient. With m the largest logit and e_i = exp(l_i - m) over the available experts
// (logit neither -inf nor NaN), the weights are scale e_j / Z with Z the sum over the chosen
// experts (normalise) or over all available ones. Gradient, s = weight / scale, G = scale dw:
// dl_i = p_i (up_i - sum_j s_j G_j), p over the chosen (normalise) or all available experts,
// up_i = G_j for a chosen expert and 0 for another.
//
// The data is small (16384 x 64 logits are 4 MB), and the k rounds cost more than it: in a captured
// graph 65536 tokens of 64 fp32 logits take 6.6 us for k = 1 and 0.8 for every further choice, 16384 take
// 3.1 and 0.27 (at k = 8, 5.0 in all, 440 vector instructions a wave, which alone take 3 us). A token
// therefore takes a group of G lanes with PL experts each, PL = 4 for up to 256 experts: a round's
// exchange between lanes (two instructions per halving) then serves several tokens of a wave, and
// what a lane does for its own PL experts costs less than more lanes would. 16384 tokens, 8 of 64,
// kernel alone: 45 us with 64-bit keys traded over LDS, 9.4 us with a lane per expert and the wave's
// largest key in a scalar register.
#include "block.h"
#include "order.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;

// A lane's experts e0 .. e0 + PL - 1 of a row of E, by one load where all are there; what is past
// the end is not available.
template <typename V, int PL>
__device__ __forceinline__ void load_logits(const V* row, int e0, int E, float (&l)[PL]) {
  V v[PL];
  if (e0 + PL <= E) {
    __builtin_memcpy(v, row + e0, sizeof(v));
#pragma unroll
    for (int i = 0; i < PL; ++i) l[i] = VT<V>::load(v, i);
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i) l[i] = e0 + i < E ? VT<V>::load(row, e0 + i) : -INFINITY;
  }
}

// k rounds: the group's largest key; the first lane that has it drops its first expert with it
// (experts ascend over lanes and within one, so this is the lowest index) and notes the round.
template <typename V, int G, int PL>
__global__ __launch_bounds__(kThreads) void k_route_fwd(const V* __restrict__ logits, int64_t T, int E, int k,
                                                        int normalise, float scale, int32_t* __restrict__ expert,
                                                        float* __restrict__ weight) {
  const int lane = lane_id(), x = lane % G;
  const int64_t mine = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const int64_t t = min(mine, T - 1);  // groups past the end repeat the last token and store nothing
  const uint64_t below = ((1ull << x) - 1ull) << (lane - x);  // the group's lanes before this one
  float l[PL];
  load_logits<V, PL>(logits + t * E, x * PL, E, l);
  uint32_t key[PL], best = 0u;
  int round[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    key[i] = order_key(l[i]);
    best = max(best, key[i]);
    round[i] = -1;
  }
  uint32_t top_key = 0u;
  int found = 0;
  for (int j = 0; j < k; ++j) {
    const uint32_t m = group_max<G>(best);
    if (j == 0) top_key = m;
    const uint64_t have = ballot(best == m);
    found += m != 0u;
    if (m && best == m && !(have & below)) {
      bool dropped = false;
      best = 0u;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        if (!dropped && key[i] == m) {
          dropped = true;
          round[i] = j;
          key[i] = 0u;
        }
        best = max(best, key[i]);
      }
    }
  }
  const float top = key_value(top_key);
  float ex[PL], Z = 0.f;
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const bool counts = normalise ? round[i] >= 0 : order_key(l[i]) != 0u;
    ex[i] = counts ? expf(l[i] - top) : 0.f;
    Z += ex[i];
  }
  Z = group_sum<G>(Z);
  if (mine >= T) return;
#pragma unroll
  for (int i = 0; i < PL; ++i)
    if (round[i] >= 0) {
      expert[t * k + round[i]] = x * PL + i;
      weight[t * k + round[i]] = scale * (ex[i] / Z);
    }
  for (int j = found + x; j < k; j += G) {
    expert[t * k + j] = -1;
    weight[t * k + j] = 0.f;
  }
}

// The same layout. The token's choices go through LDS, slot[e] = j + 1, so that a lane finds the
// slots of its own experts by one read (looking each of its experts up in the k choices: 16.5 us for
// 16384 tokens, 8 of 256, against 8.7).
template <typename V, int G, int PL>
__global__ __launch_bounds__(kThreads) void k_route_bwd(const V* __restrict__ logits, int64_t T, int E, int k,
                                                        int normalise, float scale, const int32_t* __restrict__ expert,
                                                        const float* __restrict__ dweight, V* __restrict__ dlogits) {
  __shared__ int slot[kThreads * PL];
  const int x = lane_id() % G;
  const int64_t mine = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const int64_t t = min(mine, T - 1);
  const int e0 = x * PL;
  float l[PL], up[PL];
  bool chosen[PL];
  int* group = slot + threadIdx.x / G * (G * PL);
#pragma unroll
  for (int i = 0; i < PL; ++i) group[e0 + i] = 0;
  load_logits<V, PL>(logits + t * E, e0, E, l);
  __syncthreads();
  for (int j = x; j < k; j += G) {
    const int e = expert[t * k + j];
    if (e >= 0 && e < E) group[e] = j + 1;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const int j = group[e0 + i] - 1;
    chosen[i] = j >= 0;
    up[i] = j >= 0 ? scale * dweight[t * k + j] : 0.f;
  }
  uint32_t top_key = 0u;
  bool counts[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const uint32_t key = order_key(l[i]);
    counts[i] = key != 0u && (chosen[i] || !normalise);
    top_key = max(top_key, counts[i] ? key : 0u);
  }
  const float top = key_value(group_max<G>(top_key));
  float p[PL], Z = 0.f, mean = 0.f;
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    p[i] = counts[i] ? expf(l[i] - top) : 0.f;
    Z += p[i];
  }
  const float inv = 1.f / group_sum<G>(Z);  // infinite only where no expert counts
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    p[i] = counts[i] ? p[i] * inv : 0.f;
    mean += chosen[i] && counts[i] ? p[i] * up[i] : 0.f;
  }
  mean = group_sum<G>(mean);
  if (mine >= T) return;
  V o[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) o[i] = VT<V>::cvt(counts[i] ? p[i] * (up[i] - mean) : 0.f);
  V* row = dlogits + t * E;
  if (e0 + PL <= E) {
    __builtin_memcpy(row + e0, o, sizeof(o));
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i)
      if (e0 + i < E) row[e0 + i] = o[i];
  }
}

// Calls f with the lanes per token and the experts per lane.
template <typename F> hipError_t with_layout(int E, F f) {
  using std::integral_constant;
#define SFL_ROUTE(g, pl) \
  if (E <= g * pl) return f(integral_constant<int, g>{}, integral_constant<int, pl>{});
  SFL_ROUTE(2, 4) SFL_ROUTE(4, 4) SFL_ROUTE(8, 4) SFL_ROUTE(16, 4) SFL_ROUTE(32, 4) SFL_ROUTE(64, 4)
  SFL_ROUTE(64, 8) SFL_ROUTE(64, 16)
#undef SFL_ROUTE
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_route_fwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            int32_t* expert, float* weight, hipStream_t s) {
  return with_layout(E, [&](auto g, auto pl) {
    constexpr int G = decltype(g)::value, PL = decltype(pl)::value;
    return over_tokens<kThreads, kThreads / G>(T, [&](int64_t t0, int64_t n, dim3 grid) {
      if (bf16)
        hipLaunchKernelGGL((k_route_fwd<bf16_t, G, PL>), grid, dim3(kThreads), 0, s, (const bf16_t*)logits + t0 * E, n,
                           E, k, normalise, scale, expert + t0 * k, weight + t0 * k);
      else
        hipLaunchKernelGGL((k_route_fwd<float, G, PL>), grid, dim3(kThreads), 0, s, (const float*)logits + t0 * E, n, E,
                           k, normalise, scale, expert + t0 * k, weight + t0 * k);
    });
  });
}

hipError_t launch_route_bwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            const int32_t* expert, const float* dweight, void* dlogits, hipStream_t s) {
  return with_layout(E, [&](auto g, auto pl) {
    constexpr int G = decltype(g)::value, PL = decltype(pl)::value;
    return over_tokens<kThreads, kThreads / G>(T, [&](int64_t t0, int64_t n, dim3 grid) {
      if (bf16)
        hipLaunchKernelGGL((k_route_bwd<bf16_t, G, PL>), grid, dim3(kThreads), 0, s, (const bf16_t*)logits + t0 * E, n,
                           E, k, normalise, scale, expert + t0 * k, dweight + t0 * k, (bf16_t*)dlogits + t0 * E);
      else
        hipLaunchKernelGGL((k_route_bwd<float, G, PL>), grid, dim3(kThreads), 0, s, (const float*)logits + t0 * E, n, E,
                           k, normalise, scale, expert + t0 * k, dweight + t0 * k, (float*)dlogits + t0 * E);
    });
  });
}

}  // namespace sfl
