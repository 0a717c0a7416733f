// The router: per token the k largest of its E logits and their softmax weights, and the
// gradient. With m the largest logit and e_i = exp(l_i - m) over the available experts
// (logit neither -inf nor NaN), the weights are scale e_j / Z with Z the sum over the chosen
// experts (normalise) or over all available ones. Gradient, s = weight / scale, G = scale dw:
// dl_i = p_i (up_i - sum_j s_j G_j), p over the chosen (normalise) or all available experts,
// up_i = G_j for a chosen expert and 0 for another.
#include "block.h"
#include "common.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;
constexpr int kPerLane = kRouteMaxExperts / kWave;

// A logit's place in the order of the reals as an unsigned number: larger logit, larger key; 0
// for an unavailable one (-inf or NaN). -0 and +0 have one key.
__device__ __forceinline__ uint32_t order_key(float l) {
  if (!(l > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(l + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_logit(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key);
}

__device__ __forceinline__ uint64_t wave_max64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t u = __shfl_xor((unsigned long long)v, o, 64);
    v = u > v ? u : v;
  }
  return v;
}

// One wave per token; lane l holds experts l, l + 64, ...
template <typename V>
__global__ __launch_bounds__(kThreads) void k_route_fwd(const V* __restrict__ logits, int64_t T, int E, int k,
                                                        int normalise, float scale, int32_t* __restrict__ expert,
                                                        float* __restrict__ weight) {
  const int lane = lane_id();
  const int64_t t = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
  if (t >= T) return;
  uint32_t key[kPerLane];
#pragma unroll
  for (int i = 0; i < kPerLane; ++i) {
    const int e = lane + kWave * i;
    key[i] = e < E ? order_key(VT<V>::load(logits, t * E + e)) : 0u;
  }
  float top = 0.f, all = 0.f, chosen = 0.f, mine = 0.f;
  int my_expert = -1;
  for (int j = 0; j < k; ++j) {
    uint64_t best = 0;  // key, then the lower index
#pragma unroll
    for (int i = 0; i < kPerLane; ++i) {
      const uint64_t c = ((uint64_t)key[i] << 32) | (uint32_t)~(lane + kWave * i);
      best = key[i] && c > best ? c : best;
    }
    best = wave_max64(best);
    if (best == 0) break;
    const int e = (int)~(uint32_t)best;
    const float l = key_logit((uint32_t)(best >> 32));
    if (j == 0) {
      top = l;
#pragma unroll
      for (int i = 0; i < kPerLane; ++i)
        if (key[i]) all += expf(key_logit(key[i]) - top);
      all = wave_sum(all);
    }
    const float v = expf(l - top);
    chosen += v;
    if (lane == j) {
      mine = v;
      my_expert = e;
    }
#pragma unroll
    for (int i = 0; i < kPerLane; ++i)
      if (lane + kWave * i == e) key[i] = 0u;
  }
  if (lane < k) {
    expert[t * k + lane] = my_expert;
    weight[t * k + lane] = my_expert < 0 ? 0.f : scale * (mine / (normalise ? chosen : all));
  }
}

template <typename V>
__global__ __launch_bounds__(kThreads) void k_route_bwd(const V* __restrict__ logits, int64_t T, int E, int k,
                                                        int normalise, float scale, const int32_t* __restrict__ expert,
                                                        const float* __restrict__ dweight, V* __restrict__ dlogits) {
  const int lane = lane_id();
  const int64_t t = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave;
  if (t >= T) return;
  int my_e = lane < k ? expert[t * k + lane] : -1;
  if (my_e >= E) my_e = -1;
  const float G = my_e >= 0 ? scale * dweight[t * k + lane] : 0.f;
  const float my_l = my_e >= 0 ? VT<V>::load(logits, t * E + my_e) : -INFINITY;
  float top = my_l;
  if (!normalise)
    for (int e = lane; e < E; e += kWave) {
      const float l = VT<V>::load(logits, t * E + e);
      if (order_key(l)) top = fmaxf(top, l);
    }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float mine = my_e >= 0 ? expf(my_l - top) : 0.f;
  float Z;
  if (normalise) {
    Z = wave_sum(mine);
  } else {
    Z = 0.f;
    for (int e = lane; e < E; e += kWave) {
      const float l = VT<V>::load(logits, t * E + e);
      if (order_key(l)) Z += expf(l - top);
    }
    Z = wave_sum(Z);
  }
  const float mean = wave_sum(my_e >= 0 ? mine / Z * G : 0.f);
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const int e = e0 + lane;
    int slot = -1;
    for (int j = 0; j < k; ++j)
      if (__shfl(my_e, j, 64) == e) slot = j;
    const float up = __shfl(G, slot < 0 ? 0 : slot, 64);
    if (e < E) {
      float v = 0.f;
      const float l = VT<V>::load(logits, t * E + e);
      if (slot >= 0)
        v = expf(l - top) / Z * (up - mean);
      else if (!normalise && order_key(l))
        v = -expf(l - top) / Z * mean;
      VT<V>::store(dlogits, t * E + e, v);
    }
  }
}

}  // namespace

hipError_t launch_route_fwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            int32_t* expert, float* weight, hipStream_t s) {
  const dim3 grid((unsigned)cdiv(T, kThreads / kWave));
  if (bf16)
    hipLaunchKernelGGL(k_route_fwd<bf16_t>, grid, dim3(kThreads), 0, s, (const bf16_t*)logits, T, E, k, normalise,
                       scale, expert, weight);
  else
    hipLaunchKernelGGL(k_route_fwd<float>, grid, dim3(kThreads), 0, s, (const float*)logits, T, E, k, normalise, scale,
                       expert, weight);
  return hipGetLastError();
}

hipError_t launch_route_bwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            const int32_t* expert, const float* dweight, void* dlogits, hipStream_t s) {
  const dim3 grid((unsigned)cdiv(T, kThreads / kWave));
  if (bf16)
    hipLaunchKernelGGL(k_route_bwd<bf16_t>, grid, dim3(kThreads), 0, s, (const bf16_t*)logits, T, E, k, normalise,
                       scale, expert, dweight, (bf16_t*)dlogits);
  else
    hipLaunchKernelGGL(k_route_bwd<float>, grid, dim3(kThreads), 0, s, (const float*)logits, T, E, k, normalise, scale,
                       expert, dweight, (float*)dlogits);
  return hipGetLastError();
}

}  // namespace sfl
