// The router: per token the k largest of its E logits and their softmax weights, and the
// gradient. With m the largest logit and e_i = exp(l_i - m) over the available experts
// (logit neither -inf nor NaN), the weights are scale e_j / Z with Z the sum over the chosen
// experts (normalise) or over all available ones. Gradient, s = weight / scale, G = scale dw:
// dl_i = p_i (up_i - sum_j s_j G_j), p over the chosen (normalise) or all available experts,
// up_i = G_j for a chosen expert and 0 for another.
#include "block.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;

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

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}

// Largest value of aligned groups of G lanes, in every lane (lanes trade as in group_sum).
template <int G> __device__ __forceinline__ uint32_t group_max(uint32_t v) {
  v = dpp_max<0xB1>(v);
  v = dpp_max<0x4E>(v);
  v = dpp_max<0x141>(v);
  if (G >= 16) v = dpp_max<0x140>(v);
  if (G == 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  if (G == 64)
    v = max(max((uint32_t)readlane_i((int)v, 0), (uint32_t)readlane_i((int)v, 16)),
            max((uint32_t)readlane_i((int)v, 32), (uint32_t)readlane_i((int)v, 48)));
  return v;
}

// G lanes per token, lane x with the PL experts x PL .. x PL + PL - 1 (so the lowest lane with the
// largest key has the lowest index). k rounds: the group's largest key, the first lane that has it,
// and that lane drops its first expert with it. Lane j keeps the j-th choice. What bounds it is the
// chain of the k rounds: about 12 instructions each for 64 experts, nothing through LDS
// (16384 tokens, 8 of 64: 45 us with 64-bit shuffles over LDS, one wave per token).
template <typename V, int G, int PL>
__global__ __launch_bounds__(kThreads) void k_route_fwd(const V* __restrict__ logits, int64_t T, int E, int k,
                                                        int normalise, float scale, int32_t* __restrict__ expert,
                                                        float* __restrict__ weight) {
  const int lane = lane_id(), x = lane % G;
  const int64_t mine_t = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const int64_t t = min(mine_t, T - 1);  // groups past the end repeat the last token and store nothing
  uint32_t key[PL], best = 0u;
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    const int e = x * PL + i;
    key[i] = e < E ? order_key(VT<V>::load(logits, t * E + e)) : 0u;
    best = max(best, key[i]);
  }
  float all = 0.f, top = 0.f;
  uint32_t my_key = 0u;
  int my_expert = -1;
  for (int j = 0; j < k; ++j) {
    const uint32_t m = group_max<G>(best);
    if (j == 0) {
      top = key_logit(m);  // not used where m is 0
      if (!normalise) {
#pragma unroll
        for (int i = 0; i < PL; ++i) all += key[i] ? expf(key_logit(key[i]) - top) : 0.f;
        all = group_sum<G>(all);
      }
    }
    const uint64_t have = ballot(best == m) >> (lane - x);  // m of this lane's group
    const int first = __builtin_ctzll(have);
    int at = -1;
    if (x == first && m) {
      best = 0u;
#pragma unroll
      for (int i = 0; i < PL; ++i) {
        if (at < 0 && key[i] == m) {
          at = i;
          key[i] = 0u;
        }
        best = max(best, key[i]);
      }
    }
    if (PL > 1) at = __shfl(at, (lane - x) + first, 64);
    if (x == j && m) {
      my_key = m;
      my_expert = PL > 1 ? first * PL + at : first;
    }
  }
  const float mine = my_expert >= 0 ? expf(key_logit(my_key) - top) : 0.f;
  const float Z = normalise ? group_sum<G>(mine) : all;
  if (x < k && mine_t < T) {
    expert[t * k + x] = my_expert;
    weight[t * k + x] = my_expert >= 0 ? scale * (mine / Z) : 0.f;
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

template <typename V, int G, int PL>
hipError_t route_fwd(const void* logits, int64_t T, int E, int k, int normalise, float scale, int32_t* expert,
                     float* weight, hipStream_t s) {
  hipLaunchKernelGGL((k_route_fwd<V, G, PL>), dim3((unsigned)cdiv(T, kThreads / G)), dim3(kThreads), 0, s,
                     (const V*)logits, T, E, k, normalise, scale, expert, weight);
  return hipGetLastError();
}

hipError_t launch_route_fwd(const void* logits, int bf16, int64_t T, int E, int k, int normalise, float scale,
                            int32_t* expert, float* weight, hipStream_t s) {
#define SFL_ROUTE(e, g, pl)                                                                                \
  if (E <= e)                                                                                              \
    return bf16 ? route_fwd<bf16_t, g, pl>(logits, T, E, k, normalise, scale, expert, weight, s)           \
                : route_fwd<float, g, pl>(logits, T, E, k, normalise, scale, expert, weight, s);
  SFL_ROUTE(8, 8, 1)
  SFL_ROUTE(16, 16, 1)
  SFL_ROUTE(32, 32, 1)
  SFL_ROUTE(64, 64, 1)
  SFL_ROUTE(128, 64, 2)
  SFL_ROUTE(256, 64, 4)
  SFL_ROUTE(512, 64, 8)
  SFL_ROUTE(kRouteMaxExperts, 64, 16)
#undef SFL_ROUTE
  return hipErrorInvalidValue;
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
