// The router with groups. A choice hangs on scores next to each other (16384 tokens of 256 experts have
// some hundred pairs closer than fp32 forms a sigmoid), so the scores that are compared are formed in 64
// bits and rounded to fp32 once: c = fp32(s + bias). Group worths are fp32 sums of one or two of them.
// Weights and gradients need no such care and are fp32. With m the largest logit, held to at most 0, the
// quotients of sigmoids are those of r = 1 / (e^m + e^(m - l)) = e^-m sigmoid(l), which does not underflow.
//   sigmoid, normalised: w_j = scale r_j / sum r, dl_j = share_j (G_j - sum share G) sigmoid(-l_j)
//   sigmoid:             w_j = scale s_j,         dl_j = s_j G_j sigmoid(-l_j),     G = scale dw
//   softmax, normalised: as a softmax over the chosen; else p over all: dl_i = p_i (up_i - sum p up)
#include "blocks8.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

__device__ __forceinline__ uint32_t order_key(float c) {
  if (!(c > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(c + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key);
}
__device__ __forceinline__ bool available(float l) { return l > -INFINITY; }
// l - top where both may be +inf
__device__ __forceinline__ float below(float l, float top) { return l == top ? 0.f : l - top; }

__device__ __forceinline__ uint64_t wave_top(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t w = __shfl_xor((unsigned long long)v, o, 64);
    v = w > v ? w : v;
  }
  return v;
}
__device__ __forceinline__ float wave_topf(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// LDS traffic of a wave with itself: what its lanes wrote before is what they read behind.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wave per token.
template <typename V>
__global__ __launch_bounds__(kThreads) void k_route_groups_fwd(sfl_route_groups_args_t a) {
  __shared__ uint32_t keys[kWaves][kRouteGroupsExperts];
  __shared__ uint32_t worth[kWaves][kRouteGroupsExperts];
  const int lane = lane_id(), wave = threadIdx.x / kWave, E = a.E, size = E / a.groups;
  const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
  if (t >= a.T) return;  // waves do not wait for each other
  const V* row = (const V*)a.logits + t * E;
  uint32_t* key = keys[wave];
  float top = -INFINITY;
  for (int e = lane; e < E; e += kWave) {
    const float l = VT<V>::load(row, e);
    if (available(l)) top = fmaxf(top, l);
  }
  top = wave_topf(top);
  double z = 0;
  if (a.score == SFL_SCORE_SOFTMAX) {
    for (int e = lane; e < E; e += kWave) {
      const float l = VT<V>::load(row, e);
      if (available(l)) z += l == top ? 1.0 : exp((double)l - (double)top);
    }
    z = wave_sum(z);
  }
  for (int e = lane; e < E; e += kWave) {
    const float l = VT<V>::load(row, e);
    double s = 0;
    if (available(l))
      s = a.score == SFL_SCORE_SOFTMAX ? (l == top ? 1.0 : exp((double)l - (double)top)) / z
                                       : 1.0 / (1.0 + exp(-(double)l));
    const float c = (float)(a.bias ? s + (double)a.bias[e] : s);
    key[e] = available(l) ? order_key(c) : 0u;
  }
  wave_sync();
  if (a.groups > 1) {
    for (int g = lane; g < a.groups; g += kWave) {
      uint32_t b0 = 0, b1 = 0;
      for (int e = g * size; e < (g + 1) * size; ++e) {
        const uint32_t k = key[e];
        b1 = max(b1, min(b0, k));
        b0 = max(b0, k);
      }
      float w = b0 ? key_value(b0) : -INFINITY;
      if (b0 && b1 && a.group_top == 2) w += key_value(b1);
      worth[wave][g] = b0 ? order_key(w) : 0u;
    }
    wave_sync();
    // rounds of the worthiest group; a group that was taken gets the key 0xffffffff
    for (int j = 0; j < a.group_k; ++j) {
      uint64_t best = 0;
      for (int g = lane; g < a.groups; g += kWave) {
        const uint32_t k = worth[wave][g];
        if (k && k != 0xffffffffu) {
          const uint64_t v = (uint64_t)k << 32 | (uint32_t)~g;
          best = v > best ? v : best;
        }
      }
      best = wave_top(best);
      if (!best) break;
      const int g = (int)~(uint32_t)best;
      if (lane == 0) worth[wave][g] = 0xffffffffu;
      wave_sync();
    }
    for (int e = lane; e < E; e += kWave)
      if (worth[wave][e / size] != 0xffffffffu) key[e] = 0u;
    wave_sync();
  }
  // k rounds; lane j keeps the j-th choice
  int mine = -1;
  for (int j = 0; j < a.k; ++j) {
    uint64_t best = 0;
    for (int e = lane; e < E; e += kWave)
      if (key[e]) {
        const uint64_t v = (uint64_t)key[e] << 32 | (uint32_t)~e;
        best = v > best ? v : best;
      }
    best = wave_top(best);
    if (!best) break;
    const int e = (int)~(uint32_t)best;
    if (lane == j) mine = e;
    if (lane == 0) key[e] = 0u;
    wave_sync();
  }
  const float l = mine >= 0 ? VT<V>::load(row, mine) : -INFINITY;
  float w = 0.f;
  if (a.score == SFL_SCORE_SIGMOID) {
    if (a.normalise) {
      const float m = fminf(wave_topf(l), 0.f);
      const float r = mine >= 0 ? 1.f / (expf(m) + expf(m - l)) : 0.f;
      const float sum = wave_sum(r);
      w = mine >= 0 ? r / sum : 0.f;
    } else {
      w = mine >= 0 ? 1.f / (1.f + expf(-l)) : 0.f;
    }
  } else if (a.normalise) {
    const float m = wave_topf(l);
    const float r = mine >= 0 ? expf(below(l, m)) : 0.f;
    const float sum = wave_sum(r);
    w = mine >= 0 ? r / sum : 0.f;
  } else {
    w = mine >= 0 ? expf(below(l, top)) / (float)z : 0.f;
  }
  if (lane < a.k) {
    a.expert[t * a.k + lane] = mine;
    a.weight[t * a.k + lane] = a.scale * w;
  }
}

template <typename V>
__global__ __launch_bounds__(kThreads) void k_route_groups_bwd(sfl_route_groups_bwd_args_t a) {
  __shared__ float ups[kWaves][kRouteGroupsExperts];
  const int lane = lane_id(), wave = threadIdx.x / kWave, E = a.E;
  const int64_t t = (int64_t)blockIdx.x * kWaves + wave;
  if (t >= a.T) return;
  const V* row = (const V*)a.logits + t * E;
  V* out = (V*)a.dlogits + t * E;
  float* up = ups[wave];
  for (int e = lane; e < E; e += kWave) up[e] = 0.f;
  wave_sync();
  int e = lane < a.k ? a.expert[t * a.k + lane] : -1;
  float l = e >= 0 && e < E ? VT<V>::load(row, e) : -INFINITY;
  const bool there = available(l);
  const float G = there ? a.scale * a.dweight[t * a.k + lane] : 0.f;
  if (a.score == SFL_SCORE_SOFTMAX && !a.normalise) {
    float top = -INFINITY;
    for (int i = lane; i < E; i += kWave) {
      const float x = VT<V>::load(row, i);
      if (available(x)) top = fmaxf(top, x);
    }
    top = wave_topf(top);
    float z = 0.f;
    for (int i = lane; i < E; i += kWave) {
      const float x = VT<V>::load(row, i);
      if (available(x)) z += expf(below(x, top));
    }
    z = wave_sum(z);
    const float mean = wave_sum(there ? expf(below(l, top)) / z * G : 0.f);
    if (there) up[e] = G;
    wave_sync();
    for (int i = lane; i < E; i += kWave) {
      const float x = VT<V>::load(row, i);
      VT<V>::store(out, i, available(x) ? expf(below(x, top)) / z * (up[i] - mean) : 0.f);
    }
    return;
  }
  float d = 0.f;
  if (a.normalise) {
    float m = wave_topf(l), r;
    if (a.score == SFL_SCORE_SIGMOID) {
      m = fminf(m, 0.f);
      r = there ? 1.f / (expf(m) + expf(m - l)) : 0.f;
    } else {
      r = there ? expf(below(l, m)) : 0.f;
    }
    const float sum = wave_sum(r), share = there ? r / sum : 0.f;
    d = share * (G - wave_sum(share * G));
  } else {
    d = there ? G / (1.f + expf(-l)) : 0.f;
  }
  if (a.score == SFL_SCORE_SIGMOID) d *= 1.f / (1.f + expf(l));
  if (there) up[e] = d;
  wave_sync();
  for (int i = lane; i < E; i += kWave) VT<V>::store(out, i, up[i]);
}

template <typename F> hipError_t over(int64_t T, F f) {
  const int64_t most = max_blocks(kThreads) * kWaves;
  for (int64_t t0 = 0; t0 < T; t0 += most) {
    const int64_t n = std::min(T - t0, most);
    f(t0, n, dim3((unsigned)cdiv(n, kWaves)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_route_groups_fwd(const sfl_route_groups_args_t& args, hipStream_t s) {
  return over(args.T, [&](int64_t t0, int64_t n, dim3 grid) {
    sfl_route_groups_args_t a = args;
    const bool bf16 = a.dtype == SFL_BF16;
    a.T = n;
    a.logits = (const char*)a.logits + t0 * a.E * (bf16 ? 2 : 4);
    a.expert += t0 * a.k;
    a.weight += t0 * a.k;
    if (bf16)
      hipLaunchKernelGGL(k_route_groups_fwd<bf16_t>, grid, dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL(k_route_groups_fwd<float>, grid, dim3(kThreads), 0, s, a);
  });
}

hipError_t launch_route_groups_bwd(const sfl_route_groups_bwd_args_t& args, hipStream_t s) {
  return over(args.T, [&](int64_t t0, int64_t n, dim3 grid) {
    sfl_route_groups_bwd_args_t a = args;
    const bool bf16 = a.dtype == SFL_BF16;
    const int64_t bytes = t0 * a.E * (bf16 ? 2 : 4);
    a.T = n;
    a.logits = (const char*)a.logits + bytes;
    a.dlogits = (char*)a.dlogits + bytes;
    a.expert += t0 * a.k;
    a.dweight += t0 * a.k;
    if (bf16)
      hipLaunchKernelGGL(k_route_groups_bwd<bf16_t>, grid, dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL(k_route_groups_bwd<float>, grid, dim3(kThreads), 0, s, a);
  });
}

}  // namespace sfl
