// The router with groups. A choice hangs on scores next to each other (16384 tokens of 256 experts have
// some hundred pairs closer than fp32 forms a sigmoid), so the scores that are compared are formed in 64
// bits and rounded to fp32 once: c = fp32(s + bias). Group worths are fp32 sums of one or two of them.
// Weights and gradients need no such care and are fp32. With m the largest logit, held to at most 0, the
// quotients of sigmoids are those of r = 1 / (e^m + e^(m - l)) = e^-m sigmoid(l), which does not underflow.
// 16384 tokens of 256 fp32 logits in 8 groups: 20.7 us, of it the 64-bit scores 5 and the rounds of the choice 6 to 7; 64.5
// with a wave per token and the keys in LDS (k_route_groups_fwd, for groups that are not whole lanes). Backward 9.2 us,
// 1.8 TB/s written: a wave per token passes its row through LDS and stores four bytes (of bf16, two) a lane.
//   sigmoid, normalised: w_j = scale r_j / sum r, dl_j = share_j (G_j - sum share G) sigmoid(-l_j)
//   sigmoid:             w_j = scale s_j,         dl_j = s_j G_j sigmoid(-l_j),     G = scale dw
//   softmax, normalised: as a softmax over the chosen; else p over all: dl_i = p_i (up_i - sum p up)
#include "blocks8.h"
#include "order.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;

// The key of a group's worth from those of its one or two best experts (0 for none). Two of the lowest numbers add up
// to -inf: still above a group without any expert.
__device__ __forceinline__ uint32_t worth_key(uint32_t b0, uint32_t b1, int group_top) {
  if (!b0) return 0u;
  const float w = b1 && group_top == 2 ? key_value(b0) + key_value(b1) : key_value(b0);
  return max(order_key(w), 1u);
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

// The two largest of two lanes' two largest each.
__device__ __forceinline__ void two_most(uint32_t& b0, uint32_t& b1, uint32_t o0, uint32_t o1) {
  b1 = max(max(b1, o1), min(b0, o0));
  b0 = max(b0, o0);
}
template <int CTRL> __device__ __forceinline__ void two_most(uint32_t& b0, uint32_t& b1) {
  two_most(b0, b1, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b0, CTRL, 0xf, 0xf, false),
           (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b1, CTRL, 0xf, 0xf, false));
}

// LDS traffic of a wave with itself: what its lanes wrote before is what they read behind.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// e^x in 64 bits for x from -700 to 700 (beyond: as there; what is scored by it is 0 or 1 in fp32 long before), to
// 2 in 10^16: reduced by multiples of ln 2 in two parts (those that fdlibm publishes: the first has 21 zero bits at its
// end, so that n times it is exact), then the Taylor polynomial of degree 12, whose rest is below 2 in 10^16 for
// |r| <= ln 2 / 2.
__device__ __forceinline__ double exp64(double x) {
  x = fmin(fmax(x, -700.0), 700.0);
  const double n = rint(x * 1.4426950408889634074);
  const double r = fma(n, -1.90821492927058770002e-10, fma(n, -6.93147180369123816490e-01, x));
  double p = 1.0 / 479001600;
  constexpr double c[12] = {1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720,
                            1.0 / 120,      1.0 / 24,      1.0 / 6,      1.0 / 2,     1.0,        1.0};
#pragma unroll
  for (int i = 0; i < 12; ++i) p = fma(p, r, c[i]);
  return ldexp(p, (int)n);
}
// 1 / d for normal d > 0: the hardware's estimate and two steps of Newton's method.
__device__ __forceinline__ double inverse64(double d) {
  double y = __builtin_amdgcn_rcp(d);
  y = fma(y, fma(-d, y, 1.0), y);
  return fma(y, fma(-d, y, 1.0), y);
}

template <int G> __device__ __forceinline__ double group_sum64(double v) {
#pragma unroll
  for (int o = 1; o < G; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// G lanes a token, PL experts a lane; a group of experts is 2^shift whole lanes (or there is one group).
// Rounds as in the router without groups: the largest key of the token's lanes; the first
// lane that has it drops its first expert with it, so equal ones go by ascending index.
template <typename V, int G, int PL>
__global__ __launch_bounds__(kThreads) void k_route_groups_lanes(sfl_route_groups_args_t a, int shift) {
  const int lane = lane_id(), x = lane % G, E = a.E, e0 = x * PL;
  const int64_t mine = (int64_t)blockIdx.x * (kThreads / G) + threadIdx.x / G;
  const int64_t t = min(mine, a.T - 1);  // groups past the end repeat the last token and store nothing
  const uint64_t before = ((1ull << x) - 1ull) << (lane - x);  // the token's lanes before this one
  const bool softmax = a.score == SFL_SCORE_SOFTMAX;
  const V* row = (const V*)a.logits + t * E;
  float l[PL];
  if (e0 + PL <= E) {
    V v[PL];
    __builtin_memcpy(v, row + e0, sizeof(v));
#pragma unroll
    for (int i = 0; i < PL; ++i) l[i] = VT<V>::load(v, i);
  } else {
#pragma unroll
    for (int i = 0; i < PL; ++i) l[i] = e0 + i < E ? VT<V>::load(row, e0 + i) : -INFINITY;
  }
  float bias[PL] = {};
  if (a.bias) {
    if (e0 + PL <= E) {
      __builtin_memcpy(bias, a.bias + e0, sizeof(bias));
    } else {
#pragma unroll
      for (int i = 0; i < PL; ++i) bias[i] = e0 + i < E ? a.bias[e0 + i] : 0.f;
    }
  }
  float top = -INFINITY;
  double z = 0;
  if (softmax) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) m = max(m, order_key(l[i]));
    m = group_max<G>(m);
    top = m ? key_value(m) : -INFINITY;
  }
  double s[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    if (softmax) {
      s[i] = !available(l[i]) ? 0.0 : l[i] == top ? 1.0 : exp64((double)l[i] - (double)top);
      z += s[i];
    } else {
      s[i] = inverse64(1.0 + exp64(-(double)l[i]));
    }
  }
  if (softmax) {
    z = group_sum64<G>(z);
    const double by = z > 0 ? inverse64(z) : 0.0;
#pragma unroll
    for (int i = 0; i < PL; ++i) s[i] *= by;
  }
  uint32_t key[PL], best = 0u;
#pragma unroll
  for (int i = 0; i < PL; ++i) key[i] = available(l[i]) ? order_key((float)(s[i] + (double)bias[i])) : 0u;
  if (a.groups > 1) {
    uint32_t b0 = 0, b1 = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      b1 = max(b1, min(b0, key[i]));
      b0 = max(b0, key[i]);
    }
    if (shift > 0) two_most<0xB1>(b0, b1);
    if (shift > 1) two_most<0x4E>(b0, b1);
    if (shift > 2) two_most<0x141>(b0, b1);
    if (shift > 3) two_most<0x140>(b0, b1);
    for (int o = 16; o < 1 << shift; o <<= 1) two_most(b0, b1, (uint32_t)__shfl_xor((int)b0, o, 64), (uint32_t)__shfl_xor((int)b1, o, 64));
    const uint32_t worth = x < a.groups << shift ? worth_key(b0, b1, a.group_top) : 0u;
    // a group is taken where fewer than group_k are worthier, or worth the same before it
    const int group = x >> shift;
    int ahead = 0;
    for (int g = 0; g < a.groups; ++g) {
      const int from = (lane - x) + (g << shift);
      const uint32_t other = (uint32_t)(G == 64 ? readlane_i((int)worth, g << shift) : __shfl((int)worth, from, 64));
      ahead += other > worth || (other == worth && g < group);
    }
    const bool taken = ahead < a.group_k;
#pragma unroll
    for (int i = 0; i < PL; ++i) key[i] = taken ? key[i] : 0u;
  }
  int round[PL];
#pragma unroll
  for (int i = 0; i < PL; ++i) {
    best = max(best, key[i]);
    round[i] = -1;
  }
  int found = 0;
  for (int j = 0; j < a.k; ++j) {
    const uint32_t m = group_max<G>(best);
    const uint64_t have = ballot(best == m);
    found += m != 0u;
    if (m && best == m && !(have & before)) {
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
  // quotients in 64 bits from the scores as they are, while their sum is far from where e^x was held
  float w[PL], sum = 0.f;
#pragma unroll
  for (int i = 0; i < PL; ++i) sum += round[i] >= 0 ? (float)s[i] : 0.f;
  sum = group_sum<G>(sum);
  const double by = !a.normalise ? 1.0 : sum > 0x1p-60f ? (double)(1.f / sum) : 0.0;
#pragma unroll
  for (int i = 0; i < PL; ++i) w[i] = (float)(s[i] * by);
  if (a.normalise && !(sum > 0x1p-60f)) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < PL; ++i) m = max(m, round[i] >= 0 ? order_key(l[i]) : 0u);
    m = group_max<G>(m);
    const float high = m ? key_value(m) : -INFINITY, held = fminf(high, 0.f), shifted = softmax ? 0.f : expf(held);
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < PL; ++i) {
      w[i] = round[i] < 0 ? 0.f : softmax ? expf(below(l[i], high)) : 1.f / (shifted + expf(held - l[i]));
      sum += w[i];
    }
    sum = group_sum<G>(sum);
#pragma unroll
    for (int i = 0; i < PL; ++i) w[i] /= sum;
  }
  if (mine >= a.T) return;
#pragma unroll
  for (int i = 0; i < PL; ++i)
    if (round[i] >= 0) {
      a.expert[t * a.k + round[i]] = e0 + i;
      a.weight[t * a.k + round[i]] = a.scale * w[i];
    }
  for (int j = found + x; j < a.k; j += G) {
    a.expert[t * a.k + j] = -1;
    a.weight[t * a.k + j] = 0.f;
  }
}

// Groups that are not whole lanes (a size that is no power of two times the experts of a lane): a wave per
// token, keys in LDS.
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
      worth[wave][g] = worth_key(b0, b1, a.group_top);
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

// The logarithm of the lanes that a group of experts takes where a lane has PL; -1 where it does not take whole
// lanes, as many as a power of two.
int lanes_of(const sfl_route_groups_args_t& a, int pl) {
  if (a.groups == 1) return 0;
  const int size = a.E / a.groups, lanes = size / pl;
  return size % pl || (lanes & (lanes - 1)) ? -1 : __builtin_ctz(lanes);
}

template <typename V, int G, int PL> hipError_t forward_lanes(const sfl_route_groups_args_t& args, int shift, hipStream_t s) {
  return over_tokens<kThreads, kThreads / G>(args.T, [&](int64_t t0, int64_t n, dim3 grid) {
    sfl_route_groups_args_t a = args;
    a.T = n;
    a.logits = (const V*)a.logits + t0 * a.E;
    a.expert += t0 * a.k;
    a.weight += t0 * a.k;
    hipLaunchKernelGGL((k_route_groups_lanes<V, G, PL>), grid, dim3(kThreads), 0, s, a, shift);
  });
}

template <typename V> hipError_t forward(const sfl_route_groups_args_t& args, hipStream_t s) {
#define SFL_ROUTE(g, pl) \
  if (args.E <= g * pl)  \
    if (const int shift = lanes_of(args, pl); shift >= 0) return forward_lanes<V, g, pl>(args, shift, s);
  SFL_ROUTE(2, 4) SFL_ROUTE(4, 4) SFL_ROUTE(8, 4) SFL_ROUTE(16, 4) SFL_ROUTE(32, 4) SFL_ROUTE(64, 4)
  SFL_ROUTE(64, 8) SFL_ROUTE(64, 16)
#undef SFL_ROUTE
  return over_tokens<kThreads, kWaves>(args.T, [&](int64_t t0, int64_t n, dim3 grid) {
    sfl_route_groups_args_t a = args;
    a.T = n;
    a.logits = (const V*)a.logits + t0 * a.E;
    a.expert += t0 * a.k;
    a.weight += t0 * a.k;
    hipLaunchKernelGGL(k_route_groups_fwd<V>, grid, dim3(kThreads), 0, s, a);
  });
}

}  // namespace

hipError_t launch_route_groups_fwd(const sfl_route_groups_args_t& a, hipStream_t s) {
  return a.dtype == SFL_BF16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}

hipError_t launch_route_groups_bwd(const sfl_route_groups_bwd_args_t& args, hipStream_t s) {
  return over_tokens<kThreads, kWaves>(args.T, [&](int64_t t0, int64_t n, dim3 grid) {
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
