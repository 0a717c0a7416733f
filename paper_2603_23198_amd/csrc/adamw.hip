// One step of AdamW over a list of tensors: every element of parameter, gradient and moments is read
// once and written once, and the clipping coefficient comes from the gradients' squared norm on the
// device, so that clipping costs no pass of its own. Bound by memory: 30 bytes an element with fp32
// gradients and moments and the bf16 copy (2^27 elements 735 to 755 us, 5.3 to 5.5 TB/s), 16 with bf16 gradients and
// moments in 8 bits (144 M elements 474 to 487 us, 4.7 to 4.85 TB/s; some 95 instructions an element are not far behind).
//
// Moments in 8 bits: e4m3 codes with a power of two for each 128 elements (of v the root, which has
// half the range). Three mantissa bits are coarser than what a slow average moves in a step (v by 1 part
// in 1000, a last place is 6 to 12 in 100), so a nearest rounding would hold it where it is for good: the
// rounding is drawn instead, to either neighbour with the probability that keeps the value on average. A
// root above zero is held as above zero: the denominator of the next step rests on it.
#include "blocks8.h"
#include "clip.h"
#include "order.h"
#include "rows.h"

#include <algorithm>
#include <cfloat>
#include <cmath>

namespace sfl {

namespace {

// A thread has four neighbouring elements at a time, so that every access of a wave is one run of
// memory (of fp32, 1 KiB), and 32 lanes have the 128 elements of a scale.
constexpr int kThreads = 256, kUnit = 4, kSteps = 2, kStep = kThreads * kUnit, kShare = kSteps * kStep;
constexpr int kListMax = 38, kListShort = 6;  // tensors of one launch: kernel arguments of 3.9 and 0.7 KB

struct Hyper {
  float lr, beta1, rest1, beta2, rest2, eps;
  double log_beta1, log_beta2;  // of the bias corrections
  double max_norm;
  const int64_t* step;
  const float* lr_scale;
  const double* sumsq;
  float* norm;
  uint32_t seed;
};

template <int MAX> struct List {
  sfl_adamw_t t[MAX];        // from the launch's first element of the tensor on
  uint64_t place[MAX];       // of that element in the whole list
  int32_t first[MAX + 1];    // first workgroup of each tensor
  int32_t count;
};
static_assert(sizeof(List<kListMax>) + sizeof(Hyper) <= 4096, "kernel arguments");

__device__ __forceinline__ uint32_t mix(uint32_t h) {  // MurmurHash3's 32-bit finaliser
  h ^= h >> 16;
  h *= 0x85ebca6bu;
  h ^= h >> 13;
  h *= 0xc2b2ae35u;
  return h ^ (h >> 16);
}

// Four elements from i on, of n; ALL: all are there.
template <bool ALL, typename V> __device__ __forceinline__ void load_unit4(const V* p, int64_t i, int64_t n, float (&x)[kUnit]) {
  if (ALL || i + kUnit <= n) {
    V v[kUnit];
    __builtin_memcpy(v, p + i, sizeof(v));
#pragma unroll
    for (int j = 0; j < kUnit; ++j) x[j] = VT<V>::load(v, j);
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j) x[j] = i + j < n ? VT<V>::load(p, i + j) : 0.f;
  }
}
__device__ __forceinline__ void pack(const float (&x)[kUnit], float (&v)[kUnit]) {
#pragma unroll
  for (int j = 0; j < kUnit; ++j) v[j] = x[j];
}
__device__ __forceinline__ void pack(const float (&x)[kUnit], bf16_t (&v)[kUnit]) {
  const u32x2_t w{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  __builtin_memcpy(v, &w, 8);
}
template <bool ALL, typename V> __device__ __forceinline__ void store_unit4(V* p, int64_t i, int64_t n, const float (&x)[kUnit]) {
  V v[kUnit];
  pack(x, v);
  if (ALL || i + kUnit <= n) {
    __builtin_memcpy(p + i, v, sizeof(v));
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if (i + j < n) p[i + j] = v[j];
  }
}

template <bool ALL> __device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t i, int64_t n) {
  uint32_t w = 0;
  if (ALL || i + kUnit <= n) {
    __builtin_memcpy(&w, p + i, 4);
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if (i + j < n) w |= (uint32_t)p[i + j] << (8 * j);
  }
  return w;
}
template <bool ALL> __device__ __forceinline__ void store_codes(uint8_t* p, int64_t i, int64_t n, uint32_t w) {
  if (ALL || i + kUnit <= n) {
    __builtin_memcpy(p + i, &w, 4);
  } else {
#pragma unroll
    for (int j = 0; j < kUnit; ++j)
      if (i + j < n) p[i + j] = (uint8_t)(w >> (8 * j));
  }
}
__device__ __forceinline__ void decode(uint32_t w, float by, float (&x)[kUnit]) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * by;
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * by;
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * by;
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * by;
}

// A scaled magnitude (at most 448) to e4m3's numbers, by 16 bits of noise; exact in e4m3. From 2^-6 on
// the noise is added below the last of the three mantissa bits, under it (e4m3's subnormal numbers) in
// steps of 2^-9.
__device__ __forceinline__ float drawn(float a, uint32_t noise, bool least) {
  float q;
  if (a < 0x1p-6f) {
    q = floorf(a * 512.f + (float)noise * 0x1p-16f) * 0x1p-9f;
    if (least && a > 0.f) q = fmaxf(q, 0x1p-9f);
  } else {
    q = __uint_as_float((__float_as_uint(a) + (noise << 4)) & ~0xfffffu);
  }
  return q;
}
// Four elements to codes; the scale byte is that of the 32 lanes' 128 elements.
__device__ __forceinline__ uint32_t encode(const float (&x)[kUnit], const uint32_t (&noise)[kUnit], bool least, int* byte) {
  float most = 0.f;  // a NaN has no part in it
#pragma unroll
  for (int j = 0; j < kUnit; ++j) most = fmaxf(most, fabsf(x[j]));
  uint32_t top = group_max<32>(__float_as_uint(most));
  if (top == 0x7f800000u) {  // an infinity: once more without those
    top = 0;
#pragma unroll
    for (int j = 0; j < kUnit; ++j) top = max(top, magnitude8(x[j]));
    top = group_max<32>(top);
  }
  *byte = scale_byte8(top);
  const float by = inverse8(*byte);
  float q[kUnit];
#pragma unroll
  for (int j = 0; j < kUnit; ++j) {
    const float a = fabsf(x[j]);
    q[j] = a < INFINITY ? copysignf(drawn(a * by, noise[j], least), x[j]) : NAN;
  }
  return codes8(q[0], q[1], q[2], q[3]);
}

struct Now {  // of this step
  float lr, inv1, inv2;  // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
  uint32_t key;
};

// n / d for d from the smallest normal number on, to the nearest fp32 number but where the reals' quotient lies within
// 2^-45 of itself of the middle of two: the hardware's estimate (one last place off), corrected by what it leaves of
// n. (8-bit moments, 144 M elements: 474 us, with a division as the compiler writes it 492. The estimate alone costs
// 468.) The bounds keep a quotient by infinity zero and one that fp32 does not hold infinite.
__device__ __forceinline__ float quotient(float n, float d) {
  const float r = __builtin_amdgcn_rcpf(d), q = n * r;
  const float held = __builtin_amdgcn_fmed3f(q, -FLT_MAX, FLT_MAX);
  return fmaf(fmaf(-fminf(d, FLT_MAX), held, n), r, q);
}

// The new moments and parameter of one element, and the root of the second moment, which is rounded to nearest
// (moments in 8 bits hang on it). Every operation rounds to nearest, as in any 32-bit form of the formulas.
__device__ __forceinline__ float advance(const Hyper& h, const Now& now, const Scale& clip, float decay, float grad,
                                         float& p, float& m, float& v) {
#pragma clang fp contract(off)
  const float g = clip(grad);
  m = h.beta1 * m + h.rest1 * g;
  v = h.beta2 * v + h.rest2 * (g * g);
  const float root = sqrtf(v);
  p = p - now.lr * (quotient(m * now.inv1, root * now.inv2 + h.eps) + decay * p);
  return root;
}

template <bool ALL, typename P, typename G, bool SMALL>
__device__ __forceinline__ void turn(const sfl_adamw_t& t, uint64_t place, int64_t at, const Hyper& h, const Now& now,
                                     const Scale& clip) {
  float p[kSteps][kUnit], g[kSteps][kUnit], m[kSteps][kUnit], v[kSteps][kUnit];
  uint32_t mq[kSteps], vq[kSteps];
  int mb[kSteps], vb[kSteps];
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t i = at + s * kStep + threadIdx.x * kUnit;
    load_unit4<ALL>((const P*)t.param, i, t.n, p[s]);
    load_unit4<ALL>((const G*)t.grad, i, t.n, g[s]);
    if (SMALL) {
      mq[s] = load_codes<ALL>((const uint8_t*)t.m, i, t.n);
      vq[s] = load_codes<ALL>((const uint8_t*)t.v, i, t.n);
      // 255, which no step writes, would make an infinity: zeros are zeros by any byte
      mb[s] = min(ALL || i < t.n ? (int)t.m_scale[i / kBlock8] : 127, 254);
      vb[s] = min(ALL || i < t.n ? (int)t.v_scale[i / kBlock8] : 127, 254);
    } else {
      load_unit4<ALL>((const float*)t.m, i, t.n, m[s]);
      load_unit4<ALL>((const float*)t.v, i, t.n, v[s]);
    }
  }
#pragma unroll
  for (int s = 0; s < kSteps; ++s) {
    const int64_t i = at + s * kStep + threadIdx.x * kUnit;
    if (SMALL) {
      decode(mq[s], scale8(mb[s]), m[s]);
      decode(vq[s], scale8(vb[s]), v[s]);
#pragma unroll
      for (int j = 0; j < kUnit; ++j) v[s][j] *= v[s][j];
    }
#pragma unroll
    for (int j = 0; j < kUnit; ++j) {
      const float root = advance(h, now, clip, t.weight_decay, g[s][j], p[s][j], m[s][j], v[s][j]);
      if (SMALL) v[s][j] = root;
    }
    store_unit4<ALL>((P*)t.param, i, t.n, p[s]);
    if (t.half) store_unit4<ALL>((bf16_t*)t.half, i, t.n, p[s]);
    if (SMALL) {
      // the four elements' places share their upper half: they begin at a multiple of four
      uint32_t low[kUnit], high[kUnit];
      const uint64_t at_list = place + (uint64_t)i;
      const uint32_t key = mix(now.key + (uint32_t)(at_list >> 32));
#pragma unroll
      for (int j = 0; j < kUnit; ++j) {
        const uint32_t bits = mix(key ^ ((uint32_t)at_list + j));
        low[j] = bits & 0xffffu;
        high[j] = bits >> 16;
      }
      // lanes past the end have zeros: no part in a block's largest
      int byte_m, byte_v;
      const uint32_t cm = encode(m[s], low, false, &byte_m), cv = encode(v[s], high, true, &byte_v);
      store_codes<ALL>((uint8_t*)t.m, i, t.n, cm);
      store_codes<ALL>((uint8_t*)t.v, i, t.n, cv);
      if (threadIdx.x % 32 == 0 && (ALL || i < t.n)) {
        t.m_scale[i / kBlock8] = (uint8_t)byte_m;
        t.v_scale[i / kBlock8] = (uint8_t)byte_v;
      }
    } else {
      store_unit4<ALL>((float*)t.m, i, t.n, m[s]);
      store_unit4<ALL>((float*)t.v, i, t.n, v[s]);
    }
  }
}

template <typename P, typename G, bool SMALL>
__device__ __forceinline__ void share(const sfl_adamw_t& t, uint64_t place, int64_t at, const Hyper& h, const Now& now,
                                      const Scale& clip) {
  if (at + kShare <= t.n)
    turn<true, P, G, SMALL>(t, place, at, h, now, clip);
  else
    turn<false, P, G, SMALL>(t, place, at, h, now, clip);
}

template <int MAX> __global__ __launch_bounds__(kThreads) void k_adamw(List<MAX> l, Hyper h) {
  __shared__ Now shared;
  const double nrm = h.sumsq ? sqrt(*h.sumsq) : 0.0;
  if (h.norm && blockIdx.x == 0 && threadIdx.x == 0) *h.norm = (float)nrm;
  if (l.count == 0 || !norm_is_finite(nrm)) return;
  if (threadIdx.x == 0) {
    const int64_t step = *h.step;
    const double t = (double)(step > 1 ? step : 1);
    shared.lr = h.lr_scale ? h.lr * *h.lr_scale : h.lr;
    shared.inv1 = (float)(-1.0 / expm1(t * h.log_beta1));
    shared.inv2 = (float)sqrt(-1.0 / expm1(t * h.log_beta2));
    shared.key = mix((uint32_t)(step > 1 ? step : 1) + mix(h.seed));
  }
  __syncthreads();
  const Now now = shared;
  const Scale clip(h.sumsq ? clip_coefficient(nrm, h.max_norm) : 1.0);
  int lo = 0, hi = l.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (l.first[mid] <= (int)blockIdx.x)
      lo = mid;
    else
      hi = mid - 1;
  }
  const sfl_adamw_t t = l.t[lo];  // in registers: the stores below may not change it
  const int64_t at = (int64_t)((int)blockIdx.x - l.first[lo]) * kShare;
  const uint64_t place = l.place[lo];
  const int kind = (t.param_dtype == SFL_BF16 ? 4 : 0) | (t.grad_dtype == SFL_BF16 ? 2 : 0) | (t.moments ? 1 : 0);
  switch (kind) {
    case 0: return share<float, float, false>(t, place, at, h, now, clip);
    case 1: return share<float, float, true>(t, place, at, h, now, clip);
    case 2: return share<float, bf16_t, false>(t, place, at, h, now, clip);
    case 3: return share<float, bf16_t, true>(t, place, at, h, now, clip);
    case 4: return share<bf16_t, float, false>(t, place, at, h, now, clip);
    case 5: return share<bf16_t, float, true>(t, place, at, h, now, clip);
    case 6: return share<bf16_t, bf16_t, false>(t, place, at, h, now, clip);
    default: return share<bf16_t, bf16_t, true>(t, place, at, h, now, clip);
  }
}

// The tensor from element `at` on.
sfl_adamw_t from(sfl_adamw_t t, int64_t at) {
  t.param = (char*)t.param + at * (t.param_dtype == SFL_BF16 ? 2 : 4);
  t.grad = (const char*)t.grad + at * (t.grad_dtype == SFL_BF16 ? 2 : 4);
  if (t.half) t.half = (char*)t.half + at * 2;
  const int64_t size = t.moments == SFL_MOMENTS_8BIT ? 1 : 4;
  t.m = (char*)t.m + at * size;
  t.v = (char*)t.v + at * size;
  if (t.moments == SFL_MOMENTS_8BIT) {
    t.m_scale += at / kBlock8;
    t.v_scale += at / kBlock8;
  }
  t.n -= at;
  return t;
}

void launch(const List<kListMax>& l, int blocks, const Hyper& h, hipStream_t s) {
  if (l.count > kListShort) {
    hipLaunchKernelGGL(k_adamw<kListMax>, dim3((unsigned)blocks), dim3(kThreads), 0, s, l, h);
    return;
  }
  List<kListShort> few;
  std::copy(l.t, l.t + l.count, few.t);
  std::copy(l.place, l.place + l.count, few.place);
  std::copy(l.first, l.first + l.count + 1, few.first);
  few.count = l.count;
  hipLaunchKernelGGL(k_adamw<kListShort>, dim3((unsigned)blocks), dim3(kThreads), 0, s, few, h);
}

}  // namespace

hipError_t launch_adamw(const sfl_adamw_t* list, int n, const sfl_adamw_cfg_t& cfg, hipStream_t s) {
  Hyper h{};
  h.lr = (float)cfg.lr;
  h.beta1 = (float)cfg.beta1;
  h.rest1 = (float)(1.0 - cfg.beta1);
  h.beta2 = (float)cfg.beta2;
  h.rest2 = (float)(1.0 - cfg.beta2);
  h.eps = (float)cfg.eps;
  h.log_beta1 = std::log(cfg.beta1);  // -inf for 0: its power is 0
  h.log_beta2 = std::log(cfg.beta2);
  h.max_norm = cfg.max_norm;
  h.step = cfg.step;
  h.lr_scale = cfg.lr_scale;
  h.sumsq = cfg.sumsq;
  h.norm = cfg.norm;
  h.seed = cfg.seed;
  // no launch has more work items than 2^32; a longer tensor goes on in the next one
  constexpr int64_t most = max_blocks(kThreads);
  List<kListMax> l;
  l.count = 0;
  l.first[0] = 0;
  bool any = false;
  auto flush = [&]() {
    launch(l, std::max(l.first[l.count], 1), h, s);
    h.norm = nullptr;  // the first launch writes it
    l.count = 0;
    any = true;
    return hipGetLastError();
  };
  uint64_t place = 0;
  for (int i = 0; i < n; ++i) {
    for (int64_t at = 0; at < list[i].n;) {
      const int64_t blocks = std::min(cdiv(list[i].n - at, (int64_t)kShare), most);
      if (l.count == kListMax || l.first[l.count] + blocks > most) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
        continue;
      }
      l.t[l.count] = from(list[i], at);
      l.t[l.count].n = std::min(list[i].n - at, blocks * kShare);
      l.place[l.count] = place + (uint64_t)at;
      l.first[l.count + 1] = l.first[l.count] + (int32_t)blocks;
      ++l.count;
      at += blocks * kShare;
    }
    place += (uint64_t)up(list[i].n, kBlock8);
  }
  return l.count || (h.norm && !any) ? flush() : hipSuccess;
}

}  // namespace sfl
