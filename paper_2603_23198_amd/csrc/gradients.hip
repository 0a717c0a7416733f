// Global norm of a list of gradients and clipping: q = sum g^2 over all tensors, norm = sqrt(q),
// g <- c g with c = max_norm / norm where norm > max_norm, else 1 (a norm that is not finite
// scales nothing). Squares are formed and added in 64 bits, so no finite gradient overflows or
// underflows the sum (the conversions and fp64 FMAs stay far below the rate the values arrive at),
// and the order of the sums is fixed: a thread's, a workgroup's, then the workgroups'.
//
// Bound by memory: the list is read twice and written once. The second pass walks the list from
// its end, where the first one stopped: the last 256 MiB that were read are still in the infinity
// cache, and the scaled values are stored non-temporally beside them.
#include "block.h"
#include "clip.h"
#include "rows.h"

#include <algorithm>
#include <utility>

namespace sfl {

namespace {

constexpr int kThreads = 256;
// Ranges of one launch. The list travels as a kernel argument, of 3.3 KB, and a short one (most
// lists, once adjacent tensors are joined) of 0.3 KB: norm and clipping of two times 262144 fp32
// elements 13.9 -> 13.0 us, medians of twelve processes each in turn (13.4 to 14.2 and 12.8 to 13.6;
// in a captured graph 8.39 -> 8.25).
constexpr int kListMax = 112, kListShort = 8;
constexpr int kTile = 2048;      // smallest share of a workgroup

// Elements of a workgroup's share: all of its loads go out together. Long shares are slower (their
// last round leaves CUs idle; both passes over 2^27 fp32 elements in two tensors: 304 us with shares
// of 65536, 303 with 8192, 290 with 8192 and 4096; over 192 tensors 339 and 303), shorter ones too
// (2048: 308 us). Short lists take smaller shares so that more CUs work.
constexpr int kSumShare = 4 * kTile, kScaleShare = 2 * kTile;
constexpr int64_t kFewShares = 1024;
int64_t share_of(int64_t total, int64_t most) {
  int64_t share = kTile;
  while (share < most && total / share > kFewShares) share *= 2;
  return share;
}

template <int MAX> struct GradList {
  const void* src[MAX];
  void* dst[MAX];
  int64_t n[MAX];
  int32_t first[MAX + 1];  // first workgroup of each range
  uint8_t bf16[MAX];
  int32_t count;
  int32_t share;
};

template <int MAX> __device__ __forceinline__ int range_of(const GradList<MAX>& l, int block) {
  int lo = 0, hi = l.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (l.first[mid] <= block)
      lo = mid;
    else
      hi = mid - 1;
  }
  return lo;
}

// Sum over N threads in the first of them, in a fixed order.
template <int N> __device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[N / kWave];
  v = wave_sum(v);
  if (lane_id() == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  double s = red[0];
  for (int w = 1; w < N / kWave; ++w) s += red[w];
  return s;
}

// 16 bytes per thread and step, so that every access of a wave is one run of 1 KiB (two times 16
// bytes per thread side by side: 17 % more bytes written, by the counter, for fp32).
template <typename V> struct Step {
  static constexpr int kElems = 16 / sizeof(V), kStep = kThreads * kElems;
  V e[kElems];
  __device__ __forceinline__ void load(const V* p, int c, int n) {
    if (c + kElems <= n) {
      __builtin_memcpy(e, p + c, 16);
    } else {
#pragma unroll
      for (int i = 0; i < kElems; ++i) e[i] = c + i < n ? p[c + i] : V(0);
    }
  }
  __device__ __forceinline__ void store(V* p, int c, int n) const {
    if (c + kElems <= n) {
      u32x4_t w;
      __builtin_memcpy(&w, e, 16);
      store16(p + c, w);
    } else {
#pragma unroll
      for (int i = 0; i < kElems; ++i)
        if (c + i < n) p[c + i] = e[i];
    }
  }
};

template <typename V> __device__ __forceinline__ double share_sumsq(const V* p, int n) {
  using S = Step<V>;
  constexpr int kSteps = kSumShare / S::kStep;
  double s[2] = {0, 0};
  const int c = threadIdx.x * S::kElems;
  S v[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) v[i].load(p, c + i * S::kStep, n);
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
#pragma unroll
    for (int e = 0; e < S::kElems; ++e) {
      const double g = (double)VT<V>::load(v[i].e, e);
      s[e & 1] = fma(g, g, s[e & 1]);
    }
  return s[0] + s[1];
}

template <int MAX>
__global__ __launch_bounds__(kThreads) void k_grad_sumsq(GradList<MAX> l, double* __restrict__ part) {
  const int b = blockIdx.x, i = range_of(l, b);
  const int64_t at = (int64_t)(b - l.first[i]) * l.share;
  const int n = (int)min((int64_t)l.share, l.n[i] - at);
  const double s = block_sum<kThreads>(l.bf16[i] ? share_sumsq((const bf16_t*)l.src[i] + at, n)
                                                 : share_sumsq((const float*)l.src[i] + at, n));
  if (threadIdx.x == 0) part[b] = s;
}

constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void k_grad_sum(const double* __restrict__ part, int64_t n,
                                                          double* __restrict__ sumsq) {
  double s = 0;
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += 4 * kSumThreads) {
    double q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = part[min(i0 + i * kSumThreads, n - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) s += i0 + i * kSumThreads < n ? q[i] : 0.0;
  }
  s = block_sum<kSumThreads>(s);
  if (threadIdx.x == 0) *sumsq = s;
}

template <typename V> __device__ __forceinline__ void share_scale(const V* p, V* q, int n, const Scale& scale) {
  if (p == q && scale.by == 1.f && scale.exp == 0) return;
  using S = Step<V>;
  constexpr int kSteps = kScaleShare / S::kStep;
  const int c = threadIdx.x * S::kElems;
  S v[kSteps];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) v[i].load(p, c + i * S::kStep, n);
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
#pragma unroll
    for (int e = 0; e < S::kElems; ++e) VT<V>::store(v[i].e, e, scale(VT<V>::load(v[i].e, e)));
    v[i].store(q, c + i * S::kStep, n);
  }
}

template <int MAX>
__global__ __launch_bounds__(kThreads) void k_grad_scale(GradList<MAX> l, const double* __restrict__ sumsq,
                                                         float max_norm, float* __restrict__ norm) {
  const double nrm = sqrt(*sumsq);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)nrm;
  const Scale by(clip_coefficient(nrm, (double)max_norm));
  if (l.count == 0) return;
  const int b = gridDim.x - 1 - blockIdx.x, i = range_of(l, b);
  const int64_t at = (int64_t)(b - l.first[i]) * l.share;
  const int n = (int)min((int64_t)l.share, l.n[i] - at);
  if (l.bf16[i])
    share_scale((const bf16_t*)l.src[i] + at, (bf16_t*)l.dst[i] + at, n, by);
  else
    share_scale((const float*)l.src[i] + at, (float*)l.dst[i] + at, n, by);
}

int64_t elements(const sfl_grad_t* list, int n) {
  int64_t total = 0;
  for (int i = 0; i < n; ++i) total += list[i].n;
  return total;
}

// How far a pass over the list has come: so many tensors from its start (or its end) and so many
// elements of the next one.
struct Walk {
  int tensor = 0;
  int64_t elements = 0;
};

// Fills l with the next ranges of the list, from its start on or from its end back, for as many
// workgroups as one launch takes, and moves w past them; returns the launch's workgroups. Tensors
// whose elements lie end to end at the source and at the target (views of one bucket mostly do) go
// as one range, with fewer launches and no ragged shares.
int64_t next_launch(const sfl_grad_t* list, int n, bool back, int64_t share, Walk* w, GradList<kListMax>* l) {
  constexpr int64_t most = max_blocks(kThreads);
  int64_t closed = 0;  // workgroups of the ranges before the last one
  l->count = 0;
  l->share = (int32_t)share;
  for (; w->tensor < n; ++w->tensor, w->elements = 0) {
    const sfl_grad_t& g = list[back ? n - 1 - w->tensor : w->tensor];
    const bool bf16 = g.dtype == SFL_BF16;
    const int64_t size = bf16 ? 2 : 4, rest = g.n - w->elements, len = std::min(rest, most * share);
    if (len == 0) continue;
    const int64_t at = (back ? rest - len : w->elements) * size;
    const char* src = (const char*)g.src + at;
    char* dst = (char*)(g.dst ? g.dst : const_cast<void*>(g.src)) + at;
    int m = l->count - 1;  // the range that the elements may join
    bool joins = false;
    if (m >= 0 && l->bf16[m] == bf16) {
      const int64_t by = (back ? len : -l->n[m]) * size;
      joins = src + by == (const char*)l->src[m] && dst + by == (char*)l->dst[m];
    }
    const int64_t behind = joins || m < 0 ? closed : closed + cdiv(l->n[m], share);
    const int64_t total = joins ? l->n[m] + len : len;
    if (l->count + !joins > kListMax || behind + cdiv(total, share) > most) break;
    closed = behind;
    if (!joins) m = l->count++;
    if (!joins || back) {
      l->src[m] = src;
      l->dst[m] = dst;
    }
    l->n[m] = total;
    l->bf16[m] = bf16;
    if (len < rest) {  // the launch is full
      w->elements += len;
      break;
    }
  }
  if (back)
    for (int i = 0, j = l->count - 1; i < j; ++i, --j) {
      std::swap(l->src[i], l->src[j]);
      std::swap(l->dst[i], l->dst[j]);
      std::swap(l->n[i], l->n[j]);
      std::swap(l->bf16[i], l->bf16[j]);
    }
  l->first[0] = 0;
  for (int m = 0; m < l->count; ++m) l->first[m + 1] = l->first[m] + (int32_t)cdiv(l->n[m], share);
  return l->first[l->count];
}

// Calls f with the list, as a short argument where it is short.
template <typename F> void with_list(const GradList<kListMax>& l, F f) {
  if (l.count > kListShort) return f(l);
  GradList<kListShort> s;
  for (int i = 0; i < l.count; ++i) {
    s.src[i] = l.src[i];
    s.dst[i] = l.dst[i];
    s.n[i] = l.n[i];
    s.bf16[i] = l.bf16[i];
  }
  for (int i = 0; i <= l.count; ++i) s.first[i] = l.first[i];
  s.count = l.count;
  s.share = l.share;
  f(s);
}

}  // namespace

// A sum per workgroup; ranges of several tensors have at most as many as their tensors alone. The
// shares double as lists grow and the workgroups fall, so this counts those of the largest shares and
// of any list whose shares are smaller (up to 1024, and one more per tensor): no list needs more than
// one that holds it.
size_t grad_workspace_bytes(const sfl_grad_t* list, int n) {
  int64_t smallest = 0, largest = 0, tensors = 0;
  for (int i = 0; i < n; ++i) {
    smallest += cdiv(list[i].n, kTile);
    largest += cdiv(list[i].n, kSumShare);
    tensors += list[i].n > 0;
  }
  return (size_t)std::max(largest, std::min(smallest, kFewShares + tensors)) * sizeof(double);
}

hipError_t launch_grad_sumsq(const sfl_grad_t* list, int n, double* sumsq, double* part, hipStream_t s) {
  const int64_t share = share_of(elements(list, n), kSumShare);
  int64_t done = 0;
  GradList<kListMax> l;
  for (Walk w; w.tensor < n;) {
    const int64_t blocks = next_launch(list, n, false, share, &w, &l);
    if (blocks)
      with_list(l, [&](const auto& a) {
        hipLaunchKernelGGL(k_grad_sumsq, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, part + done);
      });
    done += blocks;
  }
  hipLaunchKernelGGL(k_grad_sum, dim3(1), dim3(kSumThreads), 0, s, part, done, sumsq);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const sfl_grad_t* list, int n, const double* sumsq, float max_norm, float* norm,
                            hipStream_t s) {
  const int64_t share = share_of(elements(list, n), kScaleShare);
  GradList<kListMax> l;
  auto launch = [&](int64_t blocks) {
    with_list(l, [&](const auto& a) {
      hipLaunchKernelGGL(k_grad_scale, dim3((unsigned)blocks), dim3(kThreads), 0, s, a, sumsq, max_norm, norm);
    });
    norm = nullptr;  // the first launch writes it
  };
  for (Walk w; w.tensor < n;) {
    const int64_t blocks = next_launch(list, n, true, share, &w, &l);
    if (blocks) launch(blocks);
  }
  if (norm) {  // nothing to scale
    l.count = 0;
    l.first[0] = 0;
    l.share = (int32_t)share;
    launch(1);
  }
  return hipGetLastError();
}

}  // namespace sfl
