// Global norm of a list of gradients and clipping: q = sum g^2 over all tensors, norm = sqrt(q),
// g <- c g with c = max_norm / norm where norm > max_norm, else 1 (a norm that is not finite
// scales nothing). Squares are formed and added in 64 bits, so no finite gradient overflows or
// underflows the sum, and the order of the sums is fixed: blocks of a launch, then launches.
#include "block.h"
#include "common.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;
constexpr int kListMax = 112;        // tensors of one launch: the list travels as a kernel argument
constexpr int64_t kChunk = 1 << 14;  // elements of one block

struct GradList {
  const void* src[kListMax];
  void* dst[kListMax];
  int64_t n[kListMax];
  int32_t first[kListMax + 1];  // first block of each tensor
  uint8_t bf16[kListMax];
  int32_t count;
};

__device__ __forceinline__ int tensor_of(const GradList& l, int block) {
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

__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[kThreads / kWave];
  v = wave_sum(v);
  if (lane_id() == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  double s = red[0];
  for (int w = 1; w < kThreads / kWave; ++w) s += red[w];
  return s;
}

template <typename V>
__device__ __forceinline__ double chunk_sumsq(const V* p, int64_t i0, int64_t i1) {
  double s = 0;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kThreads) {
    const double g = (double)VT<V>::load(p, i);
    s = fma(g, g, s);
  }
  return s;
}

__global__ __launch_bounds__(kThreads) void k_grad_sumsq(GradList l, double* __restrict__ part) {
  const int b = blockIdx.x, i = tensor_of(l, b);
  const int64_t i0 = (int64_t)(b - l.first[i]) * kChunk, i1 = min(i0 + kChunk, l.n[i]);
  const double s = block_sum(l.bf16[i] ? chunk_sumsq((const bf16_t*)l.src[i], i0, i1)
                                       : chunk_sumsq((const float*)l.src[i], i0, i1));
  if (threadIdx.x == 0) part[b] = s;
}

__global__ __launch_bounds__(kThreads) void k_grad_sum(const double* __restrict__ part, int64_t n,
                                                       double* __restrict__ sumsq) {
  double s = 0;
  for (int64_t i = threadIdx.x; i < n; i += kThreads) s += part[i];
  s = block_sum(s);
  if (threadIdx.x == 0) *sumsq = s;
}

template <typename V>
__device__ __forceinline__ void chunk_scale(const V* p, V* q, int64_t i0, int64_t i1, float c) {
  if (p == q && c == 1.f) return;
  for (int64_t i = i0 + threadIdx.x; i < i1; i += kThreads) VT<V>::store(q, i, VT<V>::load(p, i) * c);
}

__global__ __launch_bounds__(kThreads) void k_grad_scale(GradList l, const double* __restrict__ sumsq, float max_norm,
                                                         float* __restrict__ norm) {
  const double nrm = sqrt(*sumsq);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)nrm;
  const float c = nrm > (double)max_norm && nrm < (double)INFINITY ? (float)((double)max_norm / nrm) : 1.f;
  if (l.count == 0) return;
  const int b = blockIdx.x, i = tensor_of(l, b);
  const int64_t i0 = (int64_t)(b - l.first[i]) * kChunk, i1 = min(i0 + kChunk, l.n[i]);
  if (l.bf16[i])
    chunk_scale((const bf16_t*)l.src[i], (bf16_t*)l.dst[i], i0, i1, c);
  else
    chunk_scale((const float*)l.src[i], (float*)l.dst[i], i0, i1, c);
}

int64_t chunks_of(int64_t n) { return cdiv(n, kChunk); }

// Calls f(list, blocks) for each launch's share of the tensors.
template <typename F>
void each_launch(const sfl_grad_t* list, int n, F f) {
  GradList l;
  l.count = 0;
  int64_t blocks = 0;
  for (int i = 0; i < n; ++i) {
    const int64_t c = chunks_of(list[i].n);
    if (c == 0) continue;
    if (l.count == kListMax || blocks + c > INT32_MAX) {
      f(l, blocks);
      l.count = 0;
      blocks = 0;
    }
    l.src[l.count] = list[i].src;
    l.dst[l.count] = list[i].dst ? list[i].dst : const_cast<void*>(list[i].src);
    l.n[l.count] = list[i].n;
    l.bf16[l.count] = list[i].dtype == SFL_BF16;
    l.first[l.count++] = (int32_t)blocks;
    blocks += c;
    l.first[l.count] = (int32_t)blocks;
  }
  if (blocks) f(l, blocks);
}

}  // namespace

size_t grad_workspace_bytes(const sfl_grad_t* list, int n) {
  int64_t blocks = 0;
  for (int i = 0; i < n; ++i) blocks += chunks_of(list[i].n);
  return (size_t)blocks * sizeof(double);
}

hipError_t launch_grad_sumsq(const sfl_grad_t* list, int n, double* sumsq, double* part, hipStream_t s) {
  int64_t total = 0;
  each_launch(list, n, [&](const GradList& l, int64_t blocks) {
    hipLaunchKernelGGL(k_grad_sumsq, dim3((unsigned)blocks), dim3(kThreads), 0, s, l, part + total);
    total += blocks;
  });
  hipLaunchKernelGGL(k_grad_sum, dim3(1), dim3(kThreads), 0, s, part, total, sumsq);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const sfl_grad_t* list, int n, const double* sumsq, float max_norm, float* norm,
                            hipStream_t s) {
  each_launch(list, n, [&](const GradList& l, int64_t blocks) {
    hipLaunchKernelGGL(k_grad_scale, dim3((unsigned)blocks), dim3(kThreads), 0, s, l, sumsq, max_norm, norm);
    norm = nullptr;  // the first launch writes it
  });
  if (norm) {
    GradList l;
    l.count = 0;
    hipLaunchKernelGGL(k_grad_scale, dim3(1), dim3(kThreads), 0, s, l, sumsq, max_norm, norm);
  }
  return hipGetLastError();
}

}  // namespace sfl
