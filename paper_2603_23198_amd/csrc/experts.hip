// Tokens to their experts and back. Slot (t, j) is the j-th choice of token t; expert order is a
// stable counting sort of the slots by expert, so an expert's rows are in token order:
//   pos(s) = #{slots of lower experts} + #{earlier slots of the same expert}, -1 for a slot of
//   no expert; Xs[pos] = X[t]; Y[t] = sum_j w Ys[pos]; dYs[pos] = w dY[t]; dw = <dY[t], Ys[pos]>.
// The gradient of the way there, dX[t] = sum_j dXs[pos], is the way back with weights of one.
// Every pass walks the tokens, so a token's row is read or written once however many experts it
// has. Sums run over j in order, in fp32: results do not depend on any other token.
#include "block.h"
#include "common.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;
constexpr int kOrderThreads = 1024;

// One workgroup sorts all slots, 1024 at a time in slot order. LDS: next[E], the next free row
// of each expert, and tile[waves][E], the current tile's slots of each wave and expert.
__global__ __launch_bounds__(kOrderThreads) void k_expert_order(const int32_t* __restrict__ expert, int64_t n, int E,
                                                                int32_t* __restrict__ pos,
                                                                int32_t* __restrict__ offsets) {
  extern __shared__ int32_t lds[];
  int32_t* next = lds;
  int32_t* tile = lds + E;
  const int waves = kOrderThreads / kWave, wave = threadIdx.x / kWave;
  for (int e = threadIdx.x; e < E; e += kOrderThreads) next[e] = 0;
  __syncthreads();
  for (int64_t i = threadIdx.x; i < n; i += kOrderThreads) {
    const int e = expert[i];
    if (e >= 0 && e < E) atomicAdd(&next[e], 1);
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int sum = 0;
    for (int e = 0; e < E; ++e) {
      const int c = next[e];
      next[e] = sum;
      offsets[e] = sum;
      sum += c;
    }
    offsets[E] = sum;
  }
  for (int64_t i0 = 0; i0 < n; i0 += kOrderThreads) {
    for (int e = threadIdx.x; e < waves * E; e += kOrderThreads) tile[e] = 0;
    __syncthreads();
    const int64_t i = i0 + threadIdx.x;
    int e = i < n ? expert[i] : -1;
    if (e >= E) e = -1;
    // lanes of this wave with the same expert
    uint64_t same = __ballot(e >= 0);
    for (int b = 0; (1 << b) < E; ++b) {
      const uint64_t m = __ballot((e >> b) & 1);
      same &= ((e >> b) & 1) ? m : ~m;
    }
    const int before = mbcnt(same);
    if (e >= 0 && before == 0) tile[wave * E + e] = __popcll(same);
    __syncthreads();
    if (e >= 0) {
      int row = next[e] + before;
      for (int w = 0; w < wave; ++w) row += tile[w * E + e];
      pos[i] = row;
    } else if (i < n) {
      pos[i] = -1;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < E; x += kOrderThreads)
      for (int w = 0; w < waves; ++w) next[x] += tile[w * E + x];
    __syncthreads();
  }
}

template <typename V>
__global__ __launch_bounds__(kThreads) void k_expert_rows(const V* __restrict__ X, int64_t T, int64_t d, int k,
                                                          const int32_t* __restrict__ pos, int64_t rows,
                                                          V* __restrict__ Xs) {
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x)
    for (int64_t c = threadIdx.x; c < d; c += kThreads) {
      const V v = X[t * d + c];
      for (int j = 0; j < k; ++j) {
        const int p = pos[t * k + j];
        if (p >= 0 && p < rows) Xs[p * d + c] = v;
      }
    }
}

template <typename V>
__global__ __launch_bounds__(kThreads) void k_expert_combine(const V* __restrict__ Ys, int64_t T, int64_t d, int k,
                                                             const int32_t* __restrict__ pos, int64_t rows,
                                                             const float* __restrict__ weight, V* __restrict__ Y) {
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x)
    for (int64_t c = threadIdx.x; c < d; c += kThreads) {
      float s = 0.f;
      for (int j = 0; j < k; ++j) {
        const int p = pos[t * k + j];
        if (p >= 0 && p < rows) s = fmaf(weight ? weight[t * k + j] : 1.f, VT<V>::load(Ys, p * d + c), s);
      }
      VT<V>::store(Y, t * d + c, s);
    }
}

// One wave per slot.
template <typename V>
__global__ __launch_bounds__(kThreads) void k_expert_combine_bwd(const V* __restrict__ dY, const V* __restrict__ Ys,
                                                                 int64_t T, int64_t d, int k,
                                                                 const int32_t* __restrict__ pos, int64_t rows,
                                                                 const float* __restrict__ weight, V* __restrict__ dYs,
                                                                 float* __restrict__ dweight) {
  const int lane = lane_id();
  for (int64_t s = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave; s < T * k;
       s += (int64_t)gridDim.x * (kThreads / kWave)) {
    const int p = pos[s];
    float dot = 0.f;
    if (p >= 0 && p < rows) {
      const float w = weight ? weight[s] : 1.f;
      for (int64_t c = lane; c < d; c += kWave) {
        const float g = VT<V>::load(dY, s / k * d + c);
        if (dweight) dot = fmaf(g, VT<V>::load(Ys, p * d + c), dot);
        if (dYs) VT<V>::store(dYs, p * d + c, w * g);
      }
    }
    dot = wave_sum(dot);
    if (dweight && lane == 0) dweight[s] = dot;
  }
}

unsigned row_grid(int64_t T) { return (unsigned)std::min<int64_t>(T, 1 << 20); }

}  // namespace

size_t expert_workspace_bytes(int64_t, int, int) { return 0; }

hipError_t launch_expert_order(const int32_t* expert, int64_t T, int k, int E, int32_t* pos, int32_t* offsets,
                               void*, hipStream_t s) {
  const size_t lds = (size_t)E * (1 + kOrderThreads / kWave) * sizeof(int32_t);
  if (lds > (64 << 10)) {
    const hipError_t e = hipFuncSetAttribute((const void*)k_expert_order, hipFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(k_expert_order, dim3(1), dim3(kOrderThreads), lds, s, expert, T * k, E, pos, offsets);
  return hipGetLastError();
}

hipError_t launch_expert_rows(const void* X, int bf16, int64_t T, int64_t d, int k, const int32_t* pos, int64_t rows,
                              void* Xs, hipStream_t s) {
  if (T == 0 || rows == 0) return hipSuccess;
  if (bf16)
    hipLaunchKernelGGL(k_expert_rows<bf16_t>, dim3(row_grid(T)), dim3(kThreads), 0, s, (const bf16_t*)X, T, d, k, pos,
                       rows, (bf16_t*)Xs);
  else
    hipLaunchKernelGGL(k_expert_rows<float>, dim3(row_grid(T)), dim3(kThreads), 0, s, (const float*)X, T, d, k, pos,
                       rows, (float*)Xs);
  return hipGetLastError();
}

hipError_t launch_expert_combine(const void* Ys, int bf16, int64_t T, int64_t d, int k, const int32_t* pos,
                                 int64_t rows, const float* weight, void* Y, hipStream_t s) {
  if (T == 0) return hipSuccess;
  if (bf16)
    hipLaunchKernelGGL(k_expert_combine<bf16_t>, dim3(row_grid(T)), dim3(kThreads), 0, s, (const bf16_t*)Ys, T, d, k,
                       pos, rows, weight, (bf16_t*)Y);
  else
    hipLaunchKernelGGL(k_expert_combine<float>, dim3(row_grid(T)), dim3(kThreads), 0, s, (const float*)Ys, T, d, k,
                       pos, rows, weight, (float*)Y);
  return hipGetLastError();
}

hipError_t launch_expert_combine_bwd(const void* dY, const void* Ys, int bf16, int64_t T, int64_t d, int k,
                                     const int32_t* pos, int64_t rows, const float* weight, void* dYs, float* dweight,
                                     hipStream_t s) {
  if (T == 0) return hipSuccess;
  const unsigned grid = row_grid(cdiv(T * k, kThreads / kWave));
  if (bf16)
    hipLaunchKernelGGL(k_expert_combine_bwd<bf16_t>, dim3(grid), dim3(kThreads), 0, s, (const bf16_t*)dY,
                       (const bf16_t*)Ys, T, d, k, pos, rows, weight, (bf16_t*)dYs, dweight);
  else
    hipLaunchKernelGGL(k_expert_combine_bwd<float>, dim3(grid), dim3(kThreads), 0, s, (const float*)dY,
                       (const float*)Ys, T, d, k, pos, rows, weight, (float*)dYs, dweight);
  return hipGetLastError();
}

}  // namespace sfl
