// The boundary between two blocks of a model: RMS norm of the block's output, its gates, the
// scaled residual sum, and the RMS norm that the next block reads. Per row t,
//   r_y = 1 / sqrt(mean(Y^2) + eps),   X' = res_scale X + gate_t gate_c w_post r_y Y,
//   r_x = 1 / sqrt(mean(X'^2) + eps),  N = w_pre r_x X'.
// Backward, with x^ = r_x X', y^ = r_y Y, u = w_post gate_c:
//   D = dX' + r_x (w_pre dN - x^ mean(w_pre dN x^)),   dX = res_scale D,
//   dY = gate_t r_y (u D - y^ mean(u D y^)),           dgate_t = sum_c u D y^,
//   A = sum_t dN x^ = dw_pre,  S = sum_t gate_t D y^:  dw_post = gate_c S, dgate_c = w_post S.
// All arithmetic in fp32; X' is rounded once when stored, and N is formed from the sum before
// that rounding.
#include "block.h"
#include "common.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;

// Sum over the block's 256 threads, in every thread.
__device__ __forceinline__ float block_sum(float v, float* red) {
  v = wave_sum(v);
  __syncthreads();
  if (lane_id() == 0) red[threadIdx.x / kWave] = v;
  __syncthreads();
  return red[0] + red[1] + red[2] + red[3];
}

template <typename V>
__global__ __launch_bounds__(kThreads) void k_norm_fwd(NormParams p) {
  __shared__ float red[4];
  const V* Y = (const V*)p.Y;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const int64_t base = t * p.d;
    float ry = 1.f;
    if (p.post) {
      float s = 0.f;
      for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
        const float y = VT<V>::load(Y, base + c);
        s = fmaf(y, y, s);
      }
      ry = 1.f / sqrtf(block_sum(s, red) / (float)p.d + p.eps);
    }
    const float gt = (p.gate_t ? p.gate_t[t] : 1.f) * ry;
    auto sum_at = [&](int64_t c) {
      float x = p.res_scale * VT<V>::load((const V*)p.X, base + c);
      if (!Y) return x;
      const float u = (p.w_post ? p.w_post[c] : 1.f) * (p.gate_c ? p.gate_c[c] : 1.f);
      return fmaf(gt * u, VT<V>::load(Y, base + c), x);
    };
    float rx = 0.f;
    if (p.pre) {
      float s = 0.f;
      for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
        const float x = sum_at(c);
        s = fmaf(x, x, s);
      }
      rx = 1.f / sqrtf(block_sum(s, red) / (float)p.d + p.eps);
    }
    for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
      const float x = sum_at(c);
      if (p.N) VT<V>::store((V*)p.N, base + c, x * rx * (p.w_pre ? p.w_pre[c] : 1.f));
      if (p.X_out) VT<V>::store((V*)p.X_out, base + c, x);
    }
  }
}

// One block walks rows b, b + grid, ...; a thread owns columns threadIdx.x + 256 i, whose
// parameter sums it keeps in LDS (A, then S) and leaves in part[b] at the end.
template <typename V>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(NormBwdParams p) {
  extern __shared__ float acc[];
  __shared__ float red[4];
  float* A = acc;
  float* S = acc + p.d;
  for (int64_t c = threadIdx.x; c < 2 * p.d; c += kThreads) acc[c] = 0.f;
  __syncthreads();
  const V* Y = (const V*)p.Y;
  const float inv_d = 1.f / (float)p.d;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    const int64_t base = t * p.d;
    float rx = 0.f, mx = 0.f, ry = 1.f;
    float s = 0.f, q = 0.f, sy = 0.f;
    for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
      if (p.pre) {
        const float x = VT<V>::load((const V*)p.X_out, base + c);
        s = fmaf(x, x, s);
        if (p.dN) q = fmaf(VT<V>::load((const V*)p.dN, base + c) * (p.w_pre ? p.w_pre[c] : 1.f), x, q);
      }
      if (p.post) {
        const float y = VT<V>::load(Y, base + c);
        sy = fmaf(y, y, sy);
      }
    }
    if (p.pre) {
      rx = 1.f / sqrtf(block_sum(s, red) * inv_d + p.eps);
      mx = block_sum(q, red) * rx * inv_d;
    }
    if (p.post) ry = 1.f / sqrtf(block_sum(sy, red) * inv_d + p.eps);
    auto grad_at = [&](int64_t c) {
      float D = p.dX_out ? VT<V>::load((const V*)p.dX_out, base + c) : 0.f;
      if (p.pre && p.dN) {
        const float xh = VT<V>::load((const V*)p.X_out, base + c) * rx;
        const float g = VT<V>::load((const V*)p.dN, base + c) * (p.w_pre ? p.w_pre[c] : 1.f);
        D += rx * (g - xh * mx);
      }
      return D;
    };
    auto u_at = [&](int64_t c) { return (p.w_post ? p.w_post[c] : 1.f) * (p.gate_c ? p.gate_c[c] : 1.f); };
    const float gt = p.gate_t ? p.gate_t[t] : 1.f;
    float Q = 0.f;
    if (Y) {
      for (int64_t c = threadIdx.x; c < p.d; c += kThreads)
        Q = fmaf(u_at(c) * grad_at(c), VT<V>::load(Y, base + c) * ry, Q);
      Q = block_sum(Q, red);
      if (p.dgate_t && threadIdx.x == 0) p.dgate_t[t] = Q;
    }
    const float my = p.post ? Q * inv_d : 0.f;
    for (int64_t c = threadIdx.x; c < p.d; c += kThreads) {
      const float D = grad_at(c);
      if (p.pre && p.dN) A[c] = fmaf(VT<V>::load((const V*)p.dN, base + c), VT<V>::load((const V*)p.X_out, base + c) * rx, A[c]);
      if (Y) {
        const float yh = VT<V>::load(Y, base + c) * ry;
        S[c] = fmaf(gt * D, yh, S[c]);
        if (p.dY) VT<V>::store((V*)p.dY, base + c, gt * ry * (u_at(c) * D - yh * my));
      }
      if (p.dX) VT<V>::store((V*)p.dX, base + c, p.res_scale * D);
    }
  }
  __syncthreads();  // a column's sums move to another thread
  for (int64_t c = threadIdx.x; c < 2 * p.d; c += kThreads) p.part[blockIdx.x * 2 * p.d + c] = acc[c];
}

// Parameter gradients from the blocks' sums, added in block order.
__global__ __launch_bounds__(kThreads) void k_norm_param_sums(NormBwdParams p, int blocks) {
  const int64_t c = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  if (c >= p.d) return;
  float A = 0.f, S = 0.f;
  for (int b = 0; b < blocks; ++b) {
    A += p.part[(int64_t)b * 2 * p.d + c];
    S += p.part[(int64_t)b * 2 * p.d + p.d + c];
  }
  if (p.dw_pre) p.dw_pre[c] = A;
  if (p.dw_post) p.dw_post[c] = S * (p.gate_c ? p.gate_c[c] : 1.f);
  if (p.dgate_c) p.dgate_c[c] = S * (p.w_post ? p.w_post[c] : 1.f);
}

int norm_blocks(int64_t T) { return (int)std::min<int64_t>(T, 512); }

}  // namespace

size_t norm_workspace_bytes(int64_t T, int64_t d) { return (size_t)norm_blocks(T) * 2 * (size_t)d * sizeof(float); }

hipError_t launch_norm_fwd(const NormParams& p, int bf16, hipStream_t s) {
  const unsigned grid = (unsigned)std::min<int64_t>(p.T, 65536);
  if (bf16)
    hipLaunchKernelGGL(k_norm_fwd<bf16_t>, dim3(grid), dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL(k_norm_fwd<float>, dim3(grid), dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

hipError_t launch_norm_bwd(const NormBwdParams& p, int bf16, hipStream_t s) {
  const int blocks = norm_blocks(p.T);
  const size_t lds = (size_t)2 * p.d * sizeof(float);
  if (blocks > 0) {
    if (lds > (64 << 10)) {
      const void* kern = bf16 ? (const void*)k_norm_bwd<bf16_t> : (const void*)k_norm_bwd<float>;
      const hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
      if (e != hipSuccess) return e;
    }
    if (bf16)
      hipLaunchKernelGGL(k_norm_bwd<bf16_t>, dim3(blocks), dim3(kThreads), lds, s, p);
    else
      hipLaunchKernelGGL(k_norm_bwd<float>, dim3(blocks), dim3(kThreads), lds, s, p);
  }
  if (p.dw_pre || p.dw_post || p.dgate_c)
    hipLaunchKernelGGL(k_norm_param_sums, dim3((unsigned)cdiv(p.d, kThreads)), dim3(kThreads), 0, s, p, blocks);
  return hipGetLastError();
}

}  // namespace sfl
