// The boundary between two blocks of a model: RMS norm of the block's output, its gates, the
// scaled residual sum, and the RMS norm that the next block reads. Per row t,
//   r_y = 1 / sqrt(mean(Y^2) + eps),   X' = res_scale X + gate_t gate_c w_post r_y Y,
//   r_x = 1 / sqrt(mean(X'^2) + eps),  N = w_pre r_x X'.
// Backward, with x^ = r_x X', y^ = r_y Y, u = w_post gate_c, g = w_pre dN:
//   D = dX' + r_x (g - x^ mean(g x^)),   dX = res_scale D,
//   dY = gate_t r_y (u D - y^ mean(u D y^)),           dgate_t = sum_c u D y^,
//   A = sum_t dN x^ = dw_pre,  S = sum_t gate_t D y^:  dw_post = gate_c S, dgate_c = w_post S.
// All arithmetic in fp32; X' is rounded once when stored, and N is formed from the sum before
// that rounding.
//
// Both directions are bound by memory: 4 (forward) and 6 (backward) rows of d elements move per
// token and about 10 to 30 operations are done per element. So a row is read once and held in
// registers between its sums and its outputs, eight elements per thread and chunk.
#include "block.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

// Layout of a launch: NT threads per row, each with CH chunks of 8 columns, chunk i of thread x at
// column (i NT + x) 8; R rows at a time per workgroup. A thread sees the same columns in all of
// its rows, so it loads their weights once and keeps their parameter sums in registers.
template <int NT> struct Rows {
  static constexpr int kThreads = NT < 256 ? 256 : NT;
  static constexpr int R = kThreads / NT;
};

// Sums of n values over the NT threads of a row, in each of them. Above a wave they go through
// LDS, two buffers in turn (one barrier per call); every wave reads the waves' sums back one per
// lane and folds them by DPP.
template <int NT, int n> struct RowSum {
  static constexpr int kWaves = NT > kWave ? NT / kWave : 1;
  float (*buf)[Rows<NT>::R][kWaves][n];
  int turn = 0;
  __device__ __forceinline__ void operator()(float (&v)[n]) {
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = group_sum<(NT < kWave ? NT : kWave)>(v[i]);
    if (NT <= kWave) return;
    if (lane_id() == 0)
#pragma unroll
      for (int i = 0; i < n; ++i) buf[turn][threadIdx.x / NT][threadIdx.x % NT / kWave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < n; ++i)
      v[i] = group_sum<(kWaves > 1 ? kWaves : 2)>(buf[turn][threadIdx.x / NT][lane_id() % kWaves][i]);
    turn ^= 1;
  }
};

// A parameter's eight values of one chunk; ones where there is no parameter.
__device__ __forceinline__ void load_param(const float* w, int c, int d, float (&v)[kVec]) {
  if (!w) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = 1.f;
    return;
  }
  const Vec8<float> p = load8(w, c, d);
#pragma unroll
  for (int i = 0; i < kVec; ++i) v[i] = p.get(i);
}

// u = w_post gate_c of one chunk.
template <typename P> __device__ __forceinline__ void load_u(const P& p, int c, int d, float (&u)[kVec]) {
  float g[kVec];
  load_param(p.w_post, c, d, u);
  load_param(p.gate_c, c, d, g);
#pragma unroll
  for (int i = 0; i < kVec; ++i) u[i] *= g[i];
}

template <typename V, int NT, int CH>
__global__ __launch_bounds__(Rows<NT>::kThreads) void k_norm_fwd(NormParams p) {
  using L = Rows<NT>;
  __shared__ float red[2][L::R][RowSum<NT, 1>::kWaves][1];
  RowSum<NT, 1> row_sum{red};
  const int x = threadIdx.x % NT, d = (int)p.d;
  const float inv_d = 1.f / (float)d;
  float u[CH][kVec], w[CH][kVec];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    load_u(p, (i * NT + x) * kVec, d, u[i]);
    load_param(p.w_pre, (i * NT + x) * kVec, d, w[i]);
  }
  const int64_t step = (int64_t)gridDim.x * L::R;
  // every thread of a workgroup takes as many turns (row_sum has barriers)
  for (int64_t t0 = (int64_t)blockIdx.x * L::R; t0 < p.T; t0 += step) {
    const int64_t t = t0 + threadIdx.x / NT;
    const bool in = L::R == 1 || t < p.T;
    const int64_t base = (in ? t : p.T - 1) * p.d;
    Vec8<V> X[CH], Y[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int c = (i * NT + x) * kVec;
      X[i] = load8((const V*)p.X + base, c, d);
      if (p.Y) Y[i] = load8((const V*)p.Y + base, c, d);
    }
    float gt = p.gate_t ? p.gate_t[in ? t : p.T - 1] : 1.f;
    if (p.post) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) s[0] = fmaf(Y[i].get(e), Y[i].get(e), s[0]);
      row_sum(s);
      gt *= 1.f / sqrtf(s[0] * inv_d + p.eps);
    }
    float o[CH][kVec], s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        o[i][e] = p.res_scale * X[i].get(e);
        if (p.Y) o[i][e] = fmaf(gt * u[i][e], Y[i].get(e), o[i][e]);
        s[0] = fmaf(o[i][e], o[i][e], s[0]);
      }
    if (p.X_out && in)
#pragma unroll
      for (int i = 0; i < CH; ++i) store8((V*)p.X_out + base, (i * NT + x) * kVec, d, o[i]);
    if (p.pre) {
      row_sum(s);
      const float rx = 1.f / sqrtf(s[0] * inv_d + p.eps);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[i][e] *= rx * w[i][e];
        if (in) store8((V*)p.N + base, (i * NT + x) * kVec, d, o[i]);
      }
    }
  }
}

// One pass per row: every sum that the outputs need is a sum over the row of products of the loaded
// values, so all six are taken together (one barrier per row). With q = sum g x, D is
// dX' + r_x g - r_x^3 q / d x, and the sum of u D y follows from those of u y dX', u y g, u y x.
// HOLD: the row and the weights stay in registers between the sums and the outputs; else (wide
// rows) they are read again, from L2, and the parameter sums are kept in LDS.
template <typename V, int NT, int CH, bool HOLD>
__global__ __launch_bounds__(Rows<NT>::kThreads) void k_norm_bwd(NormBwdParams p) {
  using L = Rows<NT>;
  constexpr int H = HOLD ? CH : 1;
  constexpr int W = CH * NT * kVec;
  extern __shared__ float sums[];  // [R][2][W], with HOLD only used at the end
  __shared__ float red[2][L::R][RowSum<NT, 6>::kWaves][6];
  RowSum<NT, 6> row_sum{red};
  const int x = threadIdx.x % NT, d = (int)p.d;
  const float inv_d = 1.f / (float)d;
  float u[H][kVec], w[H][kVec], A[H][kVec], S[H][kVec];
  float* mine = sums + threadIdx.x / NT * 2 * W + x * kVec;  // chunk i of A at i NT 8, of S at W + i NT 8
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    if (HOLD) {
      load_u(p, (i * NT + x) * kVec, d, u[i % H]);
      load_param(p.w_pre, (i * NT + x) * kVec, d, w[i % H]);
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      if (HOLD)
        A[i % H][e] = S[i % H][e] = 0.f;
      else
        mine[i * NT * kVec + e] = mine[W + i * NT * kVec + e] = 0.f;
    }
  }
  Vec8<V> X[H], Y[H], G[H], N[H];  // X_out, Y, dX_out, dN
  const int64_t step = (int64_t)gridDim.x * L::R;
  for (int64_t t0 = (int64_t)blockIdx.x * L::R; t0 < p.T; t0 += step) {
    const int64_t t = t0 + threadIdx.x / NT;
    const bool in = L::R == 1 || t < p.T;  // a group past the end goes along (barriers) and adds nothing
    const int64_t base = (in ? t : p.T - 1) * p.d;
    auto load = [&](int i) {
      const int c = (i * NT + x) * kVec, h = i % H;
      X[h] = p.pre ? load8((const V*)p.X_out + base, c, d) : Vec8<V>{};
      Y[h] = p.Y ? load8((const V*)p.Y + base, c, d) : Vec8<V>{};
      G[h] = p.dX_out ? load8((const V*)p.dX_out + base, c, d) : Vec8<V>{};
      N[h] = p.dN ? load8((const V*)p.dN + base, c, d) : Vec8<V>{};
      if (!HOLD) {
        load_u(p, c, d, u[0]);
        load_param(p.w_pre, c, d, w[0]);
      }
    };
    if (HOLD)
#pragma unroll
      for (int i = 0; i < CH; ++i) load(i);
    float s[6] = {};
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (!HOLD) {
        __builtin_amdgcn_sched_barrier(0);  // one chunk's registers at a time
        load(i);
      }
      const int h = i % H;
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float xv = X[h].get(e), yv = Y[h].get(e), g = N[h].get(e) * w[h][e], uy = u[h][e] * yv;
        s[0] = fmaf(xv, xv, s[0]);
        s[1] = fmaf(g, xv, s[1]);
        s[2] = fmaf(yv, yv, s[2]);
        s[3] = fmaf(uy, G[h].get(e), s[3]);
        s[4] = fmaf(uy, g, s[4]);
        s[5] = fmaf(uy, xv, s[5]);
      }
    }
    row_sum(s);
    const float rx = p.pre ? 1.f / sqrtf(s[0] * inv_d + p.eps) : 0.f;
    const float k = rx * rx * rx * (s[1] * inv_d);  // D = dX' + rx g - k x
    const float ry = p.post ? 1.f / sqrtf(s[2] * inv_d + p.eps) : 1.f;
    const float Q = ry * (s[3] + rx * s[4] - k * s[5]);
    if (!in) continue;
    const float gt = p.gate_t ? p.gate_t[t] : 1.f;
    if (p.dgate_t && x == 0) p.dgate_t[t] = Q;
    const float gr = gt * ry, ky = p.post ? gr * ry * Q * inv_d : 0.f;  // dY = gr u D - ky y
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      if (!HOLD) {
        __builtin_amdgcn_sched_barrier(0);
        load(i);
      }
      const int h = i % H, c = (i * NT + x) * kVec;
      float dx[kVec], dy[kVec];
      float(&a)[kVec] = HOLD ? A[h] : *(float(*)[kVec])(mine + i * NT * kVec);
      float(&b)[kVec] = HOLD ? S[h] : *(float(*)[kVec])(mine + W + i * NT * kVec);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float xv = X[h].get(e), yv = Y[h].get(e), n = N[h].get(e);
        const float D = fmaf(-k, xv, fmaf(rx, n * w[h][e], G[h].get(e)));
        a[e] = fmaf(n, xv * rx, a[e]);
        b[e] = fmaf(D, yv * gr, b[e]);
        dx[e] = p.res_scale * D;
        dy[e] = fmaf(gr * u[h][e], D, -ky * yv);
      }
      if (p.dX) store8((V*)p.dX + base, c, d, dx);
      if (p.dY) store8((V*)p.dY + base, c, d, dy);
    }
  }
  if (!p.part) return;
  float* part = p.part + (int64_t)blockIdx.x * 2 * d;
  if (HOLD && L::R == 1) {
#pragma unroll
    for (int i = 0; i < H; ++i) {
      store8(part, (i * NT + x) * kVec, d, A[i]);
      store8(part + d, (i * NT + x) * kVec, d, S[i]);
    }
    return;
  }
  // the workgroup's R rows at a time, added in row order
  if (HOLD)
#pragma unroll
    for (int i = 0; i < H; ++i)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        mine[i * NT * kVec + e] = A[i][e];
        mine[W + i * NT * kVec + e] = S[i][e];
      }
  __syncthreads();
  for (int j = threadIdx.x; j < 2 * W; j += L::kThreads) {
    float v = 0.f;
    for (int r = 0; r < L::R; ++r) v += sums[r * 2 * W + j];
    const int c = j % W;
    if (c < d) part[j / W * d + c] = v;
  }
}

// Parameter gradients from the workgroups' sums: a workgroup takes 32 columns of one of the two,
// its threads 32 groups of rows, added in a fixed order (64 columns: 7.0 us at d = 4096 for 128
// workgroups).
constexpr int kSumCols = 32, kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void k_norm_param_sums(NormBwdParams p, int blocks) {
  __shared__ float red[kSumThreads / kSumCols][kSumCols];
  const int64_t cols = cdiv(p.d, kSumCols);
  const bool second = blockIdx.x >= cols;
  if (second ? !p.dw_post && !p.dgate_c : !p.dw_pre) return;
  const int64_t c = (int64_t)(blockIdx.x - (second ? cols : 0)) * kSumCols + threadIdx.x % kSumCols;
  const int g = threadIdx.x / kSumCols;
  float v = 0.f;
  if (c < p.d) {
    const float* a = p.part + (second ? p.d : 0) + c;
    constexpr int G = kSumThreads / kSumCols;
    for (int b0 = g; b0 < blocks; b0 += 8 * G) {
      float q[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) q[i] = a[(int64_t)min(b0 + i * G, blocks - 1) * 2 * p.d];
#pragma unroll
      for (int i = 0; i < 8; ++i) v += b0 + i * G < blocks ? q[i] : 0.f;
    }
  }
  red[g][threadIdx.x % kSumCols] = v;
  __syncthreads();
  if (g != 0 || c >= p.d) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < kSumThreads / kSumCols; ++i) v += red[i][threadIdx.x];
  if (!second) {
    p.dw_pre[c] = v;
  } else {
    if (p.dw_post) p.dw_post[c] = v * (p.gate_c ? p.gate_c[c] : 1.f);
    if (p.dgate_c) p.dgate_c[c] = v * (p.w_post ? p.w_post[c] : 1.f);
  }
}

// Workgroups of the backward: what the chip holds at a time, so that each adds up as many rows as
// can be before it leaves its sums.
constexpr int kBwdBlocks = 512;

// Calls f with NT and CH for a width: one chunk per thread up to 8192 columns, then two.
template <typename F> hipError_t with_layout(int64_t d, F f) {
  using std::integral_constant;
  const int64_t n = cdiv(d, kVec);
#define SFL_NT(nt) \
  if (n <= nt) return f(integral_constant<int, nt>{}, integral_constant<int, 1>{});
  SFL_NT(8) SFL_NT(16) SFL_NT(32) SFL_NT(64) SFL_NT(128) SFL_NT(256) SFL_NT(512) SFL_NT(1024)
#undef SFL_NT
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{});
}

}  // namespace

static int64_t bwd_blocks(int64_t T, int64_t d) {
  int64_t blocks = 0;
  (void)with_layout(d, [&](auto nt, auto) {
    blocks = std::min<int64_t>(cdiv(T, Rows<decltype(nt)::value>::R), kBwdBlocks);
    return hipSuccess;
  });
  return blocks;
}

size_t norm_workspace_bytes(int64_t T, int64_t d) { return (size_t)bwd_blocks(T, d) * 2 * (size_t)d * sizeof(float); }

hipError_t launch_norm_fwd(const NormParams& p, int bf16, hipStream_t s) {
  return with_layout(p.d, [&](auto nt, auto ch) {
    constexpr int NT = decltype(nt)::value, CH = decltype(ch)::value;
    using L = Rows<NT>;
    // twice what the chip holds at a time: rows of a second round fill in where the first's end
    // (8192 x 4096 bf16: 60 us with one round, 56 with two, 64 with a workgroup per row)
    const unsigned grid = (unsigned)std::min<int64_t>(cdiv(p.T, L::R), 256 * (4096 / L::kThreads));
    if (bf16)
      hipLaunchKernelGGL((k_norm_fwd<bf16_t, NT, CH>), dim3(grid), dim3(L::kThreads), 0, s, p);
    else
      hipLaunchKernelGGL((k_norm_fwd<float, NT, CH>), dim3(grid), dim3(L::kThreads), 0, s, p);
    return hipGetLastError();
  });
}

hipError_t launch_norm_bwd(const NormBwdParams& p0, int bf16, hipStream_t s) {
  NormBwdParams p = p0;
  const int64_t blocks = bwd_blocks(p.T, p.d);
  if (!p.dw_pre && !p.dw_post && !p.dgate_c) p.part = nullptr;
  if (blocks > 0) {
    const hipError_t e = with_layout(p.d, [&](auto nt, auto ch) {
      constexpr int NT = decltype(nt)::value, CH = decltype(ch)::value;
      using L = Rows<NT>;
      constexpr bool HOLD = CH == 1;
      constexpr size_t lds = L::R > 1 || !HOLD ? (size_t)L::R * 2 * CH * NT * kVec * sizeof(float) : 0;
      const auto kern = bf16 ? k_norm_bwd<bf16_t, NT, CH, HOLD> : k_norm_bwd<float, NT, CH, HOLD>;
      if (lds > (64 << 10)) {
        const hipError_t e =
            hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
      }
      hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(L::kThreads), lds, s, p);
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
  }
  if (p0.dw_pre || p0.dw_post || p0.dgate_c)
    hipLaunchKernelGGL(k_norm_param_sums, dim3((unsigned)(2 * cdiv(p.d, kSumCols))), dim3(kSumThreads), 0, s, p,
                       (int)blocks);
  return hipGetLastError();
}

}  // namespace sfl
