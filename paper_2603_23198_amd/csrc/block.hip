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
// registers between its sums and its outputs, eight elements per thread and chunk. Measured, passes
// back to back: forward of 8192 x 4096 bf16 50 us (5.3 TB/s), backward of 16384 x 4096 bf16 with all
// parameter gradients 147 to 149 us (5.4 TB/s); a 1 GiB copy reaches 5.2. The simplest kernels (a workgroup
// of 256 threads per row, rows read again for every sum) took 186 and 1927.
#include "block.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

// Layout of a launch: rows of up to 512 columns take NT = 8 to 64 threads, R = 256 / NT rows at a
// time per workgroup; wider ones a workgroup of as many waves as they need, at most NT threads.
// Every thread has CH chunks of 8 columns. It sees the same columns in all of its rows, so it loads
// their weights once and keeps their parameter sums in registers.
template <int NT> struct Rows {
  static constexpr int kThreads = NT <= kWave ? 256 : NT;
  static constexpr int R = kThreads / NT;
};

// Sums of n values over the threads of a row, in each of them. Above a wave they go through LDS, two
// buffers in turn (one barrier per call); every wave reads the waves' sums back one per lane and
// folds them by DPP.
template <int NT, int n> struct RowSum {
  static constexpr int kWaves = NT > kWave ? NT / kWave : 1;
  float (*buf)[kWaves][n];
  int turn = 0;
  // waves that the workgroup does not have add zeros; a barrier follows before the sums are read
  __device__ __forceinline__ RowSum(float (*b)[kWaves][n]) : buf(b) {
    if (kWaves > 1 && threadIdx.x < kWave)
      for (int i = threadIdx.x; i < 2 * kWaves * n; i += kWave)
        if (i / n % kWaves >= (int)blockDim.x / kWave) (&b[0][0][0])[i] = 0.f;
  }
  __device__ __forceinline__ void operator()(float (&v)[n]) {
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = group_sum<(NT < kWave ? NT : kWave)>(v[i]);
    if (NT <= kWave) return;
    if (lane_id() == 0)
#pragma unroll
      for (int i = 0; i < n; ++i) buf[turn][threadIdx.x / kWave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = group_sum<(kWaves > 1 ? kWaves : 2)>(buf[turn][lane_id() % kWaves][i]);
    turn ^= 1;
  }
};

// A parameter's eight values of one chunk; ones where there is no parameter.
__device__ __forceinline__ void load_param(const float* w, Cols c, int d, float (&v)[kVec]) {
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
template <typename P> __device__ __forceinline__ void load_u(const P& p, Cols c, int d, float (&u)[kVec]) {
  float g[kVec];
  load_param(p.w_post, c, d, u);
  load_param(p.gate_c, c, d, g);
#pragma unroll
  for (int i = 0; i < kVec; ++i) u[i] *= g[i];
}

template <typename V, int NT, int CH>
__global__ __launch_bounds__(Rows<NT>::kThreads) void k_norm_fwd(NormParams p) {
  using L = Rows<NT>;
  __shared__ float red[2][RowSum<NT, 1>::kWaves][1];
  RowSum<NT, 1> row_sum(red);
  const int x = NT <= kWave ? threadIdx.x % NT : threadIdx.x, d = (int)p.d;
  const float inv_d = 1.f / (float)d;
  const int lanes = NT <= kWave ? NT : blockDim.x;
  float u[CH][kVec], w[CH][kVec];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    load_u(p, cols<V>(i, x, lanes), d, u[i]);
    load_param(p.w_pre, cols<V>(i, x, lanes), d, w[i]);
  }
  const int64_t step = (int64_t)gridDim.x * L::R;
  // every thread of a workgroup takes as many turns (row_sum has barriers)
  for (int64_t t0 = (int64_t)blockIdx.x * L::R; t0 < p.T; t0 += step) {
    const int64_t t = t0 + (L::R == 1 ? 0 : threadIdx.x / NT);
    const bool in = L::R == 1 || t < p.T;
    const int64_t base = (in ? t : p.T - 1) * p.d;
    Vec8<V> X[CH], Y[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const Cols c = cols<V>(i, x, lanes);
      X[i] = load_raw((const V*)p.X + base, c, d);
      if (p.Y) Y[i] = load_raw((const V*)p.Y + base, c, d);
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const Cols c = cols<V>(i, x, lanes);
      settle(X[i], c, d);
      if (p.Y) settle(Y[i], c, d);
    }
    float gt = p.gate_t ? p.gate_t[in ? t : p.T - 1] : 1.f;
    if (p.post) {
      float s[1] = {0.f};
#pragma unroll
      for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int e = 0; e < kVec; ++e) s[0] = fmaf(Y[i].get(e), Y[i].get(e), s[0]);
      row_sum(s);
      gt *= rsqrtf(s[0] * inv_d + p.eps);
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
      for (int i = 0; i < CH; ++i) store8((V*)p.X_out + base, cols<V>(i, x, lanes), d, rounded<V>(o[i]));
    if (p.pre) {
      row_sum(s);
      const float rx = rsqrtf(s[0] * inv_d + p.eps);
#pragma unroll
      for (int i = 0; i < CH; ++i) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) o[i][e] *= rx * w[i][e];
        if (in) store8((V*)p.N + base, cols<V>(i, x, lanes), d, rounded<V>(o[i]));
      }
    }
  }
}

// One pass per row: every sum that the outputs need is a sum over the row of products of the loaded
// values, so all six are taken together (one barrier per row). With q = sum g x, D is
// dX' + r_x g - r_x^3 q / d x, and the sum of u D y follows from those of u y dX', u y g, u y x.
// HOLD: the row, the weights and the parameter sums stay in registers; else (wide rows) the row and
// the weights are read again, from L2, for the outputs, and the sums are kept in LDS.
// A bf16 row's loads go out while the row before it is still being summed (16 registers; fp32 rows
// have twice the bytes in flight without). Above 512 columns that takes the bf16 kernel past its 128
// registers: four go to scratch, and so do eleven of the fp32 kernel above 4096 columns.
template <typename V> struct BwdRow {
  Vec8<V> X, Y, G, N;  // X_out, Y, dX_out, dN
  __device__ __forceinline__ void load(const NormBwdParams& p, int64_t base, Cols c, int d) {
    X = p.pre ? load_raw((const V*)p.X_out + base, c, d) : Vec8<V>{};
    Y = p.Y ? load_raw((const V*)p.Y + base, c, d) : Vec8<V>{};
    G = p.dX_out ? load_raw((const V*)p.dX_out + base, c, d) : Vec8<V>{};
    N = p.dN ? load_raw((const V*)p.dN + base, c, d) : Vec8<V>{};
  }
  __device__ __forceinline__ void settled(Cols c, int d) {
    if (raw_whole<V>(c, d)) return;
    settle(X, c, d);
    settle(Y, c, d);
    settle(G, c, d);
    settle(N, c, d);
  }
  __device__ __forceinline__ void add_to(float (&s)[6], const float (&u)[kVec], const float (&w)[kVec]) const {
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const float xv = X.get(e), yv = Y.get(e), g = N.get(e) * w[e], uy = u[e] * yv;
      s[0] = fmaf(xv, xv, s[0]);
      s[1] = fmaf(g, xv, s[1]);
      s[2] = fmaf(yv, yv, s[2]);
      s[3] = fmaf(uy, G.get(e), s[3]);
      s[4] = fmaf(uy, g, s[4]);
      s[5] = fmaf(uy, xv, s[5]);
    }
  }
};

// What the outputs of a row take from its sums.
struct BwdCoef {
  float rx, k, gr, my, Q;  // D = dX' + rx g - k x, dY = gr u D - my (gr y)
  __device__ __forceinline__ BwdCoef(const NormBwdParams& p, const float (&s)[6], float inv_d, float gt) {
    rx = p.pre ? rsqrtf(s[0] * inv_d + p.eps) : 0.f;
    k = rx * (rx * (rx * (s[1] * inv_d)));  // in this order: rx^3 alone overflows for rows of about 1e-13
    const float ry = p.post ? rsqrtf(s[2] * inv_d + p.eps) : 1.f;
    Q = ry * (s[3] + rx * s[4] - k * s[5]);
    gr = gt * ry;
    my = p.post ? ry * (Q * inv_d) : 0.f;
  }
  // A and S: the chunk's parameter sums, the second four from A[hi] on
  template <typename V>
  __device__ __forceinline__ void outputs(const NormBwdParams& p, const BwdRow<V>& r, const float (&u)[kVec],
                                          const float (&w)[kVec], float* A, float* S, int hi, int64_t base, Cols c,
                                          int d) const {
    float dx[kVec], dy[kVec];
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const int at = e < 4 ? e : hi + e - 4;
      const float xv = r.X.get(e), yg = r.Y.get(e) * gr, n = r.N.get(e);
      const float D = fmaf(-k, xv, fmaf(rx, n * w[e], r.G.get(e)));
      A[at] = fmaf(n, xv * rx, A[at]);
      S[at] = fmaf(D, yg, S[at]);
      dx[e] = p.res_scale * D;
      dy[e] = fmaf(gr * u[e], D, -my * yg);
    }
    if (p.dX) store8((V*)p.dX + base, c, d, rounded<V>(dx));
    if (p.dY) store8((V*)p.dY + base, c, d, rounded<V>(dy));
  }
};

template <typename V, int NT, int CH, bool HOLD>
__global__ __launch_bounds__(Rows<NT>::kThreads)
    __attribute__((amdgpu_waves_per_eu(sizeof(V) == 2 ? 4 : 3))) void k_norm_bwd(NormBwdParams p) {
  static_assert(!HOLD || CH == 1, "");
  using L = Rows<NT>;
  constexpr bool AHEAD = HOLD && sizeof(V) == 2;
  extern __shared__ float sums[];  // [R][2][CH * NT * 8]: A, S by column; with HOLD used at the end where R > 1
  __shared__ float red[2][RowSum<NT, 6>::kWaves][6];
  RowSum<NT, 6> row_sum(red);
  constexpr int W = CH * NT * kVec;
  const int x = NT <= kWave ? threadIdx.x % NT : threadIdx.x, d = (int)p.d, group = L::R == 1 ? 0 : threadIdx.x / NT;
  const float inv_d = 1.f / (float)d;
  const int lanes = NT <= kWave ? NT : blockDim.x;
  float* mine = sums + group * 2 * W;  // S behind A
  const Cols own = cols<V>(0, x, lanes);
  float u[kVec], w[kVec], A[kVec], S[kVec];
#pragma unroll
  for (int e = 0; e < kVec; ++e) A[e] = S[e] = 0.f;
  if (HOLD) {
    load_u(p, own, d, u);
    load_param(p.w_pre, own, d, w);
  } else {
    for (int j = threadIdx.x; j < 2 * W; j += NT) mine[j] = 0.f;  // before the barrier of the first row's sums
  }
  const int64_t step = (int64_t)gridDim.x * L::R;
  auto row_of = [&](int64_t t0) { return L::R == 1 ? t0 : min(t0 + group, p.T - 1); };
  BwdRow<V> now, next;
  if (AHEAD) next.load(p, row_of((int64_t)blockIdx.x * L::R) * p.d, own, d);
  for (int64_t t0 = (int64_t)blockIdx.x * L::R; t0 < p.T; t0 += step) {
    const int64_t t = row_of(t0), base = t * p.d;
    const bool in = L::R == 1 || t0 + group < p.T;  // a group past the end goes along (barriers) and adds nothing
    float s[6] = {};
    if (HOLD) {
      if (AHEAD)
        now = next;
      else
        now.load(p, base, own, d);
      now.settled(own, d);
      now.add_to(s, u, w);
      if (AHEAD && t0 + step < p.T) next.load(p, row_of(t0 + step) * p.d, own, d);
    } else {
#pragma unroll 1
      for (int i = 0; i < CH; ++i) {
        const Cols c = cols<V>(i, x, lanes);
        now.load(p, base, c, d);
        now.settled(c, d);
        load_u(p, c, d, u);
        load_param(p.w_pre, c, d, w);
        now.add_to(s, u, w);
      }
    }
    row_sum(s);
    if (!in) continue;
    const BwdCoef f(p, s, inv_d, p.gate_t ? p.gate_t[t] : 1.f);
    if (p.dgate_t && x == 0) p.dgate_t[t] = f.Q;
    if (HOLD) {
      f.outputs(p, now, u, w, A, S, 4, base, own, d);
    } else {
#pragma unroll 1
      for (int i = 0; i < CH; ++i) {
        const Cols c = cols<V>(i, x, lanes);
        now.load(p, base, c, d);
        now.settled(c, d);
        load_u(p, c, d, u);
        load_param(p.w_pre, c, d, w);
        f.outputs(p, now, u, w, mine + c.c0, mine + W + c.c0, c.c1 - c.c0, base, c, d);
      }
    }
  }
  if (!p.part) return;
  float* part = p.part + (int64_t)blockIdx.x * 2 * d;
  if (HOLD && L::R == 1) {
    store8(part, own, d, rounded<float>(A));
    store8(part + d, own, d, rounded<float>(S));
    return;
  }
  // the workgroup's R rows at a time, added in row order
  if (HOLD)
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const int c = e < 4 ? own.c0 + e : own.c1 + e - 4;
      mine[c] = A[e];
      mine[W + c] = S[e];
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
  const int64_t groups = cdiv(p.d, kSumCols);
  const bool second = blockIdx.x >= groups;
  if (second ? !p.dw_post && !p.dgate_c : !p.dw_pre) return;
  const int64_t c = (int64_t)(blockIdx.x - (second ? groups : 0)) * kSumCols + threadIdx.x % kSumCols;
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

// Calls f with NT, CH and the threads of a workgroup for a width: one chunk per thread up to 8192
// columns, then two (row tensors of 2^26 bytes, d = 16384: forward 56 us bf16 and 67 fp32, of which 20
// registers go to scratch; backward 142 and 134; just above 8192 columns, with nearly half the lanes'
// second chunks empty, 70 and 76, and 237 and 152).
template <typename F> hipError_t with_layout(int64_t d, F f) {
  using std::integral_constant;
  const int64_t n = cdiv(d, kVec);
  const int threads = (int)std::min<int64_t>(cdiv(n, kWave) * kWave, 1024);
#define SFL_NT(nt) \
  if (n <= nt) return f(integral_constant<int, nt>{}, integral_constant<int, 1>{}, nt <= kWave ? 256 : threads);
  SFL_NT(8) SFL_NT(16) SFL_NT(32) SFL_NT(64) SFL_NT(128) SFL_NT(256) SFL_NT(512) SFL_NT(1024)
#undef SFL_NT
  return f(integral_constant<int, 1024>{}, integral_constant<int, 2>{}, threads);
}

}  // namespace

// Workgroups of the backward. The fewer there are, the more rows each adds up before it leaves its
// sums, so a CU gets as many as fit into twelve waves (eight of fp32), and one at least, which keep the
// memory busy with full loads, or into all sixteen (twelve) that its registers hold where rows leave
// lanes idle or are not whole in units. Row tensors of 2^26 bytes, all gradients: bf16 d = 2048 (three
// workgroups of four waves) 81 us, four of them 88; d = 4096 (one of eight waves) 82, two 83 (147 and 154
// at twice the rows); d = 640 (sixteen waves) 98, twelve 114; fp32 d = 2048 (eight) 79, twelve 82; d = 640
// (twelve) 86, eight 95.
static int64_t bwd_blocks(int64_t T, int64_t d, int bf16) {
  int64_t blocks = 0;
  (void)with_layout(d, [&](auto nt, auto, int threads) {
    constexpr int NT = decltype(nt)::value;
    const int64_t chunks = cdiv(d, kVec), lanes = NT <= kWave ? NT : threads;
    const int waves = d % kVec == 0 && 4 * chunks >= 3 * lanes ? (bf16 ? 12 : 8) : (bf16 ? 16 : 12);
    blocks = std::min<int64_t>(cdiv(T, Rows<NT>::R), 256 * std::max(1, waves * kWave / threads));
    return hipSuccess;
  });
  return blocks;
}

size_t norm_workspace_bytes(int64_t T, int64_t d, int bf16) {
  return (size_t)bwd_blocks(T, d, bf16) * 2 * (size_t)d * sizeof(float);
}

hipError_t launch_norm_fwd(const NormParams& p, int bf16, hipStream_t s) {
  return with_layout(p.d, [&](auto nt, auto ch, int threads) {
    constexpr int NT = decltype(nt)::value, CH = decltype(ch)::value;
    using L = Rows<NT>;
    // twice what the chip holds at a time: rows of a second round fill in where the first's end
    // (8192 x 4096 bf16: 60 us with one round, 56 with two, 64 with a workgroup per row)
    const unsigned grid = (unsigned)std::min<int64_t>(cdiv(p.T, L::R), 256 * (4096 / threads));
    if (bf16)
      hipLaunchKernelGGL((k_norm_fwd<bf16_t, NT, CH>), dim3(grid), dim3(threads), 0, s, p);
    else
      hipLaunchKernelGGL((k_norm_fwd<float, NT, CH>), dim3(grid), dim3(threads), 0, s, p);
    return hipGetLastError();
  });
}

hipError_t launch_norm_bwd(const NormBwdParams& p0, int bf16, hipStream_t s) {
  NormBwdParams p = p0;
  const int64_t blocks = bwd_blocks(p.T, p.d, bf16);
  if (!p.dw_pre && !p.dw_post && !p.dgate_c) p.part = nullptr;
  if (blocks > 0) {
    const hipError_t e = with_layout(p.d, [&](auto nt, auto ch, int threads) {
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
      hipLaunchKernelGGL(kern, dim3((unsigned)blocks), dim3(threads), lds, s, p);
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
