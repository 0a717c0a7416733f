// Products of 8-bit codes with a power-of-two scale for each block of 128:
//   C[m][n] = sum_b 2^(sa[m][b] + sb[n][b]) sum_{k in block b} A[m][k] B[n][k]
// Rows of the result are the rows of an expert's run, or (the weights' gradients) the sum runs over the
// run's tokens. Codes become bf16 with their scale by one instruction for two of them, exactly for scales from
// 2^-117 on, and bf16 products are exact in the fp32 sums of the matrix cores. (The 8-bit matrix
// instructions are not: they add the products of eight neighbouring k with 13 bits below the largest of
// them, 1.6e-5 of the result's magnitude for normal operands, by measurement.)
#include "blocks8.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

// Eight codes times 2^(byte - 127).
__device__ __forceinline__ bf16x8_t decode8(uint32_t lo, uint32_t hi, float by) {
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, false);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, by, true);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, false);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, by, true);
  return bf16x8_t{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// One tile of a result: pointers to its first row and column.
struct Tile {
  const uint8_t* A;
  const uint8_t* As;
  const uint8_t* B;
  const uint8_t* Bs;
  int64_t lda, ldb, lsa, lsb;  // bytes between rows of codes and of scales
  int m, n;                    // rows and columns that are there
  int blocks;
  int bshift;                  // 7: rows of B share scales by 128
  int b0;                      // row of B, for them
};

constexpr int kThreads = 256, kM = 64, kN = 64;

// 64 x 64 by four waves of 16 rows; operands straight from memory.
template <typename V>
__device__ __forceinline__ void simple_tile(const Tile& t, V* C, int64_t ldc) {
  const int lane = lane_id(), wave = threadIdx.x / kWave, x = lane & 15, g = lane >> 4;
  const int m = min(wave * 16 + x, t.m - 1);
  f32x4_t acc[4] = {};
  for (int b = 0; b < t.blocks; ++b) {
    uint32_t a[8], w[8];
    __builtin_memcpy(a, t.A + m * t.lda + b * 128 + g * 32, 32);
    const float sa = scale8(t.As[m * t.lsa + b]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int n = min(j * 16 + x, t.n - 1);
      __builtin_memcpy(w, t.B + n * t.ldb + b * 128 + g * 32, 32);
      const float sb = scale8(t.Bs[(int64_t)((t.b0 + n) >> t.bshift) * t.lsb + b]);
#pragma unroll
      for (int q = 0; q < 4; ++q)  // lane: row x of A, columns 4 g .. 4 g + 3
        acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode8(w[2 * q], w[2 * q + 1], sb),
                                                         decode8(a[2 * q], a[2 * q + 1], sa), acc[j], 0, 0, 0);
    }
  }
  if (wave * 16 + x >= t.m) return;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = j * 16 + g * 4 + i;
      if (n < t.n) VT<V>::store(C, m * ldc + n, acc[j][i]);
    }
}

template <typename V> __global__ __launch_bounds__(kThreads) void k_product8(Product8 p, int64_t mtiles) {
  const int64_t ntiles = cdiv(p.N, kN), total = mtiles * ntiles, sk = scale_row8(p.K);
  for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
    const int64_t mt = id / ntiles;
    const int nt = (int)(id - mt * ntiles);
    const Unit u = unit_of(p.offsets, p.E, (int)p.rows, kM, (int)mt);
    if (u.expert < 0) return;
    Tile t;
    t.A = p.A + u.first * p.K;
    t.As = p.As + u.first * sk;
    t.B = p.B + ((int64_t)u.expert * p.N + nt * kN) * p.K;
    t.Bs = p.Bs + u.expert * blocks8(p.N) * sk;
    t.lda = t.ldb = p.K;
    t.lsa = t.lsb = sk;
    t.m = u.count;
    t.n = (int)min((int64_t)kN, p.N - (int64_t)nt * kN);
    t.blocks = (int)(p.K / kBlock8);
    t.bshift = 7;
    t.b0 = nt * kN;
    simple_tile(t, (V*)p.C + u.first * p.N + nt * kN, p.N);
  }
}

template <typename V> __global__ __launch_bounds__(kThreads) void k_product8_weights(Product8 p) {
  const int64_t mtiles = cdiv(p.N, kM), ntiles = cdiv(p.K, kN), total = p.E * mtiles * ntiles, ss = p.columns / kBlock8;
  for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
    const int e = (int)(id / (mtiles * ntiles));
    const int64_t rest = id - e * mtiles * ntiles, mt = rest / ntiles, nt = rest - mt * ntiles;
    const Run r = run_of(p.offsets, (int)p.rows, kBlock8, e);
    Tile t;
    t.A = p.A + mt * kM * p.columns + (int64_t)r.before * kBlock8;
    t.As = p.As + mt * kM * ss + r.before;
    t.B = p.B + nt * kN * p.columns + (int64_t)r.before * kBlock8;
    t.Bs = p.Bs + nt * kN * ss + r.before;
    t.lda = t.ldb = p.columns;
    t.lsa = t.lsb = ss;
    t.m = (int)min((int64_t)kM, p.N - mt * kM);
    t.n = (int)min((int64_t)kN, p.K - nt * kN);
    t.blocks = (int)min(blocks8(r.count), max(ss - r.before, (int64_t)0));
    t.bshift = 0;
    t.b0 = 0;
    simple_tile(t, (V*)p.C + ((int64_t)e * p.N + mt * kM) * p.K + nt * kN, p.K);
  }
}

dim3 grid_of(int64_t tiles, int threads) { return dim3((unsigned)std::min<int64_t>(tiles, max_blocks(threads))); }

}  // namespace

hipError_t launch_product8(const Product8& p, int bf16, hipStream_t s) {
  // every run ends in a tile that may not be full
  const int64_t mtiles = p.offsets ? std::min(p.rows, p.rows / kM + p.E) : cdiv(p.rows, kM);
  const dim3 grid = grid_of(mtiles * cdiv(p.N, kN), kThreads);
  if (mtiles == 0) return hipSuccess;
  if (bf16)
    hipLaunchKernelGGL(k_product8<bf16_t>, grid, dim3(kThreads), 0, s, p, mtiles);
  else
    hipLaunchKernelGGL(k_product8<float>, grid, dim3(kThreads), 0, s, p, mtiles);
  return hipGetLastError();
}

hipError_t launch_product8_weights(const Product8& p, int bf16, hipStream_t s) {
  const dim3 grid = grid_of(p.E * cdiv(p.N, kM) * cdiv(p.K, kN), kThreads);
  if (bf16)
    hipLaunchKernelGGL(k_product8_weights<bf16_t>, grid, dim3(kThreads), 0, s, p);
  else
    hipLaunchKernelGGL(k_product8_weights<float>, grid, dim3(kThreads), 0, s, p);
  return hipGetLastError();
}

}  // namespace sfl
