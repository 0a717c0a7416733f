// Rows, columns and weights to 8 bits: for a block of 128 elements the smallest power of two 2^e by
// which its largest magnitude comes down to 448, and the nearest e4m3 codes of x 2^-e. Blocks lie
// along a row (k_quant_rows), along a row and along a run's tokens at once, or in squares of 128 x 128
// (k_quant_tile). Bound by memory: every element is read once for both layouts.
#include "blocks8.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;

template <int CTRL> __device__ __forceinline__ uint32_t dpp_top(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}
// Largest value over aligned groups of 16 lanes, in every lane.
__device__ __forceinline__ uint32_t top16(uint32_t v) {
  v = dpp_top<0xB1>(v);
  v = dpp_top<0x4E>(v);
  v = dpp_top<0x141>(v);
  return dpp_top<0x140>(v);
}

// Eight elements from column c on, zeros from column d on.
template <typename V> __device__ __forceinline__ void load_eight(const V* row, int c, int d, float (&x)[8]) {
  if (c + 8 <= d) {
    V v[8];
    __builtin_memcpy(v, row + c, sizeof(v));
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = VT<V>::load(v, i);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = c + i < d ? VT<V>::load(row, c + i) : 0.f;
  }
}
template <typename V>
__device__ __forceinline__ void load_eight(const V* row, const V* where, int c, int d, float (&x)[8]) {
  load_eight(row, c, d, x);
  if (where) {
    float w[8];
    load_eight(where, c, d, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = w[i] > 0.f ? x[i] : 0.f;
  }
}

// Four blocks of a row per wave, 16 lanes a block.
template <typename V>
__global__ __launch_bounds__(kThreads) void k_quant_rows(const V* __restrict__ X, const V* __restrict__ where,
                                                         int64_t T, int d, const int32_t* __restrict__ offsets, int E,
                                                         uint8_t* __restrict__ Q, uint8_t* __restrict__ S) {
  const int dq = (int)up(d, kBlock8), sq = (int)scale_row8(d), units = sq / 4;
  const int64_t total = T * units, step = (int64_t)gridDim.x * (kThreads / kWave);
  const int lane = lane_id();
  int64_t t0 = 0, t1 = T;
  if (offsets) {
    t0 = offset8(offsets, 0, (int)T);
    t1 = offset8(offsets, E, (int)T);
  }
  for (int64_t i = (int64_t)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave; i < total; i += step) {
    const int64_t t = i / units;
    const int u = (int)(i - t * units), c = u * 512 + lane * 8;
    if (t < t0 || t >= t1) continue;
    float x[8];
    load_eight(X + t * d, where ? where + t * d : nullptr, c, d, x);
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, magnitude8(x[j]));
    const int byte = scale_byte8(top16(top));
    const float by = inverse8(byte);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] *= by;
    if (c < dq) {
      const u32x2_t w{codes8(x[0], x[1], x[2], x[3]), codes8(x[4], x[5], x[6], x[7])};
      __builtin_memcpy(Q + t * dq + c, &w, 8);
    }
    const uint32_t four = (uint32_t)readlane_i(byte, 0) | (uint32_t)readlane_i(byte, 16) << 8 |
                          (uint32_t)readlane_i(byte, 32) << 16 | (uint32_t)readlane_i(byte, 48) << 24;
    if (lane == 0) *(uint32_t*)(S + t * sq + u * 4) = four;
  }
}

struct TileArgs {
  const void* X;
  const void* where;
  const int32_t* offsets;
  uint8_t* Q;
  uint8_t* S;
  uint8_t* Qt;
  uint8_t* St;
  int64_t matrices, R, C;  // matrices of R x C; runs of one matrix with offsets
  int64_t ldt, lds;        // row strides of Qt and St
  int E;
};

// 128 rows x 128 columns per workgroup: thread (r, c) holds rows 8 r .. 8 r + 7 at columns 8 c ..
// 8 c + 7, so that a load of 16 lanes is a run of 128 elements of a row, and the eight tokens of a
// column are eight neighbouring bytes of the other layout, which goes through LDS.
template <typename V, bool SQUARE>
__global__ __launch_bounds__(kThreads) void k_quant_tile(TileArgs a) {
  constexpr int kRow = kBlock8 + 8;
  __shared__ uint32_t top_of[kThreads / kWave][kBlock8];
  __shared__ __attribute__((aligned(16))) uint8_t turned[kBlock8 * kRow];
  const int R = (int)a.R, C = (int)a.C, Cq = (int)up(C, kBlock8), tiles = Cq / kBlock8, sq = (int)scale_row8(C);
  const int wave = threadIdx.x / kWave, lane = lane_id(), c = threadIdx.x % 16, r = threadIdx.x / 16;
  const int64_t units = SQUARE ? a.matrices * blocks8(R) : a.ldt / kBlock8, total = units * tiles;
  for (int64_t id = blockIdx.x; id < total; id += gridDim.x) {
    const int64_t unit = id / tiles;
    const int tile = (int)(id - unit * tiles), c0 = tile * kBlock8 + c * 8;
    int64_t matrix = 0;
    int row0, count, at;  // the tile's rows, and its block along the columns
    if (SQUARE) {
      matrix = unit / blocks8(R);
      at = (int)(unit - matrix * blocks8(R));
      row0 = at * kBlock8;
      count = min(kBlock8, R - row0);
    } else {
      const Unit u = unit_of(a.offsets, a.E, R, kBlock8, (int)unit);
      if (u.expert < 0) return;  // and so for every later one
      row0 = u.first;
      count = u.count;
      at = (int)unit;
    }
    const V* X = (const V*)a.X + (matrix * R + row0) * C;
    const V* where = a.where ? (const V*)a.where + (int64_t)row0 * C : nullptr;
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t t = r * 8 + i;
      if (t < count) {
        load_eight(X + t * C, where ? where + t * C : nullptr, c0, C, x[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = 0.f;
      }
    }
    // largest magnitudes of the columns over this wave's 32 rows, then over all
    uint32_t col[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      col[j] = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) col[j] = max(col[j], magnitude8(x[i][j]));
      col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 16, 64));
      col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 32, 64));
      if (SQUARE && j) col[0] = max(col[0], col[j]);
    }
    if (SQUARE) {
      const uint32_t top = top16(col[0]);
      if (lane == 0) top_of[wave][0] = top;
    } else if (lane < 16) {
#pragma unroll
      for (int j = 0; j < 8; ++j) top_of[wave][c * 8 + j] = col[j];
    }
    __syncthreads();
    int byte[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (SQUARE && j) {
        byte[j] = byte[0];
        continue;
      }
      const int q = SQUARE ? 0 : c * 8 + j;
      byte[j] = scale_byte8(max(max(top_of[0][q], top_of[1][q]), max(top_of[2][q], top_of[3][q])));
    }
    if (a.Q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        int b = byte[0];
        if (!SQUARE) {
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) top = max(top, magnitude8(x[i][j]));
          b = scale_byte8(top16(top));
        }
        const int t = r * 8 + i;
        if (t < count) {
          const float by = inverse8(b);
          const u32x2_t w{codes8(x[i][0] * by, x[i][1] * by, x[i][2] * by, x[i][3] * by),
                          codes8(x[i][4] * by, x[i][5] * by, x[i][6] * by, x[i][7] * by)};
          const int64_t row = matrix * R + row0 + t;
          __builtin_memcpy(a.Q + row * Cq + c0, &w, 8);
          if (!SQUARE && c == 0) {
            a.S[row * sq + tile] = (uint8_t)b;
            if (tile == tiles - 1)
              for (int s = tiles; s < sq; ++s) a.S[row * sq + s] = 127;
          }
        }
      }
      if (SQUARE && threadIdx.x == 0) {
        uint8_t* S = a.S + (matrix * blocks8(R) + at) * sq;
        S[tile] = (uint8_t)byte[0];
        if (tile == tiles - 1)
          for (int s = tiles; s < sq; ++s) S[s] = 127;
      }
    }
    if (a.Qt) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float by = inverse8(byte[j]);
        const u32x2_t w{codes8(x[0][j] * by, x[1][j] * by, x[2][j] * by, x[3][j] * by),
                        codes8(x[4][j] * by, x[5][j] * by, x[6][j] * by, x[7][j] * by)};
        __builtin_memcpy(&turned[(c * 8 + j) * kRow + r * 8], &w, 8);
      }
      __syncthreads();
      const int live = min(kBlock8, C - tile * kBlock8);
      uint8_t* Qt = a.Qt + (matrix * C + tile * kBlock8) * a.ldt + (int64_t)at * kBlock8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = i * 32 + threadIdx.x / 8, k = threadIdx.x % 8 * 16;
        if (n < live) {
          u32x4_t w;
          __builtin_memcpy(&w, &turned[n * kRow + k], 16);
          *(u32x4_t*)(Qt + n * a.ldt + k) = w;
        }
      }
      if (SQUARE) {
        if (threadIdx.x == 0) {
          uint8_t* St = a.St + (matrix * tiles + tile) * a.lds;
          St[at] = (uint8_t)byte[0];
          if (at == (int)blocks8(R) - 1)
            for (int64_t s = at + 1; s < a.lds; ++s) St[s] = 127;
        }
      } else if (r == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c0 + j < C) a.St[(int64_t)(c0 + j) * a.lds + at] = (uint8_t)byte[j];
      }
    }
    __syncthreads();
  }
}

template <typename F> hipError_t over_units(int64_t units, F launch) {
  if (units == 0) return hipSuccess;
  launch(dim3((unsigned)std::min<int64_t>(units, max_blocks(kThreads))));
  return hipGetLastError();
}

template <bool SQUARE> hipError_t launch_tiles(const TileArgs& a, int bf16, int64_t units, hipStream_t s) {
  return over_units(units * blocks8(a.C), [&](dim3 grid) {
    if (bf16)
      hipLaunchKernelGGL((k_quant_tile<bf16_t, SQUARE>), grid, dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL((k_quant_tile<float, SQUARE>), grid, dim3(kThreads), 0, s, a);
  });
}

}  // namespace

hipError_t launch_quant_rows(const sfl_quant_args_t& a, hipStream_t s) {
  const int bf16 = a.dtype == SFL_BF16;
  if (a.Qt) {
    TileArgs t{a.X, a.where, a.offsets, a.Q, a.S, a.Qt, a.St, 1, a.T, a.d, a.columns, a.columns / kBlock8, a.E};
    return launch_tiles<false>(t, bf16, a.offsets ? columns8(a.T, a.E) / kBlock8 : blocks8(a.T), s);
  }
  const int64_t units = a.T * (scale_row8(a.d) / 4);
  return over_units(cdiv(units, kThreads / kWave), [&](dim3 grid) {
    if (bf16)
      hipLaunchKernelGGL(k_quant_rows<bf16_t>, grid, dim3(kThreads), 0, s, (const bf16_t*)a.X, (const bf16_t*)a.where,
                         a.T, (int)a.d, a.offsets, a.E, a.Q, a.S);
    else
      hipLaunchKernelGGL(k_quant_rows<float>, grid, dim3(kThreads), 0, s, (const float*)a.X, (const float*)a.where,
                         a.T, (int)a.d, a.offsets, a.E, a.Q, a.S);
  });
}

hipError_t launch_quant_weights(const void* W, int bf16, int64_t E, int64_t R, int64_t C, uint8_t* Q, uint8_t* S,
                                uint8_t* Qt, uint8_t* St, hipStream_t s) {
  TileArgs t{W, nullptr, nullptr, Q, S, Qt, St, E, R, C, up(R, kBlock8), scale_row8(R), 1};
  return launch_tiles<true>(t, bf16, E * blocks8(R), s);
}

}  // namespace sfl
