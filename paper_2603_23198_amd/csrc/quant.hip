// Rows, columns and weights to 8 bits: for a block of 128 elements the smallest power of two 2^e by
// which its largest magnitude comes down to 448, and the nearest e4m3 codes of x 2^-e. Blocks lie
// along a row (k_quant_rows), along a row and along a run's tokens at once, or in squares of 128 x 128
// (k_quant_tile). Bound by memory: every element is read once for both layouts. 16384 x 4096 bf16: rows
// 40 us (5.0 TB/s), both layouts 64 (4.2; 158 registers, three waves a SIMD; with a tile's elements kept
// unpacked 190, two waves and 70 us), of fp32 rows 88 (4.6); 4096 x 16384 fp32 in squares, both
// layouts, 80 us (5.1).
#include "blocks8.h"
#include "order.h"
#include "rows.h"

#include <algorithm>

namespace sfl {

namespace {

constexpr int kThreads = 256;

// Largest magnitude so far and of eight elements; a NaN has no part in it (fmaxf leaves it out), an infinity
// has: where one shows, the caller counts again without those (see finite_top).
__device__ __forceinline__ float most(float top, const float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(x[i]));
  return top;
}
__device__ __forceinline__ uint32_t finite_most(uint32_t top, const float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, magnitude8(x[i]));
  return top;
}
// The bits of the largest finite magnitude of 16 lanes' eight elements each.
__device__ __forceinline__ uint32_t top_of_row(const float (&x)[8]) {
  uint32_t top = group_max<16>(__float_as_uint(most(0.f, x)));
  if (top == 0x7f800000u) top = group_max<16>(finite_most(0u, x));
  return top;
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
    const int byte = scale_byte8(top_of_row(x));
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

// Eight neighbouring elements as they are in memory, and with those dropped where another eight are not above
// zero.
__device__ __forceinline__ void load_raw8(const bf16_t* p, Vec8<bf16_t>& v) { v.w = load16<u32x4_t>(p); }
__device__ __forceinline__ void load_raw8(const float* p, Vec8<float>& v) {
  v.a = load16<f32x4_t>(p);
  v.b = load16<f32x4_t>(p + 4);
}
__device__ __forceinline__ void set(Vec8<bf16_t>& v, int i, bf16_t x) {
  v.w[i / 2] = i & 1 ? (v.w[i / 2] & 0xffffu) | (uint32_t)x << 16 : (v.w[i / 2] & 0xffff0000u) | x;
}
__device__ __forceinline__ void set(Vec8<float>& v, int i, float x) {
  if (i < 4)
    v.a[i] = x;
  else
    v.b[i - 4] = x;
}
template <typename V> __device__ __forceinline__ void keep_where(Vec8<V>& v, const Vec8<V>& w) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (!(w.get(i) > 0.f)) set(v, i, V(0));
}
// The same of a row of d with zeros behind it, rows of fewer than eight element by element.
template <typename V> __device__ __forceinline__ void load_edge(const V* row, int c, int d, Vec8<V>& v) {
  if (d >= 8) {
    v = load8(row, Cols{c, c + 4}, d);
    return;
  }
  v = Vec8<V>{};
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    const V e = c + i < d ? row[c + i] : V(0);
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k == i) set(v, k, e);
  }
}

// The packed elements, hidden from the optimiser, which would keep all of a tile's unpacked from one use of them to
// the next.
__device__ __forceinline__ void hide(Vec8<bf16_t>& v) { asm volatile("" : "+v"(v.w)); }
__device__ __forceinline__ void hide(Vec8<float>&) {}

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

// Scale `at` of a row of n, and 127 up to `room` by the last one's writer.
__device__ __forceinline__ void store_scale(uint8_t* S, int at, int n, int room, int byte) {
  S[at] = (uint8_t)byte;
  if (at == n - 1)
    for (int s = n; s < room; ++s) S[s] = 127;
}
// A row's eight elements from column c0 on as codes.
__device__ __forceinline__ void store_codes(const TileArgs& a, int64_t row, int c0, int tile, int tiles, int Cq, int sq,
                                            int byte, const float (&v)[8], bool scale) {
  const float by = inverse8(byte);
  const u32x2_t w{codes8(v[0] * by, v[1] * by, v[2] * by, v[3] * by), codes8(v[4] * by, v[5] * by, v[6] * by, v[7] * by)};
  __builtin_memcpy(a.Q + row * Cq + c0, &w, 8);
  if (scale) store_scale(a.S + row * sq, tile, tiles, sq, byte);
}

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
    const int live = min(kBlock8, C - tile * kBlock8);
    Vec8<V> x[8];
    auto row_of = [&](int i) { return (int64_t)min(r * 8 + i, count - 1) * C; };
    if (live == kBlock8) {
#pragma unroll
      for (int i = 0; i < 8; ++i) load_raw8(X + row_of(i) + c0, x[i]);
      if (where) {
        Vec8<V> w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) load_raw8(where + row_of(i) + c0, w[i]);
#pragma unroll
        for (int i = 0; i < 8; ++i) keep_where(x[i], w[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        load_edge(X + row_of(i), c0, C, x[i]);
        if (where) {
          Vec8<V> w;
          load_edge(where + row_of(i), c0, C, w);
          keep_where(x[i], w);
        }
      }
    }
    if (count < kBlock8) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r * 8 + i >= count) x[i] = Vec8<V>{};
    }
    // Rows: their scales and codes; and the columns' largest magnitudes over this thread's rows. (The scheduling
    // barriers keep one row's or column's values alive at a time: without them all 64 are, at 240 registers.)
    uint32_t col[8] = {};
    float high[8] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[j] = x[i].get(j);
        high[j] = fmaxf(high[j], fabsf(v[j]));
      }
      if (!SQUARE && a.Q) {
        const int t = r * 8 + i, b = scale_byte8(top_of_row(v));
        if (t < count) store_codes(a, row0 + t, c0, tile, tiles, Cq, sq, b, v, c == 0);
      }
      hide(x[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    bool infinite = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      col[j] = __float_as_uint(high[j]);
      infinite |= high[j] == INFINITY;
    }
    if (ballot(infinite)) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        col[j] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) col[j] = max(col[j], magnitude8(x[i].get(j)));
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    if (SQUARE) {
#pragma unroll
      for (int j = 1; j < 8; ++j) col[0] = max(col[0], col[j]);
      col[0] = group_max<16>(col[0]);
    }
    // over the wave's 32 rows, then over all
    if (SQUARE || a.Qt) {
#pragma unroll
      for (int j = 0; j < (SQUARE ? 1 : 8); ++j) {
        col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 16, 64));
        col[j] = max(col[j], (uint32_t)__shfl_xor((int)col[j], 32, 64));
        if (lane < 16) top_of[wave][SQUARE ? 0 : c * 8 + j] = col[j];
      }
      __syncthreads();
      auto byte_of = [&](int j) {
        const int q = SQUARE ? 0 : c * 8 + j;
        return scale_byte8(max(max(top_of[0][q], top_of[1][q]), max(top_of[2][q], top_of[3][q])));
      };
      const int one = SQUARE ? byte_of(0) : 0;
      if (SQUARE && a.Q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          float v[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = x[i].get(j);
          if (r * 8 + i < count) store_codes(a, matrix * R + row0 + r * 8 + i, c0, tile, tiles, Cq, sq, one, v, false);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (threadIdx.x == 0) store_scale(a.S + (matrix * blocks8(R) + at) * sq, tile, tiles, sq, one);
      }
      if (a.Qt) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int b = SQUARE ? one : byte_of(j);
          const float by = inverse8(b);
          const u32x2_t w{codes8(x[0].get(j) * by, x[1].get(j) * by, x[2].get(j) * by, x[3].get(j) * by),
                          codes8(x[4].get(j) * by, x[5].get(j) * by, x[6].get(j) * by, x[7].get(j) * by)};
          __builtin_memcpy(&turned[(c * 8 + j) * kRow + r * 8], &w, 8);
          if (!SQUARE && r == 0 && c0 + j < C) a.St[(int64_t)(c0 + j) * a.lds + at] = (uint8_t)b;
          __builtin_amdgcn_sched_barrier(0);
        }
        __syncthreads();
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
        if (SQUARE && threadIdx.x == 0)
          store_scale(a.St + (matrix * tiles + tile) * a.lds, at, (int)blocks8(R), (int)a.lds, one);
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
