// Row access shared by the operators around the layer: eight elements of a row per thread, whatever
// the row's alignment, and sums over the threads of a row.
#pragma once

#include "common.h"

namespace sfl {

constexpr int kVec = 8;  // elements of a chunk

// A chunk: the eight columns that a thread has of a row, in 16-byte units, so that every access of a
// wave is one run of 1 KiB: eight columns from c0 in bf16, four from c0 and four from c1 in fp32. (Two
// fp32 units side by side wrote 29 % more bytes than there are, by the counter: the wave's stores
// reach a cache line in two halves.)
struct Cols {
  int c0, c1;
};
// Chunk i of thread x of the L threads of a row.
template <typename V> __device__ __forceinline__ Cols cols(int i, int x, int L) {
  if (sizeof(V) == 2) {
    const int c = (i * L + x) * kVec;
    return {c, c + 4};
  }
  const int c = i * L * kVec + x * 4;
  return {c, c + L * 4};
}

// A chunk's elements as loaded (bf16 stays packed until it is used).
template <typename V> struct Vec8;
template <> struct Vec8<bf16_t> {
  u32x4_t w;
  __device__ __forceinline__ float get(int i) const { return i & 1 ? bf16hi(w[i / 2]) : bf16lo(w[i / 2]); }
};
template <> struct Vec8<float> {
  f32x4_t a, b;
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};

// 16 bytes at an address of element alignment: one load or store (the memory system takes
// unaligned vector accesses).
template <typename T, typename P> __device__ __forceinline__ T load16(const P* p) {
  T v;
  __builtin_memcpy(&v, p, 16);
  return v;
}
// Rows that a kernel writes and does not read again are stored non-temporally: they leave their L2
// lines to the rows being read (8192 x 4096 bf16 norm forward 55.8 -> 53.7 us; with a pass that
// reads the result behind it 64.5 -> 63.0). Non-temporal loads lose (68.5 us).
typedef uint32_t u32x4_any_t __attribute__((ext_vector_type(4), aligned(2)));
template <typename T, typename P> __device__ __forceinline__ void store16(P* p, T v) {
  u32x4_any_t w;
  __builtin_memcpy(&w, &v, 16);
  __builtin_nontemporal_store(w, (u32x4_any_t*)p);
}

// Drops the first s elements (at most all) of a unit and lets zeros in behind them.
__device__ __forceinline__ void drop(u32x4_t& w, int s) {
  uint64_t lo = (uint64_t)w[1] << 32 | w[0], hi = (uint64_t)w[3] << 32 | w[2];
  if (s & 4) {
    lo = hi;
    hi = 0;
  }
  const int bits = (s & 3) * 16;
  if (bits) {
    lo = lo >> bits | hi << (64 - bits);
    hi >>= bits;
  }
  if (s & 8) lo = hi = 0;
  w = u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ void drop(f32x4_t& v, int s) {
  if (s & 2) v = f32x4_t{v[2], v[3], 0.f, 0.f};
  if (s & 1) v = f32x4_t{v[1], v[2], v[3], 0.f};
  if (s & 4) v = f32x4_t{};
}

// Units of N elements of type V, held as U. Where a unit passes the row's end, load_unit takes the
// row's last N elements instead, with no branch around the load, so that the loads of several rows
// go out together; settle_unit then shifts them to their places, with zeros past the end. (Rows of
// fewer than N elements are read one by one and need no settling.)
template <typename U, typename V> __device__ __forceinline__ U load_unit(const V* row, int c, int d) {
  constexpr int N = 16 / sizeof(V);
  if (d >= N) return load16<U>(row + min(c, d - N));
  V e[N] = {};
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (c + i < d) e[i] = row[c + i];
  U v;
  __builtin_memcpy(&v, e, 16);
  return v;
}
template <int N, typename U> __device__ __forceinline__ void settle_unit(U& v, int c, int d) {
  if (c + N > d && d >= N) drop(v, min(c + N - d, N));
}
// What is past the row's end is left out (N / 2, ... and one element at a time).
template <typename U, typename V> __device__ __forceinline__ void store_unit(V* row, int c, int d, U v) {
  constexpr int N = 16 / sizeof(V);
  if (c + N <= d) return store16(row + c, v);
  if (c >= d) return;
  V* p = row + c;
#pragma unroll
  for (int n = N / 2; n > 0; n /= 2)
    if ((d - c) & n) {
      __builtin_memcpy(p, &v, n * sizeof(V));
      p += n;
      drop(v, n);
    }
}
// Where a unit's elements go one by one to the same place of another row, a unit that load_unit moved
// back may be stored where it was loaded: its neighbour stores the same values there.
template <typename U, typename V> __device__ __forceinline__ void store_unit_raw(V* row, int c, int d, const U& v) {
  constexpr int N = 16 / sizeof(V);
  if (c >= d) return;
  if (d >= N)
    store16(row + min(c, d - N), v);
  else
    store_unit(row, c, d, v);
}

// The same for chunks.
__device__ __forceinline__ Vec8<bf16_t> load_raw(const bf16_t* row, Cols c, int d) { return {load_unit<u32x4_t>(row, c.c0, d)}; }
__device__ __forceinline__ Vec8<float> load_raw(const float* row, Cols c, int d) {
  return {load_unit<f32x4_t>(row, c.c0, d), load_unit<f32x4_t>(row, c.c1, d)};
}
__device__ __forceinline__ void settle(Vec8<bf16_t>& v, Cols c, int d) { settle_unit<8>(v.w, c.c0, d); }
__device__ __forceinline__ void settle(Vec8<float>& v, Cols c, int d) {
  settle_unit<4>(v.a, c.c0, d);
  settle_unit<4>(v.b, c.c1, d);
}
template <typename V> __device__ __forceinline__ Vec8<V> load8(const V* row, Cols c, int d) {
  Vec8<V> v = load_raw(row, c, d);
  settle(v, c, d);
  return v;
}
__device__ __forceinline__ void store8(bf16_t* row, Cols c, int d, const Vec8<bf16_t>& v) { store_unit(row, c.c0, d, v.w); }
__device__ __forceinline__ void store8(float* row, Cols c, int d, const Vec8<float>& v) {
  store_unit(row, c.c0, d, v.a);
  store_unit(row, c.c1, d, v.b);
}
__device__ __forceinline__ void store_raw(bf16_t* row, Cols c, int d, const Vec8<bf16_t>& v) {
  store_unit_raw(row, c.c0, d, v.w);
}
__device__ __forceinline__ void store_raw(float* row, Cols c, int d, const Vec8<float>& v) {
  store_unit_raw(row, c.c0, d, v.a);
  store_unit_raw(row, c.c1, d, v.b);
}
// Whether element e of a raw chunk is there and not its neighbour's (all are where every unit is
// whole: ask raw_whole first).
template <typename V> __device__ __forceinline__ bool raw_whole(Cols c, int d) {
  return (sizeof(V) == 2 ? c.c0 + 8 : c.c1 + 4) <= d;
}
template <typename V> __device__ __forceinline__ bool raw_own(int e, Cols c, int d) {
  constexpr int N = 16 / sizeof(V);
  const int at = e < N ? c.c0 : c.c1;
  return d < N || e % N >= at + N - d;
}

// Two floats to packed bf16, each to nearest even (NaN stays a NaN): one v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t v = __builtin_convertvector((f32x2_t{lo, hi}), bf16x2_t);
  uint32_t w;
  __builtin_memcpy(&w, &v, 4);
  return w;
}
template <typename V> __device__ __forceinline__ Vec8<V> rounded(const float (&v)[kVec]);
template <> __device__ __forceinline__ Vec8<bf16_t> rounded<bf16_t>(const float (&v)[kVec]) {
  return {u32x4_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}};
}
template <> __device__ __forceinline__ Vec8<float> rounded<float>(const float (&v)[kVec]) {
  return {f32x4_t{v[0], v[1], v[2], v[3]}, f32x4_t{v[4], v[5], v[6], v[7]}};
}

template <int CTRL> __device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}

// Sum over aligned groups of N <= 64 lanes, in every lane. Lanes trade inside a row of 16 by DPP
// (no LDS round trip); the four rows of a wave are read out and added in lane order.
template <int N> __device__ __forceinline__ float group_sum(float v) {
  static_assert(N >= 2 && N <= 64 && (N & (N - 1)) == 0, "");
  v = dpp_add<0xB1>(v);               // quad_perm: lane ^ 1
  if (N >= 4) v = dpp_add<0x4E>(v);   // quad_perm: lane ^ 2
  if (N >= 8) v = dpp_add<0x141>(v);  // row_half_mirror: the other quad of eight lanes
  if (N >= 16) v = dpp_add<0x140>(v);  // row_mirror: the other eight of the row
  if (N == 32) v += __shfl_xor(v, 16, 64);
  if (N == 64) v = (readlane_f(v, 0) + readlane_f(v, 16)) + (readlane_f(v, 32) + readlane_f(v, 48));
  return v;
}

// Calls f with a first token, a number of tokens and their workgroups (of THREADS threads, PER tokens
// each), for as many tokens at a time as one launch takes: 2^24 - 1 workgroups of 256 threads.
template <int THREADS, int PER, typename F> hipError_t over_tokens(int64_t T, F f) {
  constexpr int64_t most = max_blocks(THREADS) * PER;
  for (int64_t t0 = 0; t0 < T; t0 += most) {
    const int64_t n = T - t0 < most ? T - t0 : most;
    f(t0, n, dim3((unsigned)cdiv(n, PER)));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace sfl
