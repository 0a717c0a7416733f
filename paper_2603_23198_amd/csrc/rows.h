// Row access shared by the operators around the layer: eight consecutive elements of a row per
// thread, whatever the row's alignment, and sums over the threads of a row.
#pragma once

#include "common.h"

namespace sfl {

constexpr int kVec = 8;  // elements of one load: 16 bytes of bf16, two times 16 of fp32

// Eight elements as loaded (bf16 stays packed until it is used).
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

__device__ __forceinline__ Vec8<bf16_t> load_full(const bf16_t* p) { return {load16<u32x4_t>(p)}; }
__device__ __forceinline__ Vec8<float> load_full(const float* p) { return {load16<f32x4_t>(p), load16<f32x4_t>(p + 4)}; }

// Drops the first s <= 8 of eight elements and lets zeros in behind them.
__device__ __forceinline__ void drop(Vec8<bf16_t>& v, int s) {
  uint64_t lo = (uint64_t)v.w[1] << 32 | v.w[0], hi = (uint64_t)v.w[3] << 32 | v.w[2];
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
  v.w = u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}
__device__ __forceinline__ void drop(Vec8<float>& v, int s) {
  if (s & 4) {
    v.a = v.b;
    v.b = f32x4_t{};
  }
  if (s & 2) {
    v.a = f32x4_t{v.a[2], v.a[3], v.b[0], v.b[1]};
    v.b = f32x4_t{v.b[2], v.b[3], 0.f, 0.f};
  }
  if (s & 1) {
    v.a = f32x4_t{v.a[1], v.a[2], v.a[3], v.b[0]};
    v.b = f32x4_t{v.b[1], v.b[2], v.b[3], 0.f};
  }
  if (s & 8) v.a = v.b = f32x4_t{};
}

// A chunk is the elements c .. c + 7 of a row of d. Where it passes the row's end, load_raw takes
// the row's last eight elements instead, with no branch around the load, so that the loads of several
// rows go out together; settle then shifts them to their places, with zeros past the end. (Rows of
// fewer than eight elements are read one by one and need no settling.)
template <typename V> __device__ __forceinline__ Vec8<V> load_raw(const V* row, int c, int d) {
  if (d >= kVec) return load_full(row + min(c, d - kVec));
  V e[kVec] = {};
#pragma unroll
  for (int i = 0; i < kVec; ++i)
    if (c + i < d) e[i] = row[c + i];
  Vec8<V> v;
  __builtin_memcpy(&v, e, sizeof(e));
  return v;
}
template <typename V> __device__ __forceinline__ void settle(Vec8<V>& v, int c, int d) {
  if (c + kVec > d && d >= kVec) drop(v, min(c + kVec - d, kVec));
}
template <typename V> __device__ __forceinline__ Vec8<V> load8(const V* row, int c, int d) {
  Vec8<V> v = load_raw(row, c, d);
  settle(v, c, d);
  return v;
}

__device__ __forceinline__ void store_full(bf16_t* p, const Vec8<bf16_t>& v) { store16(p, v.w); }
__device__ __forceinline__ void store_full(float* p, const Vec8<float>& v) {
  store16(p, v.a);
  store16(p + 4, v.b);
}

// Eight elements to a chunk; what is past the row's end is left out (four, two and one elements at
// a time).
template <typename V> __device__ __forceinline__ void copy8(V* row, int c, int d, Vec8<V> v) {
  if (c + kVec <= d) return store_full(row + c, v);
  if (c >= d) return;
  V* p = row + c;
  const int left = d - c;
  if (left & 4) {
    __builtin_memcpy(p, &v, 4 * sizeof(V));
    p += 4;
    drop(v, 4);
  }
  if (left & 2) {
    __builtin_memcpy(p, &v, 2 * sizeof(V));
    p += 2;
    drop(v, 2);
  }
  if (left & 1) __builtin_memcpy(p, &v, sizeof(V));
}

// Where a chunk's elements go one by one to the same place of another row, a chunk that load_raw
// moved back may be stored where it was loaded: its neighbour stores the same values there.
template <typename V> __device__ __forceinline__ void store_raw(V* row, int c, int d, const Vec8<V>& v) {
  if (c >= d) return;
  if (d >= kVec)
    store_full(row + min(c, d - kVec), v);
  else
    copy8(row, c, d, v);
}
// Elements of a raw chunk that are its neighbour's.
__device__ __forceinline__ int raw_overlap(int c, int d) { return d >= kVec ? max(c + kVec - d, 0) : 0; }

// Two floats to packed bf16, each to nearest even (NaN stays a NaN): one v_cvt_pk_bf16_f32.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  typedef float f32x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t v = __builtin_convertvector((f32x2_t{lo, hi}), bf16x2_t);
  uint32_t w;
  __builtin_memcpy(&w, &v, 4);
  return w;
}

__device__ __forceinline__ Vec8<bf16_t> rounded(const float (&v)[kVec], bf16_t) {
  return {u32x4_t{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])}};
}
__device__ __forceinline__ Vec8<float> rounded(const float (&v)[kVec], float) {
  return {f32x4_t{v[0], v[1], v[2], v[3]}, f32x4_t{v[4], v[5], v[6], v[7]}};
}
template <typename V> __device__ __forceinline__ void store8_raw(V* row, int c, int d, const float (&v)[kVec]) {
  store_raw(row, c, d, rounded(v, V{}));
}
template <typename V> __device__ __forceinline__ void store8(V* row, int c, int d, const float (&v)[kVec]) {
  copy8(row, c, d, rounded(v, V{}));
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

}  // namespace sfl
