// Numbers in the order of the reals as unsigned keys, and the largest key of lanes.
#pragma once

#include "common.h"

namespace sfl {

// A number's place in the order of the reals: larger number, larger key; 0 for one that stands for nothing (-inf or
// NaN). -0 and +0 have one key.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (!(x > -INFINITY)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t key) {
  return __uint_as_float((key & 0x80000000u) ? (key & 0x7fffffffu) : ~key);
}

template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false));
}

// Largest value of aligned groups of G lanes, in every lane (lanes trade as in group_sum).
template <int G> __device__ __forceinline__ uint32_t group_max(uint32_t v) {
  if (G >= 2) v = dpp_max<0xB1>(v);
  if (G >= 4) v = dpp_max<0x4E>(v);
  if (G >= 8) v = dpp_max<0x141>(v);
  if (G >= 16) v = dpp_max<0x140>(v);
  if (G == 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16, 64));
  if (G == 64)
    v = max(max((uint32_t)readlane_i((int)v, 0), (uint32_t)readlane_i((int)v, 16)),
            max((uint32_t)readlane_i((int)v, 32), (uint32_t)readlane_i((int)v, 48)));
  return v;
}

}  // namespace sfl
