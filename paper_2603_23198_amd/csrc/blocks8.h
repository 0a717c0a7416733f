// Numbers in 8 bits on the device: e4m3 codes and a power of two for each block of 128; runs of tokens
// in whole blocks.
#pragma once

#include "common.h"
#include "routed.h"

namespace sfl {

// |x| as bits that order like the reals, 0 for an element that is not finite: the largest one of a
// block decides its scale.
__device__ __forceinline__ uint32_t magnitude8(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
  return u < 0x7f800000u ? u : 0u;
}

// The scale byte (exponent + 127) for a largest magnitude with these bits: 448 = 1.75 * 2^8, so the
// exponent is that of the magnitude less 8, and one more for a mantissa above 1.75. 0 gives 2^0;
// magnitudes whose scale would be below 2^-127 take that.
__device__ __forceinline__ int scale_byte8(uint32_t top) {
  if (top == 0) return 127;
  const int b = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);
  return max(b, 0);
}

// 2^(127 - byte), 2^(byte - 127)
__device__ __forceinline__ float inverse8(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }
__device__ __forceinline__ float scale8(int byte) {
  return __uint_as_float(byte > 0 ? (uint32_t)byte << 23 : 1u << 22);
}

// Four codes: halves to even. The scaled magnitudes of finite elements end at 448; an infinity, which e4m3 does
// not have, becomes NaN like a NaN.
__device__ __forceinline__ uint32_t codes8(float a, float b, float c, float d) {
  const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// A unit of a run: `count` rows from `first` on, all of one expert. expert < 0: there is no such unit.
struct Unit {
  int expert, first, count;
};

__device__ __forceinline__ int offset8(const int32_t* offsets, int e, int rows) { return min(max(offsets[e], 0), rows); }

// Unit `index` when every run takes whole units of `size` rows, found by one wave: a lane counts the
// units of its experts. Offsets are held to [0, rows], a run that descends has no rows.
__device__ __forceinline__ Unit unit_of(const int32_t* __restrict__ offsets, int E, int rows, int size, int index) {
  Unit u{-1, 0, 0};
  if (!offsets) {
    if ((int64_t)index * size < rows) {
      u.expert = 0;
      u.first = index * size;
      u.count = min(size, rows - u.first);
    }
    return u;
  }
  const int lane = lane_id(), per = (E + kWave - 1) / kWave, e0 = min(lane * per, E), e1 = min(e0 + per, E);
  const int first0 = offset8(offsets, e0, rows);
  int mine = 0, at = first0, end0 = first0;  // the lane's first run is first0 .. end0
  for (int e = e0; e < e1; ++e) {
    const int end = offset8(offsets, e + 1, rows);
    mine += (max(end - at, 0) + size - 1) / size;
    if (e == e0) end0 = end;
    at = end;
  }
  const int incl = wave_incl_scan(mine);
  const uint64_t past = ballot(incl > index);
  if (past == 0) return u;
  const int l = __builtin_ctzll(past);
  int before = readlane_i(incl - mine, l), first = readlane_i(first0, l), end = readlane_i(end0, l);
  for (int e = l * per;;) {
    const int n = (max(end - first, 0) + size - 1) / size;
    if (index < before + n) {
      u.expert = e;
      u.first = first + (index - before) * size;
      u.count = min(size, end - u.first);
      return u;
    }
    before += n;
    if (++e >= E) return u;
    first = end;
    end = offset8(offsets, e + 1, rows);
  }
}

}  // namespace sfl
