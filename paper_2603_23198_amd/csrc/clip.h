// The coefficient of clipping by a global norm.
#pragma once

#include "common.h"

namespace sfl {

// Whether fp32 holds the norm; where it does not, nothing is scaled and no step is taken.
__device__ __forceinline__ bool norm_is_finite(double norm) { return (float)norm < INFINITY; }

__device__ __forceinline__ double clip_coefficient(double norm, double max_norm) {
  return norm > max_norm && norm_is_finite(norm) ? max_norm / norm : 1.0;
}

// A clipping coefficient, by 2^exp. exp is 0 where by alone is a normal fp32 number: a subnormal one has
// fewer bits than the gradients (max_norm = 1e-3 of a norm of 3e38: 1e-4 off), and a smaller one is 0.
struct Scale {
  float by;
  int exp;
  __device__ __forceinline__ Scale(double c) : by((float)c), exp(0) {
    if (c > 0 && c < 0x1p-126) by = (float)frexp(c, &exp);
  }
  __device__ __forceinline__ float operator()(float g) const { return ldexpf(g * by, exp); }
};

}  // namespace sfl
