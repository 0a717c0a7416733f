// Launch interfaces of the operators for many routed experts in 8 bits (route_groups.hip, quant.hip,
// product8.hip, adamw.hip); api_routed.cpp checks the arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/sfl.h"

namespace sfl {

constexpr int kRouteGroupsExperts = 1024;
hipError_t launch_route_groups_fwd(const sfl_route_groups_args_t& a, hipStream_t s);
hipError_t launch_route_groups_bwd(const sfl_route_groups_bwd_args_t& a, hipStream_t s);

// --------------------------------------------------------------- numbers in 8 bits ----
constexpr int kBlock8 = 128;           // elements that share a scale
constexpr int kMaxExperts8 = 1024;
constexpr int64_t kMaxWidth8 = 1 << 20;
constexpr int64_t kMaxColumns8 = 1 << 22;  // of a product: 256 rows of them lie within 32-bit offsets

constexpr int64_t up(int64_t n, int64_t m) { return (n + m - 1) / m * m; }
constexpr int64_t blocks8(int64_t n) { return (n + kBlock8 - 1) / kBlock8; }
// Bytes of a row of scales: a whole four of blocks.
constexpr int64_t scale_row8(int64_t n) { return up(blocks8(n), 4); }
// Columns that hold the runs of any E experts with T tokens in all: a run of n takes up(n, 128), of
// at most min(E, T) runs that are not empty.
constexpr int64_t columns8(int64_t T, int64_t E) { return up(T / kBlock8 * kBlock8 + kBlock8 * (E < T ? E : T), 512); }

hipError_t launch_quant_rows(const sfl_quant_args_t& a, hipStream_t s);
hipError_t launch_quant_weights(const void* W, int bf16, int64_t E, int64_t R, int64_t C, uint8_t* Q, uint8_t* S,
                                uint8_t* Qt, uint8_t* St, hipStream_t s);

struct Product8 {
  const uint8_t* A;  // rows of the result: [rows][K], or [N][columns] for the weights' gradients
  const uint8_t* As;
  const uint8_t* B;  // its columns: [E][N][K], or [K][columns]
  const uint8_t* Bs;
  void* C;
  const int32_t* offsets;  // null: one expert of all rows
  int64_t rows, N, K, columns;
  int E;
};
hipError_t launch_product8(const Product8& p, int32_t dtype, hipStream_t s);
hipError_t launch_product8_weights(const Product8& p, int32_t dtype, hipStream_t s);

hipError_t launch_adamw(const sfl_adamw_t* list, int n, const sfl_adamw_cfg_t& cfg, hipStream_t s);

}  // namespace sfl
