// Loads from a buffer straight into LDS, and the compute units of the device.
#pragma once

#include <atomic>

#include "common.h"

namespace sfl {

constexpr uint32_t kOOB = 0x80000000u;  // an offset that is always out of range

// The four descriptor words of a raw buffer resource, for inline assembly operands.
__device__ __forceinline__ u32x4_t rsrc_words(const void* base, int64_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)base;
  const uint32_t n = bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes;
  u32x4_t w;
  w[0] = __builtin_amdgcn_readfirstlane((uint32_t)a);
  w[1] = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu);  // stride 0
  w[2] = n;
  w[3] = 0x00020000u;
  return w;
}

// 16 bytes per lane from a buffer straight into LDS at lds_off + 16 * lane. Written as
// inline assembly: the compiler does not count these loads and so does not make every
// later LDS read wait for all of them; the K loop waits for them itself (s_waitcnt vmcnt)
// and orders them with barriers. Counting stays safe for the compiler's own loads: loads
// complete in order, so extra loads in flight only make its waits stricter.
__device__ __forceinline__ void load_lds16(u32x4_t rsrc, uint32_t lds_off, uint32_t voff, uint32_t soff) {
  asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds"
               :
               : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds_off)
               : "memory");
}
// The same, and for 4 bytes per lane, where a scalar operand may have been written by a vector instruction right
// before: the memory instruction may read it five wait states later at the earliest, and the compiler, which
// does that for its own loads, does not look into inline assembly. (Spilled scalars come back by v_readlane.)
__device__ __forceinline__ void load_lds16_settled(u32x4_t rsrc, uint32_t lds_off, uint32_t voff, uint32_t soff) {
  asm volatile("s_nop 4\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
               :
               : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds_off)
               : "memory");
}
__device__ __forceinline__ void load_lds4_settled(u32x4_t rsrc, uint32_t lds_off, uint32_t voff, uint32_t soff) {
  asm volatile("s_nop 4\n\tbuffer_load_dword %0, %1, %2 offen lds"
               :
               : "v"(voff), "s"(rsrc), "s"(soff), "{m0}"(lds_off)
               : "memory");
}

// Compute units of the current device (cached per device; threads that race on the first
// query store the same value).
inline int device_cus() {
  static std::atomic<int> cus[64];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  int n = cus[dev].load(std::memory_order_relaxed);
  if (n <= 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cus[dev].store(n, std::memory_order_relaxed);
  }
  return n;
}

}  // namespace sfl
