// Loads from global memory straight into LDS, and the order of what follows them.
#pragma once

#include "ra_device.h"

namespace ra {

// 16 bytes a lane from global memory (base + the lane's byte offset) to LDS, lane l's at
// `lds` + 16 l; base and lds are the wave's. In assembly: behind the builtin the compiler
// waits for all such loads before any LDS read; here await_loads() does, before the
// barrier that hands the tile over.
__device__ __forceinline__ void load_to_lds(const uint16_t *base, uint32_t offset, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(offset), "s"(base)
      : "memory", "m0");
}
__device__ __forceinline__ void await_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// The same for loads with kStores stores issued behind them (counted in order): the stores
// may still be on their way.
template <int kStores>
__device__ __forceinline__ void await_loads_before() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kStores) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const uint16_t *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// Nothing moves across: reads placed before a group of products are issued before it.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

}  // namespace ra
