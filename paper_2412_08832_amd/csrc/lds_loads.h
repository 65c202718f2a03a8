// lds_loads.h -- loads from global memory straight to LDS, and the waits for them.
#ifndef HADACORE_LDS_LOADS_H
#define HADACORE_LDS_LOADS_H

#include <hip/hip_runtime.h>

#include <stdint.h>

namespace hadacore {
namespace {

typedef uint32_t lds_buffer __attribute__((ext_vector_type(4)));

// Asynchronous loads into LDS: lane l's 16 bytes from base + offset + uniform_offset go to
// `lds` + 16 l.  In asm, because the compiler waits for all outstanding loads of this kind
// before any LDS read, which would undo the loading ahead: the kernel waits itself
// (wait_stages) before the barrier that publishes the data.  The instruction writes no
// register; the wait state is the one that it needs after a write of M0 (which no other
// instruction of these kernels uses, and which may not be named as clobbered).
// NT: with the streaming cache policy, for data that nobody reads again.
template <bool NT = false>
__device__ __forceinline__ void load_to_lds(lds_buffer base, uint32_t lds, int offset, int uniform_offset) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
                 :
                 : "s"(lds), "v"(offset), "s"(base), "s"(uniform_offset)
                 : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds), "v"(offset), "s"(base), "s"(uniform_offset)
                 : "memory");
}

// The same for one 4-byte word of each lane's own address.
__device__ __forceinline__ void load_word_to_lds(const void *from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off"
               :
               : "s"(lds), "v"(from)
               : "memory");
}

// 16 bytes of each lane's own address; the address and the LDS are multiples of 16.
__device__ __forceinline__ void load_lane_to_lds(const void *from, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(lds), "v"(from)
               : "memory");
}

// Waits until at most the loads of `ahead` later stages of `LOADS` loads are in flight,
// `ahead` being at most MOST.
template <int MOST, int LOADS>
__device__ __forceinline__ void wait_stages(int ahead) {
  if constexpr (MOST > 0) {
    if (ahead < MOST) {
      wait_stages<MOST - 1, LOADS>(ahead);
      return;
    }
  }
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(MOST * LOADS) : "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

}  // namespace
}  // namespace hadacore

#endif  // HADACORE_LDS_LOADS_H
