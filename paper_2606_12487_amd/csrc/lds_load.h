// Direct loads from global memory into LDS, a wavefront at a time: lane l's 16
// (or 4) bytes come from base + voff and go to LDS byte lds_off + 16 * l (4 * l).
// base and lds_off are uniform over the wavefront, voff is the lane's own.
//
// As asm, so that the compiler does not drain the loads before every LDS read:
// it cannot tell the buffers of a ring apart.  The callers wait for the loads
// they need (vmcnt), and a barrier follows where other wavefronts read them.
//
// The load takes the LDS base from M0, and a scalar write of M0 needs one wait
// state before it: the s_nop.  The compiler inserts none inside an asm statement.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dptq {

__device__ __forceinline__ void load_lds16(const void* base, uint32_t voff, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(voff), "s"(base), "s"(lds_off)
               : "memory", "m0");
}

// The same to lds_base + OFF, formed in M0 by one scalar add.
template <uint32_t OFF>
__device__ __forceinline__ void load_lds16_at(const void* base, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(voff), "s"(base), "s"(lds_base), "i"(OFF)
               : "memory", "m0", "scc");
}

__device__ __forceinline__ void load_lds4(const void* base, uint32_t voff, uint32_t lds_off) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(voff), "s"(base), "s"(lds_off)
               : "memory", "m0");
}

}  // namespace dptq
