// LDS-direct loads, counted waits and the workgroup barrier of the tiled GEMM
// kernels (gfx950).
#pragma once

#include "pw_device.hpp"

namespace pw {
namespace {

#define PW_LDS __attribute__((address_space(3)))
typedef PW_LDS uint8_t* lds_u8_t;
__device__ __forceinline__ u32x4 lds16(lds_u8_t p) { return *reinterpret_cast<const PW_LDS u32x4*>(p); }

// ---- LDS-direct loads -------------------------------------------------------
// A wave-wide load that lands in LDS: lane l's 16 (or 4) bytes from base +
// voff go to LDS byte address `dst` + 16 l (4 l), wave-uniform base and dst.
// Written as asm because the compiler, which cannot tell what such a load
// writes, waits for all of them before any LDS access; here the waits are
// counted by hand (wait_vm). No register receives data, so nothing can be
// reallocated under a load in flight. (M0 holds the LDS address; one wait
// state between its write and the load.)
__device__ __forceinline__ void lds_load16(uint32_t dst, uint32_t voff, const uint8_t* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :: "s"(dst), "v"(voff), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void lds_load4(uint32_t dst, uint32_t voff, const uint8_t* base) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :: "s"(dst), "v"(voff), "s"(base) : "memory", "m0");
}
template <int N>
__device__ __forceinline__ void wait_vm() {
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_lds() {
  asm volatile("s_waitcnt lgkmcnt(%0)" :: "n"(N) : "memory");
}
__device__ __forceinline__ void wg_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_barrier" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ const uint8_t* uniform_ptr(const uint8_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<const uint8_t*>((static_cast<uint64_t>(hi) << 32) | lo);
}

}  // namespace
}  // namespace pw
