// What the product kernels that go through LDS share: loads that need no registers, and the barriers that wait for them.
#pragma once

#include "product.h"

#if defined(__HIPCC__)
namespace qgtc {

// Wave-wide loads straight to LDS address `to` (+ 16 or 4 bytes per lane); assembly because the compiler would make every later
// read of LDS wait for them.  What lies behind the buffer's end is not read (LDS gets zeros).  The scalar offset is held to the
// buffer's size: the unit compares the lane's offset with size - scalar offset, which must not wrap.
__device__ __forceinline__ void load16_lds(const v4i& rsrc, uint32_t voff, uint32_t soff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
               :: "v"(voff), "s"(rsrc), "s"(min(soff, (uint32_t)rsrc[2])), "s"(to) : "m0");
}
__device__ __forceinline__ void load4_lds(const v4i& rsrc, uint32_t voff, uint32_t soff, uint32_t to) {
  asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dword %0, %1, %2 offen lds"
               :: "v"(voff), "s"(rsrc), "s"(min(soff, (uint32_t)rsrc[2])), "s"(to) : "m0");
}
__device__ __forceinline__ uint32_t scalar(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ v4i buffer_of(const void* base, uint32_t bytes) {
  const uint64_t b = (uint64_t)base;
  return (v4i){(int)scalar((uint32_t)b), (int)scalar((uint32_t)(b >> 32)), (int)scalar(bytes), 0x00020000};
}

// What this wave has asked of LDS has come, and of memory all but the last LATER loads; then every wave's.
template <int LATER>
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LATER) : "memory");
}

__device__ __forceinline__ void meet_lds() {       // LDS alone: loads and stores stay on their way
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

}  // namespace qgtc
#endif  // __HIPCC__
