// Loads straight to LDS.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace obf {

// Four (two) times 16 bytes per lane from base + off to LDS at `lds` + 16 lane and 4096 further each time, without registers between; complete when vmcnt
// says so.  (The builtin would have the compiler wait for the youngest of these loads before every read of LDS.)  m0 is left as it was: the compiler
// reserves it and would not be told by a clobber.
__device__ __forceinline__ void load_to_lds(const uint32_t lds, const uint32_t (&off)[4], const void* base) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %6\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %6\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, %6\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, %6\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(lds), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base) : "memory", "scc");
}
__device__ __forceinline__ void load_to_lds(const uint32_t lds, const uint32_t (&off)[2], const void* base) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %4\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %4\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(lds), "v"(off[0]), "v"(off[1]), "s"(base) : "memory", "scc");
}
// The same from an address per lane and load.
__device__ __forceinline__ void load_to_lds(const uint32_t lds, const void* const (&from)[4]) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, off\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, off\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, off\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(lds), "v"(from[0]), "v"(from[1]), "v"(from[2]), "v"(from[3]) : "memory", "scc");
}
__device__ __forceinline__ void load_to_lds(const uint32_t lds, const void* const (&from)[2]) {
  uint32_t m0;
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\t"
               "s_add_u32 m0, m0, 0x1000\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, off\n\ts_mov_b32 m0, %0"
               : "=&s"(m0) : "s"(lds), "v"(from[0]), "v"(from[1]) : "memory", "scc");
}
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

}  // namespace obf
