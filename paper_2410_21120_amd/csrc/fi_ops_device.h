// Device-side helpers that the decoder operators' kernels share: direct loads to LDS, and the waits for them.
#pragma once

#include "fi_device.h"

namespace fi {

// One direct load: the active lanes' N bytes (1 and 2: as a dword) at `from` go to at + max(N, 4) * lane (at: the same for the wave).  In assembler, which has
// no output register: the compiler knows nothing of the load, so it puts no wait of its own before other reads of LDS (it does before transposed ones,
// whose tile it cannot tell from the one under way); every wait is written out in the kernels.
// (The low word of a pointer into LDS is its offset there.  m0 is the compiler's for such instructions only, and it sets it before each of its own.)
template <int N>
__device__ __forceinline__ void load_lds_from(const void* from, uint8_t* at) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)at);
  if constexpr (N == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(m0), "v"(from) : "memory");
  else if constexpr (N == 4) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(m0), "v"(from) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, off" ::"s"(m0), "v"(from) : "memory");
}

// The same from a base that the wave shares, at a lane's offset in bytes (unsigned, 32 bits).  The waits: a scalar register that the vector unit wrote may be read
// by a load five instructions later.
template <int N>
__device__ __forceinline__ void load_lds_off(const void* base, uint32_t off, uint8_t* at) {
  const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)at);
  const uint32_t low = __builtin_amdgcn_readfirstlane((uint32_t)(uint64_t)base), high = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)base >> 32));
  const uint64_t shared = (uint64_t)high << 32 | low;
  if constexpr (N == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(m0), "v"(off), "s"(shared) : "memory");
  else if constexpr (N == 4) asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dword %1, %2" ::"s"(m0), "v"(off), "s"(shared) : "memory");
  else if constexpr (N == 2) asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_ushort %1, %2" ::"s"(m0), "v"(off), "s"(shared) : "memory");
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_ubyte %1, %2" ::"s"(m0), "v"(off), "s"(shared) : "memory");
}

// This wave's direct loads have arrived and its reads are done; behind the barrier that holds for all waves.
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void meet() {
  arrived();
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
template <int LATER>
__device__ __forceinline__ void arrived_but() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory"); }   // but for the LATER last loads
// The same, with the `LATER` last loads still in flight.
template <int LATER>
__device__ __forceinline__ void meet_but() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// The same for what the waves wrote to LDS themselves; loads stay in flight.
__device__ __forceinline__ void meet_lds() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

}  // namespace fi
