// Loads from global memory straight into LDS, their hand-counted waits, and the
// placement of key rows in LDS: what the paged attention kernels share.
#pragma once
#include "device_common.h"

namespace adaserve {

typedef __attribute__((address_space(3))) char lds_char;

// LDS byte address of a __shared__ object (what M0 takes).
__device__ __forceinline__ uint32_t lds_addr(const void *p) {
  return (uint32_t)(uintptr_t)(const lds_char *)p;
}

// 16-byte loads from global memory straight into LDS (global_load_lds):
// lane l writes LDS bytes [lds + 16 l, +16).  Written as asm so that the
// compiler does not try to track these loads itself (it cannot follow a
// ring of stages across the loop and would wait for every load in flight
// before each LDS read); the "memory" clobber keeps every LDS access in
// program order around them, and the waits below are counted by hand.
// Setting M0 needs one wait state before the load that reads it.  The
// compiler reserves M0 and warns about the clobber; nothing else in this
// library uses M0 (LDS instructions on gfx950 do not read it).
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// With NT the loads carry the non-temporal hint: used when every K/V byte of
// the launch is read by one workgroup only (single-tile requests), so the
// lines are not kept for a reuse that never comes (measured 3-6% faster on
// a 1 GB long-context batch, 6% slower where row tiles share a chunk).
template <bool NT>
__device__ __forceinline__ void dma16(const void *src, uint32_t lds) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off nt"
                 :: "v"(src), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 :: "v"(src), "s"(lds) : "memory", "m0");
}
// Same with a wave-uniform base address and a 32-bit per-lane offset.
template <bool NT>
__device__ __forceinline__ void dma16_off(const void *base, uint32_t off, uint32_t lds) {
  if constexpr (NT)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
                 :: "v"(off), "s"(base), "s"(lds) : "memory", "m0");
  else
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
#pragma clang diagnostic pop

// s_waitcnt vmcnt(N) with the other counters left open (for loads the
// compiler issued itself).
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 16, "vmcnt immediate");
  __builtin_amdgcn_s_waitcnt(0xF70 | N);
}

// Waits until at most N of this wave's loads are in flight and its LDS
// operations are done, then the workgroup barrier.  No memory access moves
// across it.
template <int N>
__device__ __forceinline__ void wait_loads_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt immediate");
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(N) : "memory");
}

// 16-byte chunk permutation of LDS row `row`: chunk c of the row is stored in
// slot c ^ swizzle(row).  Any 16 consecutive rows keep one chunk in 16
// distinct places (K reads); rows 4k .. 4k+3 keep four neighbouring chunks in
// 16 distinct places (V reads).
template <int NCH>
__device__ __forceinline__ int swizzle(int row) {
  if (NCH == 16) return ((row & 3) << 2) | ((row >> 2) & 3);
  return ((row & 2) << 1) | ((row >> 2) & 3);
}

}  // namespace adaserve
