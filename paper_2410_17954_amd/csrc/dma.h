// Loads from memory straight to LDS that the compiler does not count.
#pragma once

#include "common.h"

namespace moe {

typedef __attribute__((address_space(3))) void lds_void;

// Address of LDS memory, the same for the whole wave.
__device__ __forceinline__ uint32_t lds_address(void* p) {
  return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void*)p);
}

// Raw buffer over n rows of `width` bytes, `row` bytes apart, from row `first` of base on.
__device__ __forceinline__ u32x4_t dma_rows(const void* base, int64_t first, int n, uint32_t row,
                                            uint32_t width) {
  const uint64_t p = reinterpret_cast<uint64_t>(base) + (uint64_t)(first * row);
  return u32x4_t{(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, (uint32_t)(n - 1) * row + width,
                 0x00027000u};
}

// SIZE bytes a lane of a raw buffer into LDS: 16 at lds + 16 * lane; 4, 2 or 1 as a word at
// lds + 4 * lane. Past its end: zeros. The compiler does not see that these are on their
// way: it would wait for all of them at every transposing read. wait_loads does; loads
// that the compiler counts as well make its own waits longer, never shorter. m0 is a register
// that it reserves and keeps no value in.
template <int SIZE>
__device__ __forceinline__ void dma(uint32_t lds, uint32_t voff, u32x4_t rs) {
  if constexpr (SIZE == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(rs) : "memory");
  else if constexpr (SIZE == 4)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(rs) : "memory");
  else if constexpr (SIZE == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ushort %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(rs) : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_ubyte %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(voff), "s"(rs) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {   // until at most N are on their way
  static_assert(N < 64, "the counter's range");
  asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory");
}
// This wave's LDS accesses have been done.
__device__ __forceinline__ void wait_lds() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

}  // namespace moe
