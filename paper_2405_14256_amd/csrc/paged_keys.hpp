// Keys in pages: where 16 of them lie, how many of them a unit of work reads, their way to LDS.  (16 consecutive keys lie in one page, so
// all of this is scalar work.)
#pragma once

#include "mfma_tiles.hpp"

namespace zc {

// The page of 16 keys from key0 on, of a row of the table (past its end: any, no key is read).
__device__ inline int page_of(const int32_t* row, int cols, int shift, int key0) {
  typedef __attribute__((address_space(4))) const int32_t* scalar;
  return ((scalar)(uintptr_t)row)[min(key0 >> shift, cols - 1)];
}
// Of 16 keys from key0 on, how many a unit reads: none of a missing page, of those that no row's window reaches, from `end` on.
// What is not read arrives as zeros.  (behind: 16 keys from key0 on are behind every window of the unit's if key0 - sinks, without sign, is less.)
__device__ inline int keys_read(int n_pages, int sinks, uint32_t behind, int end, int key0, int id) {
  int n = max(end - key0, 0);
  asm("" : "+s"(n));                                       // (both bounds at once would be a vector instruction, and what follows too)
  n = min(n, 16);
  if ((uint32_t)id >= (uint32_t)n_pages) n = 0;
  if ((uint32_t)(key0 - sinks) < behind) n = 0;
  return n;
}
// Where they are (of no keys: anywhere, nothing is read).
__device__ inline __amdgpu_buffer_rsrc_t keys_at(int shift, const uint8_t* head, uint32_t sB, uint32_t row, int key0, int id, int n) {
  const uint64_t at = (uint64_t)(uint32_t)id * sB + ((uint32_t)key0 & ((1u << shift) - 1)) * row;
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(head + at), 0, n * row, kBufFlags);
}

// 16 keys to LDS in N transfers of 1024 bytes, to consecutive places.  The descriptor changes with every page, and the compiler may have
// brought a part of it (or the place) from a vector register the instruction before: a memory instruction must not read
// such a scalar register for five wait states, and does not see that it does inside an assembly block.
#define ZC_KEYS_NEXT(v) "s_add_u32 m0, m0, 0x400\n\ts_nop 0\n\tbuffer_load_dwordx4 " v ", %1, 0 offen lds\n\t"
#define ZC_KEYS_FIRST "s_nop 4\n\ts_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %1, 0 offen lds\n\t"
template <int N>
__device__ inline void move_keys(uint32_t lds, __amdgpu_buffer_rsrc_t rs, const int (&v)[N]) {
  static_assert(N == 2 || N == 4 || N == 8, "16 rows of 128, 256 or 512 bytes");
  if constexpr (N == 2)
    asm volatile(ZC_KEYS_FIRST ZC_KEYS_NEXT("%3") :: "s"(lds), "s"(rs), "v"(v[0]), "v"(v[1]) : "memory", "scc");
  else if constexpr (N == 4)
    asm volatile(ZC_KEYS_FIRST ZC_KEYS_NEXT("%3") ZC_KEYS_NEXT("%4") ZC_KEYS_NEXT("%5")
                 :: "s"(lds), "s"(rs), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]) : "memory", "scc");
  else
    asm volatile(ZC_KEYS_FIRST ZC_KEYS_NEXT("%3") ZC_KEYS_NEXT("%4") ZC_KEYS_NEXT("%5") ZC_KEYS_NEXT("%6") ZC_KEYS_NEXT("%7") ZC_KEYS_NEXT("%8") ZC_KEYS_NEXT("%9")
                 :: "s"(lds), "s"(rs), "v"(v[0]), "v"(v[1]), "v"(v[2]), "v"(v[3]), "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]) : "memory", "scc");
}
#undef ZC_KEYS_NEXT
#undef ZC_KEYS_FIRST

}  // namespace zc
