// What the product of 8-bit rows and its gradient share: loads from memory to LDS.
#pragma once

#include <type_traits>

#include "codes.hpp"
#include "tiles.hpp"

namespace gg {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16 v2bf __attribute__((ext_vector_type(2)));
typedef bf16 v8bf __attribute__((ext_vector_type(8)));

// A wave's 64 lanes' pieces of 16 bytes, or words, from base + off to consecutive places of LDS
// at byte `to`.  Written out, since before the next read of LDS the compiler waits for all such
// loads that it knows of; these are waited for by their number.  They write no register but m0,
// which is an output so that the compiler knows (as a clobber it is warned of).  A base that a
// vector instruction wrote may be read five wait states later, which the compiler does not see
// to in here: s_mov and s_nop 3 are five.  (The weights' gradient of 16,384 rows, 4,096 x 8,192
// 913 us, with two states 910; the product the same.)
__device__ __forceinline__ void load_to_lds16(const char* base, uint32_t off, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 3\n\tglobal_load_lds_dwordx4 %2, %3"
               : "=&{m0}"(m0)
               : "s"(to), "v"(off), "s"(base)
               : "memory");
}
__device__ __forceinline__ void load_to_lds16_at(const char* p, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off"
               : "=&{m0}"(m0)
               : "s"(to), "v"(p)
               : "memory");
}
__device__ __forceinline__ void load_to_lds4(const char* p, uint32_t to) {
  uint32_t m0;
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %2, off"
               : "=&{m0}"(m0)
               : "s"(to), "v"(p)
               : "memory");
}
__device__ __forceinline__ uint32_t lds_at(const void* p) {
  return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

}  // namespace gg
