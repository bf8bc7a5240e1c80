// What the product of 8-bit rows, its gradient and the weights' quantiser share: tiles'
// places, and loads from memory to LDS.
#pragma once

#include <type_traits>

#include "codes.hpp"

namespace gg {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16 v2bf __attribute__((ext_vector_type(2)));
typedef bf16 v8bf __attribute__((ext_vector_type(8)));

// A tile's place: each of the 8 XCDs, which take blocks in turn, has a run of tiles,
// and in it bands of kBand tiles of rows, so that the blocks on one L2 at a time share
// rows and weights.
constexpr int32_t kXcds = 8, kBand = 4;

__device__ __forceinline__ uint32_t xcd_turn(uint32_t b, uint32_t total) {
  const uint32_t x = b % kXcds, q = total / kXcds, r = total % kXcds;
  return x * q + min(x, r) + b / kXcds;
}

__device__ __forceinline__ void tile_place(int32_t tiles_i, int32_t tiles_j, int32_t* ti, int32_t* tj) {
  const uint32_t t = xcd_turn(blockIdx.x, gridDim.x);
  const uint32_t width = kBand * tiles_j, band = t / width, first = band * kBand,
                 rows = min((uint32_t)tiles_i - first, (uint32_t)kBand), at = t - band * width;
  *ti = (int32_t)(first + at % rows);
  *tj = (int32_t)(at / rows);
}

// A wave's 64 lanes' pieces of 16 bytes, or words, from base + off to consecutive places of LDS
// at byte `to`.  Written out, since before the next read of LDS the compiler waits for all such
// loads that it knows of; these are waited for by their number.  They write no register but m0,
// which is an output so that the compiler knows (as a clobber it is warned of).  A base that a
// vector instruction wrote may be read five wait states later, which the compiler does not see
// to in here: s_mov and s_nop 3 are five.  (They cost nothing that can be measured.)
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
