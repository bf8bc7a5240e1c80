// Loads to LDS right behind what their addresses come from, and among the compiler's own: built
// to assembly only.
#include "product.hpp"

using namespace gg;

typedef __attribute__((address_space(3))) void lds_void;

// The base comes from lanes' registers just before.
extern "C" __global__ void base_from_lanes(const uint64_t* p, int* out) {
  __shared__ int lds[256];
  const uint64_t at = p[threadIdx.x];
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at),
                 hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
  load_to_lds16((const char*)((uint64_t)hi << 32 | lo), threadIdx.x * 16, lds_at(lds));
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  out[threadIdx.x] = lds[threadIdx.x];
}

// The compiler's loads to one place of LDS, with others between them.
template <int KIND>
__device__ void between(const char* p, int* out) {
  __shared__ int lds[1024];
  const auto own = [&] {
    __builtin_amdgcn_global_load_lds((const GG_GLOBAL void*)(p + threadIdx.x * 4), (lds_void*)(lds + 512), 4, 0, 0);
  };
  own();
  if (KIND == 0) load_to_lds16(p, threadIdx.x * 16, lds_at(lds));
  if (KIND == 1) load_to_lds16_at(p + threadIdx.x * 16, lds_at(lds));
  if (KIND == 2) load_to_lds4(p + threadIdx.x * 4, lds_at(lds));
  own();
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  out[threadIdx.x] = lds[threadIdx.x + 512];
}
extern "C" __global__ void m0_16(const char* p, int* out) { between<0>(p, out); }
extern "C" __global__ void m0_16_at(const char* p, int* out) { between<1>(p, out); }
extern "C" __global__ void m0_4(const char* p, int* out) { between<2>(p, out); }
