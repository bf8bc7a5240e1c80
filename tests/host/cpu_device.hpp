// A .hip source as a CPU program: included before it (with clang), the words of the HIP
// language mean one lane that runs by itself, and a launch hands its blocks to `on_launch`.
// Waits for other lanes do nothing and exchanges between them give a lane its own value back,
// so that what a lane touches can be seen, not what a block computes.
#pragma once

#define __HIP_PLATFORM_AMD__ 1
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <setjmp.h>
#include <signal.h>
#include <stdint.h>
#include <string.h>
#include <sys/mman.h>

#include <algorithm>
#include <functional>
#include <utility>

#define HIP_INCLUDE_HIP_HIP_RUNTIME_H    // the language's own header is not wanted

struct Uint3 {
  unsigned x, y, z;
};
static Uint3 threadIdx, blockIdx;
static dim3 blockDim, gridDim;

#undef __global__
#undef __device__
#undef __shared__
#undef __forceinline__
#undef __launch_bounds__
#define __global__ static
#define __device__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __syncthreads()

using std::max;
using std::min;

static inline float __uint_as_float(uint32_t v) { return __builtin_bit_cast(float, v); }
static inline uint32_t __float_as_uint(float v) { return __builtin_bit_cast(uint32_t, v); }
template <typename T>
static T __shfl_xor(T v, int, int) { return v; }
template <typename T>
static T __shfl(T v, ...) { return v; }
template <typename T>
static T __shfl_up(T v, ...) { return v; }
template <typename T, typename V>
static T atomicAdd(T* p, V v) { return std::exchange(*p, *p + v); }
template <typename T, typename V>
static T atomicOr(T* p, V v) { return std::exchange(*p, *p | v); }
static inline uint64_t __ballot(bool b) { return b; }
static inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
static inline int __ffsll(uint64_t v) { return __builtin_ffsll((long long)v); }
static inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }

typedef float cpu_float2 __attribute__((ext_vector_type(2)));
#define __builtin_amdgcn_mov_dpp(v, ...) (v)
#define __builtin_amdgcn_mbcnt_lo(m, v) (v)
#define __builtin_amdgcn_mbcnt_hi(m, v) (v)
#define __builtin_amdgcn_rcpf(v) (1.0f / (v))
#define __builtin_amdgcn_perm(a, b, s) ((a) ^ (b) ^ (s))
#define __builtin_amdgcn_cvt_f32_fp8(v, i) ((float)(v))
#define __builtin_amdgcn_cvt_pk_f32_fp8(v, h) (cpu_float2{(float)(v), (float)(v)})
#define __builtin_amdgcn_cvt_pk_fp8_f32(a, b, old, h) ((int)(a) ^ (int)(b) ^ (old))

// What a launch does: each test sets it.
static std::function<void(dim3 grid, dim3 block, const std::function<void()>& lane)> on_launch;

#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) \
  on_launch(grid, block, [&] { kernel(__VA_ARGS__); })

static sigjmp_buf after_fault;
static void at_fault(int) { siglongjmp(after_fault, 1); }

// Runs a lane; whether it touched memory that may not be.
static inline bool faults(dim3 grid, dim3 block, int64_t b, unsigned t, const std::function<void()>& lane) {
  gridDim = grid;
  blockDim = block;
  blockIdx = {(unsigned)(b % grid.x), (unsigned)(b / grid.x), 0};
  threadIdx = {t, 0, 0};
  signal(SIGSEGV, at_fault);
  if (sigsetjmp(after_fault, 1)) return true;
  lane();
  return false;
}

// Addresses that nothing may touch.
static inline char* no_memory(size_t bytes) {
  void* p = mmap(nullptr, bytes, PROT_NONE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  return p == MAP_FAILED ? nullptr : (char*)p;
}
