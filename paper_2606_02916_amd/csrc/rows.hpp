// Rows of typed elements: host-side checks of gg_rows_t, and the device code
// that moves pieces of rows between memory and fp32 registers.
#pragma once

#include "gg_host.hpp"

namespace gg {

// A matrix of rows, passed by value: row r's elements at p + r * stride.
struct KRows {
  char* p;
  int64_t stride;
  char* scales;      // 8-bit rows: fp32 scales of row r at scales + r * sstride
  int64_t sstride;
  int32_t group;     // elements per scale; 0: one scale per row
};

constexpr uint32_t kBitF32 = 1u << GG_F32, kBitF16 = 1u << GG_F16, kBitBF16 = 1u << GG_BF16,
                   kBitE4M3 = 1u << GG_E4M3;
constexpr uint32_t kBitFloats = kBitF32 | kBitF16 | kBitBF16;

inline int64_t elem_bytes(int32_t dtype) {
  return dtype == GG_F32 ? 4 : dtype == GG_E4M3 ? 1 : 2;
}

// Checks n rows of dim elements and packs them.  `types`: the accepted
// dtypes; `written`: the rows are an output (and may not overlap).
int pack_rows(const gg_rows_t* r, const char* name, int64_t n, int64_t dim, uint32_t types,
              bool written, KRows* out);

// ---------------------------------------------------------------------------
// Element types.  Everything is computed in fp32; a store rounds once, to
// nearest even.
// ---------------------------------------------------------------------------
struct e4m3 {
  uint8_t b;
};
typedef __bf16 bf16;
typedef _Float16 f16;

// Elements of a 16-byte access: the width of a lane's piece of a row.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// Accesses are aligned to the element only: gfx950 takes 16-byte global
// accesses at any byte address.
template <typename T, int V>
struct Raw {
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef vec mem __attribute__((aligned(sizeof(T))));
};
template <int V>
struct Raw<e4m3, V> {
  typedef uint8_t vec __attribute__((ext_vector_type(V)));
  typedef vec mem __attribute__((aligned(1)));
};
template <typename T>
struct Raw<T, 1> {
  typedef T vec;
  typedef T mem;
};
template <>
struct Raw<e4m3, 1> {
  typedef uint8_t vec;
  typedef uint8_t mem;
};

template <typename T, int V>
__device__ __forceinline__ typename Raw<T, V>::vec raw_load(const char* p) {
  return *(const GG_GLOBAL typename Raw<T, V>::mem*)p;
}

template <typename T, int V>
__device__ __forceinline__ void to_f32(typename Raw<T, V>::vec r, float (&v)[V]) {
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 1)
      v[0] = __builtin_amdgcn_cvt_f32_fp8((int)r, 0);
    else
      v[0] = (float)r;
  } else if constexpr (sizeof(T) == 1) {
    static_assert(V % 4 == 0, "whole words of codes");
    union {
      typename Raw<T, V>::vec r;
      uint32_t w[V / 4];
    } u;
    u.r = r;
#pragma unroll
    for (int i = 0; i < V / 4; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.w[i], false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)u.w[i], true);
      v[4 * i] = lo[0];
      v[4 * i + 1] = lo[1];
      v[4 * i + 2] = hi[0];
      v[4 * i + 3] = hi[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)r[i];
  }
}

template <typename T, int V>
__device__ __forceinline__ void row_load(const char* p, float (&v)[V]) {
  to_f32<T, V>(raw_load<T, V>(p), v);
}

// Codes of four values that lie within +-448.
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// Outputs of more bytes than this are stored past the caches: they would push
// out what the call reads, and the next kernel would find no more than their
// end.  (67 MB rows looked up, normed and multiplied: 124 us with plain stores,
// 111 this way; 17 MB, which the caches hold: 34 and 37 through a norm's
// forward and backward call.)
constexpr int64_t kStreamBytes = 32 << 20;

template <typename V, typename M>
__device__ __forceinline__ void put(GG_GLOBAL M* p, V v, bool stream) {
  if (stream) {
    // (the empty statements keep the compiler from merging both stores into
    // a plain one)
    asm volatile("");
    __builtin_nontemporal_store(v, p);
    asm volatile("");
  } else {
    *p = v;
  }
}

template <typename T, int V>
__device__ __forceinline__ void row_store(char* p, const float (&v)[V], bool stream = false) {
  typedef typename Raw<T, V>::mem mem;
  GG_GLOBAL mem* to = (GG_GLOBAL mem*)p;
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 1)
      *to = (uint8_t)to_codes(v[0], 0.f, 0.f, 0.f);
    else
      *to = (T)v[0];
  } else if constexpr (sizeof(T) == 1) {
    union {
      typename Raw<T, V>::vec r;
      uint32_t w[V / 4];
    } u;
#pragma unroll
    for (int i = 0; i < V / 4; ++i)
      u.w[i] = to_codes(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
    put(to, u.r, stream);
  } else {
    typename Raw<T, V>::vec r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)v[i];
    put(to, r, stream);
  }
}

// A row is cut into pieces of V elements; the last one starts at dim - V and
// overlaps the one before (dim >= V), so that no lane has a shorter piece.
// skip: leading elements of piece p that belong to the piece before.
template <int V>
__device__ __forceinline__ int32_t piece_start(int32_t p, int32_t dim, int32_t* skip) {
  const int32_t at = p * V, e = at < dim - V ? at : dim - V;
  *skip = at - e;
  return e;
}

// Reductions over groups of `lanes` lanes of a wave (a power of two), the
// result in every lane: neighbours by DPP, which costs an operand, up to 16
// lanes, shuffles beyond.  Every lane of a group must call it.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(v), CTRL, 0xf, 0xf,
                                                            true));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xf, 0xf, true);
}

template <typename T, typename F>
__device__ __forceinline__ T lanes_reduce(T v, int lanes, F f) {
  if (lanes >= 2) v = f(v, dpp<0xB1>(v));      // quad_perm 1,0,3,2
  if (lanes >= 4) v = f(v, dpp<0x4E>(v));      // quad_perm 2,3,0,1
  if (lanes >= 8) v = f(v, dpp<0x141>(v));     // row_half_mirror: the other quad
  if (lanes >= 16) v = f(v, dpp<0x140>(v));    // row_mirror: the other eight
  if (lanes >= 32) v = f(v, __shfl_xor(v, 16, kWave));
  if (lanes >= 64) v = f(v, __shfl_xor(v, 32, kWave));
  return v;
}

__device__ __forceinline__ float lanes_sum(float v, int lanes) {
  return lanes_reduce(v, lanes, [](float x, float y) { return x + y; });
}
__device__ __forceinline__ float lanes_maxf(float v, int lanes) {
  return lanes_reduce(v, lanes, [](float x, float y) { return fmaxf(x, y); });
}
// Of magnitudes as bits: a NaN is more than every number.
__device__ __forceinline__ uint32_t lanes_max(uint32_t v, int lanes) {
  return lanes_reduce(v, lanes, [](uint32_t x, uint32_t y) { return max(x, y); });
}

// A launch of `blocks` blocks: one dimension holds fewer than 2^32 lanes.
constexpr int64_t kGridX = 1 << 21;

inline dim3 grid_of(int64_t blocks) {
  return dim3((unsigned)std::min(blocks, kGridX), (unsigned)cdiv(blocks, kGridX));
}

__device__ __forceinline__ int64_t block_index() {
  return (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
}

// Runs the statements with T as the dtype's element type.
#define GG_FOR_FLOAT(dtype, T, ...)      \
  do {                                   \
    if ((dtype) == GG_F32) {             \
      typedef float T;                   \
      __VA_ARGS__;                       \
    } else if ((dtype) == GG_F16) {      \
      typedef ::gg::f16 T;               \
      __VA_ARGS__;                       \
    } else {                             \
      typedef ::gg::bf16 T;              \
      __VA_ARGS__;                       \
    }                                    \
  } while (0)

}  // namespace gg
