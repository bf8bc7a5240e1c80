// 8-bit rows: the scale of a group of elements, and their codes.
#pragma once

#include "rows.hpp"

namespace gg {

constexpr float kE4M3Max = 448.0f;
constexpr float kScaleMin = 1.17549435e-38f;   // 2^-126
constexpr float kLargest = 3.4028235e38f;

// Weights in 8 bits, passed by value: row r's codes at p + r * stride, the scale of
// its columns 128 c .. 128 c + 127 at scales + r / 128 * sstride + 4 c.
struct KBlocks {
  char* p;
  int64_t stride;
  char* scales;
  int64_t sstride;
};

constexpr int32_t kScaleBlock = GG_SCALE_BLOCK;

// Checks [rows][cols] weights in 8 bits and packs them.
int pack_blocks(const gg_blocks_t* b, const char* name, int64_t rows, int64_t cols, bool written,
                KBlocks* out);

// Largest magnitude, as bits, of a piece's own elements: only a row's last
// piece has others (skip > 0).
template <int V>
__device__ __forceinline__ uint32_t magnitude(const float (&v)[V], int32_t skip) {
  uint32_t m = 0;
  if (skip == 0) {
#pragma unroll
    for (int k = 0; k < V; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) m = max(m, k >= skip ? __float_as_uint(v[k]) & 0x7fffffffu : 0u);
  }
  return m;
}

// max / 448 rounded as a division, and the least scale; a NaN or an infinity stays.
__device__ __forceinline__ float scale_of(float m) {
  constexpr float kInv = 1.0f / kE4M3Max;
  const float q = m * kInv;
  const float scale = __builtin_fmaf(__builtin_fmaf(-fminf(q, kLargest), kE4M3Max, m), kInv, q);
  return scale < kScaleMin ? kScaleMin : scale;
}

// The codes of a group are the quotients by its scale, by a reciprocal in two
// parts: at one operation an element more than a product with its first part, which
// is a unit off and now and then another code (233,000 rows of 602 fp32 in groups of 64
// normed 137 us so, 144 this way, a quarter more divided outright).  Of all pairs of an
// element and a group's largest one in bf16 and fp16 none has another quotient than the
// division's, whichever way the reciprocal is rounded.  (A zero may lose its sign.)
struct Quotient {
  float inv, low;
  __device__ __forceinline__ explicit Quotient(float scale) {
    inv = __builtin_amdgcn_rcpf(scale);
    low = __builtin_fmaf(-fminf(scale, kLargest), inv, 1.0f) * inv;
  }
  __device__ __forceinline__ float operator()(float v) const {
    return __builtin_fmaf(v, inv, v * low);
  }
};

typedef int v4i __attribute__((ext_vector_type(4)));

// 16 bytes moved down by 0 to 15 of them, zeros behind.
__device__ __forceinline__ v4i move_down(v4i v, int32_t bytes) {
  typedef uint64_t two __attribute__((ext_vector_type(2)));
  const two w = __builtin_bit_cast(two, v);
  const int32_t s = 8 * min(bytes, 15);
  const uint64_t lo = s < 64 ? w[0] >> s | w[1] << 1 << (63 - s) : w[1] >> (s - 64),
                 hi = s < 64 ? w[1] >> s : 0;
  return v4i{(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}

// 16 bytes of a row's codes from column c on, zeros behind its end: there the row's
// last 16 bytes are read and moved down, with no branch, so that several such loads can
// be under way before the first is used.  (Of fewer than 16 columns c is 0 or behind them.)
__device__ __forceinline__ v4i codes_read(const char* row, int32_t c, int32_t k) {
  typedef v4i mem __attribute__((aligned(1)));
  if (k >= 16) return *(const GG_GLOBAL mem*)(row + min(c, k - 16));
  uint64_t w[2] = {};
#pragma unroll 1
  for (int32_t i = 0; i < k; ++i)
    w[i / 8] |= (uint64_t) * (const GG_GLOBAL uint8_t*)(row + i) << 8 * (i % 8);
  return v4i{(int)w[0], (int)(w[0] >> 32), (int)w[1], (int)(w[1] >> 32)};
}
__device__ __forceinline__ v4i codes_moved(const v4i& v, int32_t c, int32_t k) {
  return c >= k ? v4i{} : c + 16 <= k || k < 16 ? v : move_down(v, c + 16 - k);
}
__device__ __forceinline__ v4i load_codes(const char* row, int32_t c, int32_t k) {
  return codes_moved(codes_read(row, c, k), c, k);
}

}  // namespace gg
