// Root-mean-square norm with the residual's addition and 8-bit rows with
// scales, forward and backward.
#include "rows.hpp"

namespace gg {
namespace {

constexpr float kE4M3Max = 448.0f;
constexpr float kScaleMin = 1.17549435e-38f;   // 2^-126
constexpr float kLargest = 3.4028235e38f;

// A row's pieces are dealt to a group of lanes: piece p = step * lanes + lane.
// A group is 2^lanes_log lanes of a wave (several rows per wave for narrow
// rows), or the whole block for wide ones.
struct NormArgs {
  KRows x, res, sum, y, q;     // p == nullptr: absent
  const char* w;               // nullptr: ones
  int32_t w_f32;
  float eps;
  float* rstd;
  int64_t n;
  int32_t dim, pieces, lanes_log;
  int32_t group_lanes_log;     // lanes that share a scale; -1: the row
  int32_t group_log;
  bool stream;                 // the outputs go past the caches
};

template <bool BLK>
__device__ __forceinline__ float group_sum(float v, int lanes, float* lds) {
  if constexpr (BLK) {
    v = lanes_sum(v, kWave);
    __syncthreads();
    if (lane_id() == 0) lds[threadIdx.x / kWave] = v;
    __syncthreads();
    const int waves = lanes / kWave;
    float t = 0.0f;
    for (int i = 0; i < waves; ++i) t += lds[i];
    return t;
  } else {
    return lanes_sum(v, lanes);
  }
}

// Sum of squares, and largest magnitude, of a piece's own elements: only a
// row's last piece has others (skip > 0).
template <int V>
__device__ __forceinline__ float squares(const float (&v)[V], int32_t skip) {
  float s = 0.0f;
  if (skip == 0) {
#pragma unroll
    for (int k = 0; k < V; ++k) s += v[k] * v[k];
  } else {
#pragma unroll
    for (int k = 0; k < V; ++k) s += k >= skip ? v[k] * v[k] : 0.0f;
  }
  return s;
}

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

template <typename T, int V, int STEPS>
__device__ __forceinline__ void load_weights(const char* w, int32_t w_f32, const int32_t (&e)[STEPS],
                                             float (&v)[STEPS][V]) {
  if (!w) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
#pragma unroll
      for (int k = 0; k < V; ++k) v[t][k] = 1.0f;
  } else if (sizeof(T) == 4 || w_f32) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t) row_load<float, V>(w + e[t] * 4LL, v[t]);
  } else {
#pragma unroll
    for (int t = 0; t < STEPS; ++t) row_load<T, V>(w + e[t] * (int64_t)sizeof(T), v[t]);
  }
}

// s = x + r; y = s * rstd * w; scale = max(amax|y| / 448, 2^-126) per group,
// code = y / scale rounded to e4m3.
//
// Bound by memory: each input is read once, the row stays in registers
// between the sum of squares and the outputs.  Nothing is stored before the
// row is read whole, so outputs may lie on the inputs.  A wave has a row of up to
// 256 pieces to itself, several where they are narrow, so that a sum needs no
// barrier.  32,768 rows of 4,096 bf16 with residual and sum take 182 us, 5.9
// TB/s; 200,000 of 602 fp32 364 us, 5.3; 2M of 33 fp32 177 us, 6.0; without a
// residual, 65,536 of 1,000 bf16 39 us, 6.7 (a 1 GiB copy: 5.0).
template <typename T, typename R, int V, int STEPS, bool BLK>
__global__ void __launch_bounds__(BLK ? 1024 : kBlock) k_norm(NormArgs a) {
  __shared__ float lds[BLK ? 1024 / kWave : 1];
  const int lanes = BLK ? (int)blockDim.x : 1 << a.lanes_log;
  const int64_t row = BLK ? block_index() : (block_index() * kBlock + threadIdx.x) >> a.lanes_log;
  if (row >= a.n) return;
  const int l = BLK ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
  // All loads before any use, so that the row is one wait; lanes behind the
  // last piece repeat it and count nothing.
  typename Raw<T, V>::vec rx[STEPS];
  typename Raw<R, V>::vec rr[STEPS];
  float s[STEPS][V], w[STEPS][V];
  int32_t e[STEPS], skip[STEPS];
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    e[t] = piece_start<V>(min(t * lanes + l, a.pieces - 1), a.dim, &skip[t]);
    rx[t] = raw_load<T, V>(a.x.p + row * a.x.stride + e[t] * (int64_t)sizeof(T));
  }
  if (a.res.p) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
      rr[t] = raw_load<R, V>(a.res.p + row * a.res.stride + e[t] * (int64_t)sizeof(R));
  }
  load_weights<T, V, STEPS>(a.w, a.w_f32, e, w);
  float sq = 0.0f;
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    to_f32<T, V>(rx[t], s[t]);
    if (a.res.p) {
      float r[V];
      to_f32<R, V>(rr[t], r);
#pragma unroll
      for (int k = 0; k < V; ++k) s[t][k] += r[k];
    }
    if (t * lanes + l < a.pieces) sq += squares<V>(s[t], skip[t]);
  }
  sq = group_sum<BLK>(sq, lanes, lds);
  const float rstd = 1.0f / sqrtf(sq / (float)a.dim + a.eps);
  if (a.rstd && l == 0) a.rstd[row] = rstd;

#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const int p = t * lanes + l;
    if (p < a.pieces) {
      if (a.sum.p) row_store<R, V>(a.sum.p + row * a.sum.stride + e[t] * (int64_t)sizeof(R), s[t],
                                 a.stream);
#pragma unroll
      for (int k = 0; k < V; ++k) s[t][k] = s[t][k] * rstd * w[t][k];
      if (a.y.p)
        row_store<T, V>(a.y.p + row * a.y.stride + e[t] * (int64_t)sizeof(T), s[t], a.stream);
    }
  }
  if (!a.q.p) return;

  // Largest magnitudes, each piece's own elements only.
  uint32_t top[STEPS], all = 0;
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    top[t] = 0;
    if (t * lanes + l < a.pieces)
      top[t] = magnitude<V>(s[t], skip[t]);
    all = max(all, top[t]);
  }
  const bool per_row = a.group_lanes_log < 0;
  if (per_row) {
    all = lanes_max(all, min(lanes, kWave));
    if constexpr (BLK) {
      __syncthreads();
      if (lane_id() == 0) ((uint32_t*)lds)[threadIdx.x / kWave] = all;
      __syncthreads();
      for (int i = 0; i < lanes / kWave; ++i) all = max(all, ((uint32_t*)lds)[i]);
    }
  }
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const int p = t * lanes + l;
    const uint32_t m = per_row ? all : lanes_max(top[t], 1 << a.group_lanes_log);
    if (p >= a.pieces) continue;
    const float scale = scale_of(__uint_as_float(m));
    // The reciprocal in two parts, so that the codes are those of the quotient
    // rounded to fp32, at one operation an element more than a product with its
    // first part, which is a unit off and now and then another code (233,000 rows of
    // 602 fp32 in groups of 64 137 us so, 144 this way, a quarter more divided outright).
    const float inv = __builtin_amdgcn_rcpf(scale);
    const float low = __builtin_fmaf(-fminf(scale, kLargest), inv, 1.0f) * inv;
    const bool first = per_row ? p == 0 : (p & ((1 << a.group_lanes_log) - 1)) == 0;
    if (first)
      ((float*)(a.q.scales + row * a.q.sstride))[per_row ? 0 : (p * V) >> a.group_log] = scale;
    float c[V];
#pragma unroll
    for (int k = 0; k < V; ++k) c[k] = __builtin_fmaf(s[t][k], inv, s[t][k] * low);
    char* to = a.q.p + row * a.q.stride + e[t];
    if (skip[t] == 0) {
      row_store<e4m3, V>(to, c, a.stream);
    } else {
      // the skipped elements have their own piece's scale
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float one[1] = {c[k]};
        if (k >= skip[t]) row_store<e4m3, 1>(to + k, one);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Backward.  With g = dy * w and rho = rstd:
//   dx = dsum + rho * (g - s * rho^2 * mean(g * s)),  dw = sum_rows dy * s * rho.
// Blocks stay for many rows and keep their share of dw in registers; the
// shares of all blocks are added in a second launch, in the order of the
// blocks.  Bound by memory: 32,768 rows of 4,096 bf16 209 us, 5.1 TB/s; 200,000 of
// 602 fp32 376 us, 5.1.
// ---------------------------------------------------------------------------
struct NormBackArgs {
  KRows dy, dsum, s, dx;
  const char* w;
  int32_t w_f32;
  const float* rstd;
  int64_t n;
  int32_t dim, pieces, lanes_log;
  float* part;                 // [blocks][dim], or nullptr: no dw
  bool stream;
};

template <typename T, typename R, int V, int STEPS, bool BLK>
__global__ void __launch_bounds__(BLK ? 1024 : kBlock) k_norm_back(NormBackArgs a) {
  __shared__ float lds[BLK ? 1024 / kWave : kBlock * V];
  const int lanes = BLK ? (int)blockDim.x : 1 << a.lanes_log;
  const int groups = BLK ? 1 : kBlock >> a.lanes_log;
  const int g = BLK ? 0 : (int)threadIdx.x >> a.lanes_log;
  const int l = BLK ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
  float w[STEPS][V], acc[STEPS][V];
  int32_t e[STEPS], skip[STEPS];
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    e[t] = piece_start<V>(min(t * lanes + l, a.pieces - 1), a.dim, &skip[t]);
#pragma unroll
    for (int k = 0; k < V; ++k) acc[t][k] = 0.0f;
  }
  load_weights<T, V, STEPS>(a.w, a.w_f32, e, w);
  // A row's loads are issued together (lanes behind the last piece repeat it),
  // and those of the next row before this one's sum is known, where the
  // registers hold both.
  constexpr bool kAhead = STEPS * V < 16;
  typename Raw<T, V>::vec rd[STEPS];
  typename Raw<R, V>::vec rs[STEPS], ra[STEPS];
  float rho_next = 0.0f;
  const auto load_row = [&](int64_t row) {
    rho_next = a.rstd[row];
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      rd[t] = raw_load<T, V>(a.dy.p + row * a.dy.stride + e[t] * (int64_t)sizeof(T));
      rs[t] = raw_load<R, V>(a.s.p + row * a.s.stride + e[t] * (int64_t)sizeof(R));
      ra[t] = {};
    }
    if (a.dsum.p) {
#pragma unroll
      for (int t = 0; t < STEPS; ++t)
        ra[t] = raw_load<R, V>(a.dsum.p + row * a.dsum.stride + e[t] * (int64_t)sizeof(R));
    }
  };
  const int64_t step = (int64_t)gridDim.x * groups;
  int64_t row = (int64_t)blockIdx.x * groups + g;
  if (kAhead && row < a.n) load_row(row);
  for (; row < a.n; row += step) {
    if (!kAhead) load_row(row);
    const float rho = rho_next;
    float s[STEPS][V], d[STEPS][V], ds[STEPS][V];
    float dot = 0.0f;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      to_f32<T, V>(rd[t], d[t]);
      to_f32<R, V>(rs[t], s[t]);
      to_f32<R, V>(ra[t], ds[t]);
      float part = 0.0f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        s[t][k] *= rho;
        acc[t][k] += d[t][k] * s[t][k];
        d[t][k] *= w[t][k];
        part += k >= skip[t] ? d[t][k] * s[t][k] : 0.0f;
      }
      dot += t * lanes + l < a.pieces ? part : 0.0f;
    }
    if (kAhead && row + step < a.n) load_row(row + step);
    dot = group_sum<BLK>(dot, lanes, lds);
    const float mean = dot / (float)a.dim;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      const int p = t * lanes + l;
      if (p < a.pieces) {
#pragma unroll
        for (int k = 0; k < V; ++k) d[t][k] = ds[t][k] + rho * (d[t][k] - s[t][k] * mean);
        row_store<R, V>(a.dx.p + row * a.dx.stride + e[t] * (int64_t)sizeof(R), d[t], a.stream);
      }
    }
  }
  if (!a.part) return;
  float* part = a.part + (int64_t)blockIdx.x * a.dim;
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    if constexpr (!BLK) {
      // the block's groups, in order
      __syncthreads();
#pragma unroll
      for (int k = 0; k < V; ++k) lds[k * kBlock + threadIdx.x] = acc[t][k];
      __syncthreads();
      if (g == 0)
        for (int x = 1; x < groups; ++x)
#pragma unroll
          for (int k = 0; k < V; ++k) acc[t][k] += lds[k * kBlock + x * lanes + l];
    }
    const int p = t * lanes + l;
    if (g == 0 && p < a.pieces) {
      row_store<float, V>((char*)(part + e[t]), acc[t]);
    }
  }
}

// dw[j] = sum of the blocks' shares: 64 columns a block, its waves take the
// shares in turn.  768 shares of 4,096 columns from the caches: 4.8 us, most of it
// the launch and two waits.
constexpr int kSumWaves = 16;

__global__ void __launch_bounds__(kSumWaves * kWave) k_norm_dw(const float* part, int32_t blocks,
                                                              int32_t dim, float* dw) {
  __shared__ float lds[kSumWaves][kWave];
  const int w = threadIdx.x / kWave, l = lane_id();
  const int32_t j = (int32_t)blockIdx.x * kWave + l;
  float v = 0.0f;
  if (j < dim)
#pragma unroll 8
    for (int32_t b = w; b < blocks; b += kSumWaves) v += part[(int64_t)b * dim + j];
  lds[w][l] = v;
  __syncthreads();
  if (w == 0 && j < dim) {
#pragma unroll
    for (int x = 1; x < kSumWaves; ++x) v += lds[x][l];
    dw[j] = v;
  }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct Shape {
  bool blk;
  int32_t pieces, lanes_log, steps;   // steps: 1 .. 4
  int threads;
};

// A wave (or part of one) per row up to `wave_steps` pieces per lane, a block
// per row beyond, of threads with about `blk_steps` pieces each.
Shape shape_of(int32_t dim, int vec, int wave_steps, int blk_steps) {
  Shape s;
  s.pieces = (int32_t)cdiv(dim, vec);
  s.lanes_log = 0;
  while (s.lanes_log < 6 && (1 << s.lanes_log) < s.pieces) ++s.lanes_log;
  s.blk = s.pieces > kWave * wave_steps;
  s.threads = kBlock;
  int lanes = 1 << s.lanes_log;
  if (s.blk) {
    s.threads = 128;
    while (s.threads < 1024 && s.threads * blk_steps < s.pieces) s.threads *= 2;
    lanes = s.threads;
  }
  s.steps = (int32_t)cdiv(s.pieces, lanes);
  return s;
}

// Instantiations: a block per row takes 2 pieces per lane, or 4 of fp32 rows
// (16,384 elements, 1,024 lanes); a wave per row up to MW.
#define GG_NORM_LAUNCH(K, T, R, V, MW, S)                                                       \
  do {                                                                                          \
    const dim3 threads((unsigned)(S).threads);                                                  \
    if ((S).blk) {                                                                              \
      if ((S).steps == 1)                                                                       \
        hipLaunchKernelGGL((K<T, R, V, 1, true>), grid, threads, 0, stream, a);                 \
      else if (V > 4 || (S).steps == 2)                                                         \
        hipLaunchKernelGGL((K<T, R, V, 2, true>), grid, threads, 0, stream, a);                 \
      else                                                                                      \
        hipLaunchKernelGGL((K<T, R, V, (V > 4 ? 2 : 4), true>), grid, threads, 0, stream, a);   \
    } else {                                                                                    \
      if ((S).steps == 1)                                                                       \
        hipLaunchKernelGGL((K<T, R, V, 1, false>), grid, threads, 0, stream, a);                \
      else if (MW == 2 || (S).steps == 2)                                                       \
        hipLaunchKernelGGL((K<T, R, V, 2, false>), grid, threads, 0, stream, a);                \
      else if ((S).steps == 3)                                                                  \
        hipLaunchKernelGGL((K<T, R, V, (MW > 2 ? 3 : 2), false>), grid, threads, 0, stream, a); \
      else                                                                                      \
        hipLaunchKernelGGL((K<T, R, V, (MW > 2 ? MW : 2), false>), grid, threads, 0, stream, a); \
    }                                                                                           \
  } while (0)

constexpr int kWaveSteps = 4, kBackWaveSteps = 2;

template <typename T, typename R>
int launch_norm(NormArgs& a, hipStream_t stream) {
  constexpr int V = kVec<T>;
  const bool wide = a.dim >= V;
  const int vec = wide ? V : 1;
  const Shape s = shape_of(a.dim, vec, kWaveSteps, a.n < 256 ? 1 : 2);
  a.pieces = s.pieces;
  a.lanes_log = s.lanes_log;
  a.group_lanes_log = -1;
  if (a.q.p && a.q.group && a.q.group < a.dim) {
    a.group_log = __builtin_ctz((unsigned)a.q.group);
    a.group_lanes_log = a.group_log - __builtin_ctz((unsigned)vec);
  }
  const int64_t out = (a.sum.p ? sizeof(R) : 0) + (a.y.p ? sizeof(T) : 0) + (a.q.p ? 1 : 0);
  a.stream = out * a.n * a.dim > kStreamBytes;
  const dim3 grid = grid_of(s.blk ? a.n : cdiv(a.n << s.lanes_log, kBlock));
  if (!wide)
    hipLaunchKernelGGL((k_norm<T, R, 1, 1, false>), grid, dim3(kBlock), 0, stream, a);
  else
    GG_NORM_LAUNCH(k_norm, T, R, V, kWaveSteps, s);
  GG_LAUNCH_CHECK("k_norm");
  return GG_OK;
}

// Blocks of the backward pass: three for each of 256 CUs, four where a block's
// row is below 4 KB (100,000 x 602 fp32: 149 us with 768 blocks, 134 with
// 1,024; 65,536 x 2,048 bf16: 188 and 215).
int back_blocks(int64_t n, int64_t row_bytes, const Shape& s) {
  const int64_t rows = s.blk ? 1 : kBlock >> s.lanes_log;   // at a time in a block
  return (int)std::min<int64_t>(cdiv(n, rows), s.blk && row_bytes < 4096 ? 1024 : 768);
}

template <typename T, typename R>
int launch_back(NormBackArgs& a, float* dw, hipStream_t stream) {
  constexpr int V = kVec<T>;
  const bool wide = a.dim >= V;
  const Shape s = shape_of(a.dim, wide ? V : 1, kBackWaveSteps, 1);
  a.pieces = s.pieces;
  a.lanes_log = s.lanes_log;
  a.stream = (int64_t)sizeof(R) * a.n * a.dim > kStreamBytes;
  const int blocks = back_blocks(a.n, a.dim * (int64_t)sizeof(T), s);
  const dim3 grid((unsigned)blocks);
  if (blocks > 0) {
    if (!wide)
      hipLaunchKernelGGL((k_norm_back<T, R, 1, 1, false>), grid, dim3(kBlock), 0, stream, a);
    else
      GG_NORM_LAUNCH(k_norm_back, T, R, V, kBackWaveSteps, s);
    GG_LAUNCH_CHECK("k_norm_back");
  }
  if (dw) {
    hipLaunchKernelGGL(k_norm_dw, dim3((unsigned)cdiv(a.dim, kWave)), dim3(kSumWaves * kWave), 0,
                       stream, a.part, blocks, a.dim, dw);
    GG_LAUNCH_CHECK("k_norm_dw");
  }
  return GG_OK;
}

// Optional rows: absent (p stays NULL) or checked.
int pack_optional(const gg_rows_t* r, const char* name, int64_t n, int64_t dim, uint32_t types,
                  bool written, KRows* out) {
  if (!r) return GG_OK;
  return pack_rows(r, name, n, dim, types, written, out);
}

}  // namespace
}  // namespace gg

using namespace gg;

extern "C" int gg_rmsnorm_forward(const gg_rows_t* x, const gg_rows_t* res, int64_t n, int32_t dim,
                                  const void* w_d, int32_t w_dtype, float eps,
                                  const gg_rows_t* sum, const gg_rows_t* y, const gg_rows_t* q,
                                  float* rstd_d, hipStream_t stream) {
  GG_REQUIRE(dim >= 1 && dim <= GG_NORM_MAX_DIM, "dim %d outside 1..%d", dim, GG_NORM_MAX_DIM);
  GG_REQUIRE(n >= 0 && n <= GG_NORM_MAX_ROWS, "n = %lld unsupported", (long long)n);
  GG_REQUIRE(eps >= 0.0f, "eps must not be negative");
  GG_REQUIRE(sum || y || q || rstd_d, "no output asked for");
  NormArgs a = {};
  int rc = pack_rows(x, "x", n, dim, kBitFloats, false, &a.x);
  if (rc != GG_OK) return rc;
  const int32_t t = x->dtype;
  GG_REQUIRE(!w_d || w_dtype == t || w_dtype == GG_F32, "weights of dtype %d for x of dtype %d",
             w_dtype, t);
  GG_REQUIRE(!w_d || (uintptr_t)w_d % elem_bytes(w_dtype) == 0, "weights are not aligned");
  GG_REQUIRE((uintptr_t)rstd_d % 4 == 0, "rstd is not aligned");
  const uint32_t stream_types = (1u << t) | kBitF32;
  rc = pack_optional(res, "res", n, dim, stream_types, false, &a.res);
  if (rc == GG_OK) rc = pack_optional(sum, "sum", n, dim, stream_types, true, &a.sum);
  if (rc == GG_OK) rc = pack_optional(y, "y", n, dim, 1u << t, true, &a.y);
  if (rc == GG_OK) rc = pack_optional(q, "q", n, dim, kBitE4M3, true, &a.q);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(!res || !sum || res->dtype == sum->dtype, "res and sum differ in dtype");
  if (n == 0) return GG_OK;
  const int32_t r = res ? res->dtype : sum ? sum->dtype : t;
  a.w = (const char*)w_d;
  a.w_f32 = w_dtype == GG_F32;
  a.eps = eps;
  a.rstd = rstd_d;
  a.n = n;
  a.dim = dim;
  GG_FOR_FLOAT(t, T, {
    if (r == t) return launch_norm<T, T>(a, stream);
    return launch_norm<T, float>(a, stream);
  });
}

extern "C" size_t gg_ws_rmsnorm(int64_t n, int32_t dim) {
  if (n < 0 || n > GG_NORM_MAX_ROWS || dim < 1 || dim > GG_NORM_MAX_DIM) return 0;
  return align_up((size_t)std::min<int64_t>(n, 1024) * dim * sizeof(float), 256);
}

extern "C" int gg_rmsnorm_backward(const gg_rows_t* dy, const gg_rows_t* dsum, const gg_rows_t* s,
                                   const float* rstd_d, int64_t n, int32_t dim, const void* w_d,
                                   int32_t w_dtype, const gg_rows_t* dx, float* dw_d, void* ws,
                                   size_t ws_bytes, hipStream_t stream) {
  GG_REQUIRE(dim >= 1 && dim <= GG_NORM_MAX_DIM, "dim %d outside 1..%d", dim, GG_NORM_MAX_DIM);
  GG_REQUIRE(n >= 0 && n <= GG_NORM_MAX_ROWS, "n = %lld unsupported", (long long)n);
  NormBackArgs a = {};
  int rc = pack_rows(dy, "dy", n, dim, kBitFloats, false, &a.dy);
  if (rc != GG_OK) return rc;
  const int32_t t = dy->dtype;
  rc = pack_rows(s, "s", n, dim, (1u << t) | kBitF32, false, &a.s);
  if (rc != GG_OK) return rc;
  const int32_t r = s->dtype;
  rc = pack_rows(dx, "dx", n, dim, 1u << r, true, &a.dx);
  if (rc == GG_OK) rc = pack_optional(dsum, "dsum", n, dim, 1u << r, false, &a.dsum);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(n == 0 || rstd_d, "rstd is NULL");
  GG_REQUIRE((uintptr_t)rstd_d % 4 == 0 && (uintptr_t)dw_d % 4 == 0, "rstd or dw is not aligned");
  GG_REQUIRE(!w_d || w_dtype == t || w_dtype == GG_F32, "weights of dtype %d for dy of dtype %d",
             w_dtype, t);
  GG_REQUIRE(!w_d || (uintptr_t)w_d % elem_bytes(w_dtype) == 0, "weights are not aligned");
  const size_t need = gg_ws_rmsnorm(n, dim);
  GG_REQUIRE(!dw_d || need == 0 || (ws && (uintptr_t)ws % 16 == 0 && ws_bytes >= need),
             "workspace of %zu bytes < %zu, or not aligned", ws_bytes, need);
  a.w = (const char*)w_d;
  a.w_f32 = w_dtype == GG_F32;
  a.rstd = rstd_d;
  a.n = n;
  a.dim = dim;
  a.part = dw_d ? (float*)ws : nullptr;
  GG_FOR_FLOAT(t, T, {
    if (r == t) return launch_back<T, T>(a, dw_d, stream);
    return launch_back<T, float>(a, dw_d, stream);
  });
}
