// Kernels of the root-mean-square norm and the layer norm, with the residual's
// addition and 8-bit rows with scales, forward and backward.
#pragma once

#include "codes.hpp"

namespace gg {
namespace {

// A row's pieces are dealt to a group of lanes: piece p = step * lanes + lane.
// A group is 2^lanes_log lanes of a wave (several rows per wave for narrow
// rows), or the whole block for wide ones.
struct CodeRows {
  KRows r;
  int32_t group_lanes_log;     // lanes that share a scale; -1: the row
  int32_t group_log;
};

struct NormArgs {
  KRows x, res, sum, y;        // p == nullptr: absent
  CodeRows q, kept;            // y and s in 8 bits
  const char* w;               // nullptr: ones
  const char* b;               // nullptr: zeros
  int32_t w_f32;
  float eps;
  float* mean;
  float* rstd;
  int64_t n;
  int32_t dim, pieces, lanes_log;
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

// Sum of squares, and sum, of a piece's own elements.
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
__device__ __forceinline__ float total(const float (&v)[V], int32_t skip) {
  float s = 0.0f;
#pragma unroll
  for (int k = 0; k < V; ++k) s += k >= skip ? v[k] : 0.0f;
  return s;
}

template <typename T, int V, int STEPS>
__device__ __forceinline__ void load_weights(const char* w, int32_t w_f32, const int32_t (&e)[STEPS],
                                             float (&v)[STEPS][V], float absent = 1.0f) {
  if (!w) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
#pragma unroll
      for (int k = 0; k < V; ++k) v[t][k] = absent;
  } else if (sizeof(T) == 4 || w_f32) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t) row_load<float, V>(w + e[t] * 4LL, v[t]);
  } else {
#pragma unroll
    for (int t = 0; t < STEPS; ++t) row_load<T, V>(w + e[t] * (int64_t)sizeof(T), v[t]);
  }
}

// scale = max(amax|v| / 448, 2^-126) per group, code = v / scale rounded to e4m3.
// The lanes of a row all call it.
template <int V, int STEPS, bool BLK>
__device__ __forceinline__ void store_codes(const CodeRows& q, int64_t row, int lanes, int l,
                                            int32_t pieces, const int32_t (&e)[STEPS],
                                            const int32_t (&skip)[STEPS],
                                            const float (&v)[STEPS][V], float* lds, bool stream) {
  // Largest magnitudes, each piece's own elements only.
  uint32_t top[STEPS], all = 0;
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    top[t] = 0;
    if (t * lanes + l < pieces)
      top[t] = magnitude<V>(v[t], skip[t]);
    all = max(all, top[t]);
  }
  const bool per_row = q.group_lanes_log < 0;
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
    const uint32_t m = per_row ? all : lanes_max(top[t], 1 << q.group_lanes_log);
    if (p >= pieces) continue;
    const float scale = scale_of(__uint_as_float(m));
    const Quotient by(scale);
    const bool first = per_row ? p == 0 : (p & ((1 << q.group_lanes_log) - 1)) == 0;
    if (first)
      ((float*)(q.r.scales + row * q.r.sstride))[per_row ? 0 : (p * V) >> q.group_log] = scale;
    float c[V];
#pragma unroll
    for (int k = 0; k < V; ++k) c[k] = by(v[t][k]);
    char* to = q.r.p + row * q.r.stride + e[t];
    if (skip[t] == 0) {
      row_store<e4m3, V>(to, c, stream);
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

// s = x + r; y = s * rstd * w, or with LAYER (s - mean) * rstd * w + b, the variance
// taken of the row in registers about its mean; y, and with LAYER s, in 8 bits.
//
// Bound by memory: each input is read once, the row stays in registers
// between the sum of squares and the outputs.  Nothing is stored before the
// row is read whole, so outputs may lie on the inputs.  A wave has a row of up to
// 256 pieces to itself, several where they are narrow, so that a sum needs no
// barrier.  32,768 rows of 4,096 bf16 with residual and sum take 182 us, 5.9
// TB/s; 200,000 of 602 fp32 364 us, 5.3; 2M of 33 fp32 177 us, 6.0; without a
// residual, 65,536 of 1,000 bf16 39 us, 6.7 (a 1 GiB copy: 5.0).  With LAYER 32,768
// of 4,096 bf16 with residual, sum and both 8-bit rows 187 us, 5.8 TB/s, call behind call; a
// kernel trace has each at 197.
template <typename T, typename R, bool LAYER, int V, int STEPS, bool BLK>
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
  float s[STEPS][V], w[STEPS][V], b[STEPS][V];
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
  if constexpr (LAYER) load_weights<T, V, STEPS>(a.b, a.w_f32, e, b, 0.0f);
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    to_f32<T, V>(rx[t], s[t]);
    if (a.res.p) {
      float r[V];
      to_f32<R, V>(rr[t], r);
#pragma unroll
      for (int k = 0; k < V; ++k) s[t][k] += r[k];
    }
  }
  float mean = 0.0f, sq = 0.0f;
  if constexpr (LAYER) {
    float part = 0.0f;
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
      if (t * lanes + l < a.pieces) part += total<V>(s[t], skip[t]);
    mean = group_sum<BLK>(part, lanes, lds) / (float)a.dim;
    if (a.mean && l == 0) a.mean[row] = mean;
  }
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const int p = t * lanes + l;
    if constexpr (LAYER) {
      // s leaves before its mean is taken off it
      if (p < a.pieces && a.sum.p)
        row_store<R, V>(a.sum.p + row * a.sum.stride + e[t] * (int64_t)sizeof(R), s[t], a.stream);
      float c[V];
#pragma unroll
      for (int k = 0; k < V; ++k) c[k] = s[t][k] - mean;
      if (p < a.pieces) sq += squares<V>(c, skip[t]);
    } else {
      if (p < a.pieces) sq += squares<V>(s[t], skip[t]);
    }
  }
  if constexpr (LAYER)
    if (a.kept.r.p)
      store_codes<V, STEPS, BLK>(a.kept, row, lanes, l, a.pieces, e, skip, s, lds, a.stream);
  sq = group_sum<BLK>(sq, lanes, lds);
  const float rstd = 1.0f / sqrtf(sq / (float)a.dim + a.eps);
  if (a.rstd && l == 0) a.rstd[row] = rstd;

#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    const int p = t * lanes + l;
    if constexpr (LAYER) {
#pragma unroll
      for (int k = 0; k < V; ++k)
        s[t][k] = __builtin_fmaf((s[t][k] - mean) * rstd, w[t][k], b[t][k]);
      if (p < a.pieces && a.y.p)
        row_store<T, V>(a.y.p + row * a.y.stride + e[t] * (int64_t)sizeof(T), s[t], a.stream);
    } else if (p < a.pieces) {
      if (a.sum.p) row_store<R, V>(a.sum.p + row * a.sum.stride + e[t] * (int64_t)sizeof(R), s[t],
                                 a.stream);
#pragma unroll
      for (int k = 0; k < V; ++k) s[t][k] = s[t][k] * rstd * w[t][k];
      if (a.y.p)
        row_store<T, V>(a.y.p + row * a.y.stride + e[t] * (int64_t)sizeof(T), s[t], a.stream);
    }
  }
  if (!a.q.r.p) return;
  store_codes<V, STEPS, BLK>(a.q, row, lanes, l, a.pieces, e, skip, s, lds, a.stream);
}

// ---------------------------------------------------------------------------
// Backward.  With g = dy * w, rho = rstd and h = s * rho, or with LAYER
// (s - mean) * rho:
//   dx = dsum + rho * (g - h * mean(g * h)), with LAYER also - rho * mean(g),
//   dw = sum_rows dy * h, db = sum_rows dy.
// s may be 8-bit rows, what a forward pass kept of it.
// Blocks stay for many rows and keep their share of dw and db in registers; the
// shares of all blocks are added in a second launch, in the order of the
// blocks.  Bound by memory: 32,768 rows of 4,096 bf16 209 us, 5.1 TB/s; 200,000 of
// 602 fp32 376 us, 5.1.  With LAYER 233,000 of 602 fp32 336 us, 5.0; 16,383 of 4,096
// bf16 from 8-bit rows 100 us, 4.7, both launches (98 and 6 by a trace).
// ---------------------------------------------------------------------------
struct NormBackArgs {
  KRows dy, dsum, s, dx;
  const char* w;
  int32_t w_f32;
  const float* mean;
  const float* rstd;
  int64_t n;
  int32_t dim, pieces, lanes_log;
  int32_t group_log;           // of s in 8 bits; 31: a scale per row
  float* part;                 // [dw, with LAYER db][blocks][dim], or nullptr: neither
  bool stream;
};

// Two sums over a row's lanes with one wait.
template <bool BLK>
__device__ __forceinline__ void group_sums(float* u, float* v, int lanes, float* lds) {
  if constexpr (BLK) {
    *u = lanes_sum(*u, kWave);
    *v = lanes_sum(*v, kWave);
    __syncthreads();
    if (lane_id() == 0) {
      lds[2 * (threadIdx.x / kWave)] = *u;
      lds[2 * (threadIdx.x / kWave) + 1] = *v;
    }
    __syncthreads();
    const int waves = lanes / kWave;
    float x = 0.0f, y = 0.0f;
    for (int i = 0; i < waves; ++i) {
      x += lds[2 * i];
      y += lds[2 * i + 1];
    }
    *u = x;
    *v = y;
  } else {
    *u = lanes_sum(*u, lanes);
    *v = lanes_sum(*v, lanes);
  }
}

template <typename T, typename R, typename S, bool LAYER, int V, int STEPS, bool BLK>
__global__ void __launch_bounds__(BLK ? 1024 : kBlock) k_norm_back(NormBackArgs a) {
  constexpr bool kCodes = sizeof(S) == 1;
  __shared__ float lds[BLK ? 2 * 1024 / kWave : kBlock * V];
  const int lanes = BLK ? (int)blockDim.x : 1 << a.lanes_log;
  const int groups = BLK ? 1 : kBlock >> a.lanes_log;
  const int g = BLK ? 0 : (int)threadIdx.x >> a.lanes_log;
  const int l = BLK ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
  float w[STEPS][V], acc[STEPS][V], acc_b[LAYER ? STEPS : 1][V];
  int32_t e[STEPS], skip[STEPS];
#pragma unroll
  for (int t = 0; t < STEPS; ++t) {
    e[t] = piece_start<V>(min(t * lanes + l, a.pieces - 1), a.dim, &skip[t]);
#pragma unroll
    for (int k = 0; k < V; ++k) acc[t][k] = 0.0f;
    if constexpr (LAYER)
#pragma unroll
      for (int k = 0; k < V; ++k) acc_b[t][k] = 0.0f;
  }
  // (rows of more than 8,192 elements leave no registers for the weights beside both
  // sums' shares or the codes: they come from the caches with every row)
  constexpr bool kHoldW = !(BLK && STEPS * V >= 16 && (LAYER || kCodes));
  if (kHoldW) load_weights<T, V, STEPS>(a.w, a.w_f32, e, w);
  // A row's loads are issued together (lanes behind the last piece repeat it),
  // and those of the next row before this one's sum is known, where the
  // registers hold both.
  constexpr bool kAhead = STEPS * V < 16;
  typename Raw<T, V>::vec rd[STEPS];
  typename Raw<R, V>::vec ra[STEPS];
  typename Raw<S, V>::vec rs[STEPS];
  // A piece of codes lies in one group, but for a row's last one, whose skipped
  // elements may be of the group before.
  float scale[kCodes ? STEPS : 1], scale_end[kCodes ? STEPS : 1];
  float rho_next = 0.0f, mean_next = 0.0f;
  const auto load_row = [&](int64_t row) {
    rho_next = a.rstd[row];
    if constexpr (LAYER) mean_next = a.mean[row];
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      rd[t] = raw_load<T, V>(a.dy.p + row * a.dy.stride + e[t] * (int64_t)sizeof(T));
      rs[t] = raw_load<S, V>(a.s.p + row * a.s.stride + e[t] * (int64_t)sizeof(S));
      if constexpr (kCodes) {
        const float* sc = (const float*)(a.s.scales + row * a.s.sstride);
        scale[t] = sc[e[t] >> a.group_log];
        scale_end[t] = sc[(e[t] + V - 1) >> a.group_log];
      }
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
    if (!kHoldW) load_weights<T, V, STEPS>(a.w, a.w_f32, e, w);
    const float rho = rho_next, mu = mean_next;
    float s[STEPS][V], d[STEPS][V], ds[STEPS][V];
    float dot = 0.0f, sum = 0.0f;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      to_f32<T, V>(rd[t], d[t]);
      to_f32<S, V>(rs[t], s[t]);
      to_f32<R, V>(ra[t], ds[t]);
      if constexpr (kCodes) {
        const int32_t cut = skip[t] == 0 ? 0 : ((e[t] + V - 1) >> a.group_log << a.group_log) - e[t];
#pragma unroll
        for (int k = 0; k < V; ++k) s[t][k] *= k >= cut ? scale_end[t] : scale[t];
      }
      float part = 0.0f, gs = 0.0f;
#pragma unroll
      for (int k = 0; k < V; ++k) {
        if constexpr (LAYER) s[t][k] -= mu;
        s[t][k] *= rho;
        acc[t][k] += d[t][k] * s[t][k];
        if constexpr (LAYER) acc_b[t][k] += d[t][k];
        d[t][k] *= w[t][k];
        part += k >= skip[t] ? d[t][k] * s[t][k] : 0.0f;
        if constexpr (LAYER) gs += k >= skip[t] ? d[t][k] : 0.0f;
      }
      dot += t * lanes + l < a.pieces ? part : 0.0f;
      if constexpr (LAYER) sum += t * lanes + l < a.pieces ? gs : 0.0f;
    }
    if (kAhead && row + step < a.n) load_row(row + step);
    if constexpr (LAYER)
      group_sums<BLK>(&dot, &sum, lanes, lds);
    else
      dot = group_sum<BLK>(dot, lanes, lds);
    const float mean = dot / (float)a.dim, off = sum / (float)a.dim;
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      const int p = t * lanes + l;
      if (p < a.pieces) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          if constexpr (LAYER)
            d[t][k] = ds[t][k] + rho * (d[t][k] - off - s[t][k] * mean);
          else
            d[t][k] = ds[t][k] + rho * (d[t][k] - s[t][k] * mean);
        }
        row_store<R, V>(a.dx.p + row * a.dx.stride + e[t] * (int64_t)sizeof(R), d[t], a.stream);
      }
    }
  }
  if (!a.part) return;
  const auto share = [&](float* part, float (&v)[STEPS][V]) {
#pragma unroll
    for (int t = 0; t < STEPS; ++t) {
      if constexpr (!BLK) {
        // the block's groups, in order
        __syncthreads();
#pragma unroll
        for (int k = 0; k < V; ++k) lds[k * kBlock + threadIdx.x] = v[t][k];
        __syncthreads();
        if (g == 0)
          for (int x = 1; x < groups; ++x)
#pragma unroll
            for (int k = 0; k < V; ++k) v[t][k] += lds[k * kBlock + x * lanes + l];
      }
      const int p = t * lanes + l;
      if (g == 0 && p < a.pieces) {
        row_store<float, V>((char*)(part + e[t]), v[t]);
      }
    }
  };
  share(a.part + (int64_t)blockIdx.x * a.dim, acc);
  if constexpr (LAYER) share(a.part + ((int64_t)gridDim.x + blockIdx.x) * a.dim, acc_b);
}

// dw[j] = sum of the blocks' shares: 64 columns a block, its waves take the
// shares in turn.  768 shares of 4,096 columns from the caches: 4.8 us, most of it
// the launch and two waits.  db's shares lie behind dw's, its blocks in a second row.
constexpr int kSumWaves = 16;

__global__ void __launch_bounds__(kSumWaves * kWave) k_norm_dw(const float* part, int32_t blocks,
                                                              int32_t dim, float* dw, float* db) {
  __shared__ float lds[kSumWaves][kWave];
  const int w = threadIdx.x / kWave, l = lane_id();
  const int32_t j = (int32_t)blockIdx.x * kWave + l;
  float* out = blockIdx.y ? db : dw;
  if (!out) return;
  part += (int64_t)blockIdx.y * blocks * dim;
  float v = 0.0f;
  if (j < dim)
#pragma unroll 8
    for (int32_t b = w; b < blocks; b += kSumWaves) v += part[(int64_t)b * dim + j];
  lds[w][l] = v;
  __syncthreads();
  if (w == 0 && j < dim) {
#pragma unroll
    for (int x = 1; x < kSumWaves; ++x) v += lds[x][l];
    out[j] = v;
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
inline Shape shape_of(int32_t dim, int vec, int wave_steps, int blk_steps) {
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
#define GG_NORM_LAUNCH(V, MW, S, ...)                                                           \
  do {                                                                                          \
    const dim3 threads((unsigned)(S).threads);                                                  \
    if ((S).blk) {                                                                              \
      if ((S).steps == 1)                                                                       \
        hipLaunchKernelGGL((__VA_ARGS__, V, 1, true>), grid, threads, 0, stream, a);                 \
      else if (V > 4 || (S).steps == 2)                                                         \
        hipLaunchKernelGGL((__VA_ARGS__, V, 2, true>), grid, threads, 0, stream, a);                 \
      else                                                                                      \
        hipLaunchKernelGGL((__VA_ARGS__, V, (V > 4 ? 2 : 4), true>), grid, threads, 0, stream, a);   \
    } else {                                                                                    \
      if ((S).steps == 1)                                                                       \
        hipLaunchKernelGGL((__VA_ARGS__, V, 1, false>), grid, threads, 0, stream, a);                \
      else if (MW == 2 || (S).steps == 2)                                                       \
        hipLaunchKernelGGL((__VA_ARGS__, V, 2, false>), grid, threads, 0, stream, a);                \
      else if ((S).steps == 3)                                                                  \
        hipLaunchKernelGGL((__VA_ARGS__, V, (MW > 2 ? 3 : 2), false>), grid, threads, 0, stream, a); \
      else                                                                                      \
        hipLaunchKernelGGL((__VA_ARGS__, V, (MW > 2 ? MW : 2), false>), grid, threads, 0, stream, a); \
    }                                                                                           \
  } while (0)

constexpr int kWaveSteps = 4, kBackWaveSteps = 2;

// A group's lanes, for pieces of vec elements.
inline void spread_groups(CodeRows* q, int32_t dim, int vec) {
  q->group_lanes_log = -1;
  if (q->r.p && q->r.group && q->r.group < dim) {
    q->group_log = __builtin_ctz((unsigned)q->r.group);
    q->group_lanes_log = q->group_log - __builtin_ctz((unsigned)vec);
  }
}

template <typename T, typename R, bool LAYER>
int launch_norm(NormArgs& a, hipStream_t stream) {
  constexpr int V = kVec<T>;
  const bool wide = a.dim >= V;
  const int vec = wide ? V : 1;
  const Shape s = shape_of(a.dim, vec, kWaveSteps, a.n < 256 ? 1 : 2);
  a.pieces = s.pieces;
  a.lanes_log = s.lanes_log;
  spread_groups(&a.q, a.dim, vec);
  spread_groups(&a.kept, a.dim, vec);
  const int64_t out = (a.sum.p ? sizeof(R) : 0) + (a.y.p ? sizeof(T) : 0) + (a.q.r.p ? 1 : 0) +
                      (a.kept.r.p ? 1 : 0);
  a.stream = out * a.n * a.dim > kStreamBytes;
  const dim3 grid = grid_of(s.blk ? a.n : cdiv(a.n << s.lanes_log, kBlock));
  if (!wide)
    hipLaunchKernelGGL((k_norm<T, R, LAYER, 1, 1, false>), grid, dim3(kBlock), 0, stream, a);
  else
    GG_NORM_LAUNCH(V, kWaveSteps, s, k_norm<T, R, LAYER);
  GG_LAUNCH_CHECK("k_norm");
  return GG_OK;
}

// Blocks of the backward pass: three for each of 256 CUs, four where a block's
// row is below 4 KB (100,000 x 602 fp32: 149 us with 768 blocks, 134 with
// 1,024; 65,536 x 2,048 bf16: 188 and 215).
inline int back_blocks(int64_t n, int64_t row_bytes, const Shape& s) {
  const int64_t rows = s.blk ? 1 : kBlock >> s.lanes_log;   // at a time in a block
  return (int)std::min<int64_t>(cdiv(n, rows), s.blk && row_bytes < 4096 ? 1024 : 768);
}

template <typename T, typename R, typename S, bool LAYER>
int launch_back(NormBackArgs& a, float* dw, float* db, hipStream_t stream) {
  constexpr int V = kVec<T>;
  const bool wide = a.dim >= V;
  const Shape s = shape_of(a.dim, wide ? V : 1, kBackWaveSteps, 1);
  a.pieces = s.pieces;
  a.lanes_log = s.lanes_log;
  a.group_log = a.s.group ? __builtin_ctz((unsigned)a.s.group) : 31;
  a.stream = (int64_t)sizeof(R) * a.n * a.dim > kStreamBytes;
  const int blocks = back_blocks(a.n, a.dim * (int64_t)sizeof(T), s);
  const dim3 grid((unsigned)blocks);
  if (blocks > 0) {
    if (!wide)
      hipLaunchKernelGGL((k_norm_back<T, R, S, LAYER, 1, 1, false>), grid, dim3(kBlock), 0, stream, a);
    else
      GG_NORM_LAUNCH(V, kBackWaveSteps, s, k_norm_back<T, R, S, LAYER);
    GG_LAUNCH_CHECK("k_norm_back");
  }
  if (dw || db) {
    hipLaunchKernelGGL(k_norm_dw, dim3((unsigned)cdiv(a.dim, kWave), LAYER ? 2u : 1u),
                       dim3(kSumWaves * kWave), 0, stream, a.part, blocks, a.dim, dw, db);
    GG_LAUNCH_CHECK("k_norm_dw");
  }
  return GG_OK;
}

// Optional rows: absent (p stays NULL) or checked.
inline int pack_optional(const gg_rows_t* r, const char* name, int64_t n, int64_t dim, uint32_t types,
                         bool written, KRows* out) {
  if (!r) return GG_OK;
  return pack_rows(r, name, n, dim, types, written, out);
}

// What the forward calls of both norms take, checked and packed.
inline int pack_norm(const gg_rows_t* x, const gg_rows_t* res, int64_t n, int32_t dim,
                     const void* w_d, const void* b_d, int32_t w_dtype, float eps,
                     const gg_rows_t* sum, const gg_rows_t* y, const gg_rows_t* q,
                     const gg_rows_t* kept, float* mean_d, float* rstd_d, NormArgs* a) {
  GG_REQUIRE(dim >= 1 && dim <= GG_NORM_MAX_DIM, "dim %d outside 1..%d", dim, GG_NORM_MAX_DIM);
  GG_REQUIRE(n >= 0 && n <= GG_NORM_MAX_ROWS, "n = %lld unsupported", (long long)n);
  GG_REQUIRE(eps >= 0.0f, "eps must not be negative");
  GG_REQUIRE(sum || y || q || kept || mean_d || rstd_d, "no output asked for");
  int rc = pack_rows(x, "x", n, dim, kBitFloats, false, &a->x);
  if (rc != GG_OK) return rc;
  const int32_t t = x->dtype;
  GG_REQUIRE(!(w_d || b_d) || w_dtype == t || w_dtype == GG_F32,
             "weights of dtype %d for x of dtype %d", w_dtype, t);
  GG_REQUIRE(!w_d || (uintptr_t)w_d % elem_bytes(w_dtype) == 0, "weights are not aligned");
  GG_REQUIRE(!b_d || (uintptr_t)b_d % elem_bytes(w_dtype) == 0, "bias is not aligned");
  GG_REQUIRE((uintptr_t)mean_d % 4 == 0, "mean is not aligned");
  GG_REQUIRE((uintptr_t)rstd_d % 4 == 0, "rstd is not aligned");
  const uint32_t stream_types = (1u << t) | kBitF32;
  rc = pack_optional(res, "res", n, dim, stream_types, false, &a->res);
  if (rc == GG_OK) rc = pack_optional(sum, "sum", n, dim, stream_types, true, &a->sum);
  if (rc == GG_OK) rc = pack_optional(y, "y", n, dim, 1u << t, true, &a->y);
  if (rc == GG_OK) rc = pack_optional(q, "q", n, dim, kBitE4M3, true, &a->q.r);
  if (rc == GG_OK) rc = pack_optional(kept, "kept", n, dim, kBitE4M3, true, &a->kept.r);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(!res || !sum || res->dtype == sum->dtype, "res and sum differ in dtype");
  a->w = (const char*)w_d;
  a->b = (const char*)b_d;
  a->w_f32 = w_dtype == GG_F32;
  a->eps = eps;
  a->mean = mean_d;
  a->rstd = rstd_d;
  a->n = n;
  a->dim = dim;
  return GG_OK;
}

template <bool LAYER>
int run_norm(NormArgs& a, int32_t t, const gg_rows_t* res, const gg_rows_t* sum,
             hipStream_t stream) {
  const int32_t r = res ? res->dtype : sum ? sum->dtype : t;
  GG_FOR_FLOAT(t, T, {
    if (r == t) return launch_norm<T, T, LAYER>(a, stream);
    return launch_norm<T, float, LAYER>(a, stream);
  });
}

// And the backward calls; `ws` holds the shares of dw, with LAYER of db too.
template <bool LAYER>
int run_back(const gg_rows_t* dy, const gg_rows_t* dsum, const gg_rows_t* s, const float* mean_d,
             const float* rstd_d, int64_t n, int32_t dim, const void* w_d, int32_t w_dtype,
             const gg_rows_t* dx, float* dw_d, float* db_d, void* ws, size_t ws_bytes, size_t need,
             hipStream_t stream) {
  GG_REQUIRE(dim >= 1 && dim <= GG_NORM_MAX_DIM, "dim %d outside 1..%d", dim, GG_NORM_MAX_DIM);
  GG_REQUIRE(n >= 0 && n <= GG_NORM_MAX_ROWS, "n = %lld unsupported", (long long)n);
  NormBackArgs a = {};
  int rc = pack_rows(dy, "dy", n, dim, kBitFloats, false, &a.dy);
  if (rc != GG_OK) return rc;
  const int32_t t = dy->dtype;
  rc = pack_rows(s, "s", n, dim, (1u << t) | kBitF32 | kBitE4M3, false, &a.s);
  if (rc != GG_OK) return rc;
  const bool codes = s->dtype == GG_E4M3;
  rc = pack_rows(dx, "dx", n, dim, codes ? (1u << t) | kBitF32 : 1u << s->dtype, true, &a.dx);
  if (rc != GG_OK) return rc;
  const int32_t r = dx->dtype;
  rc = pack_optional(dsum, "dsum", n, dim, 1u << r, false, &a.dsum);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(n == 0 || !LAYER || mean_d, "mean is NULL");
  GG_REQUIRE(n == 0 || rstd_d, "rstd is NULL");
  GG_REQUIRE((uintptr_t)mean_d % 4 == 0, "mean is not aligned");
  GG_REQUIRE((uintptr_t)rstd_d % 4 == 0 && (uintptr_t)dw_d % 4 == 0 && (uintptr_t)db_d % 4 == 0,
             "rstd, dw or db is not aligned");
  GG_REQUIRE(!w_d || w_dtype == t || w_dtype == GG_F32, "weights of dtype %d for dy of dtype %d",
             w_dtype, t);
  GG_REQUIRE(!w_d || (uintptr_t)w_d % elem_bytes(w_dtype) == 0, "weights are not aligned");
  const bool shares = dw_d || db_d;
  GG_REQUIRE(!shares || need == 0 || (ws && (uintptr_t)ws % 16 == 0 && ws_bytes >= need),
             "workspace of %zu bytes < %zu, or not aligned", ws_bytes, need);
  a.w = (const char*)w_d;
  a.w_f32 = w_dtype == GG_F32;
  a.mean = mean_d;
  a.rstd = rstd_d;
  a.n = n;
  a.dim = dim;
  a.part = shares ? (float*)ws : nullptr;
  GG_FOR_FLOAT(t, T, {
    if (codes) {
      if (r == t) return launch_back<T, T, e4m3, LAYER>(a, dw_d, db_d, stream);
      return launch_back<T, float, e4m3, LAYER>(a, dw_d, db_d, stream);
    }
    if (r == t) return launch_back<T, T, T, LAYER>(a, dw_d, db_d, stream);
    return launch_back<T, float, float, LAYER>(a, dw_d, db_d, stream);
  });
}

}  // namespace
}  // namespace gg
