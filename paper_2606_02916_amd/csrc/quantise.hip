// Rows and weights into 8 bits: a scale for each group of a row's elements, or
// for each 128 x 128 elements of the weights, which may leave transposed too.
#include "codes.hpp"
#include "tiles.hpp"

namespace gg {
namespace {

// ---------------------------------------------------------------------------
// Rows.
// ---------------------------------------------------------------------------
struct RowsArgs {
  KRows x, q;
  int64_t n;
  int64_t lanes;               // of all rows together
  int32_t dim, pieces;
  int32_t group_lanes_log;     // lanes that share a scale
  int32_t group_log;           // its elements; 31: a scale per row
  int32_t row_lanes;           // lanes of a row: whole groups
  bool stream;
};

constexpr int kRowSteps = 4;   // pieces of a lane

// Lanes of all rows lie in one line, a row's groups side by side, so that rows of
// any width fill the waves; a lane takes a piece at each of four places a block apart.
// Bound by memory: each element is read once and stays in registers between the
// largest magnitude and the codes.  8,191 rows of 16,384 bf16 by 128 70 us, 5.8 TB/s; at
// odd bytes, 16,384 of 4,095 37 us, beside 4,096 34.
template <typename T, int V>
__global__ void __launch_bounds__(kBlock) k_rows_codes(RowsArgs a) {
  const int64_t base = block_index() * (kBlock * kRowSteps);
  // the block's first row by one division, the lanes' from there in 32 bits
  const int64_t row0 = base / a.row_lanes;
  const uint32_t off = (uint32_t)(base - row0 * a.row_lanes);
  typename Raw<T, V>::vec raw[kRowSteps];
  int64_t row[kRowSteps];
  int32_t p[kRowSteps], e[kRowSteps], skip[kRowSteps];
  bool here[kRowSteps];
#pragma unroll
  for (int t = 0; t < kRowSteps; ++t) {
    const uint32_t i = off + t * kBlock + threadIdx.x;
    const uint32_t r = i / (uint32_t)a.row_lanes;
    p[t] = (int32_t)(i - r * (uint32_t)a.row_lanes);
    row[t] = row0 + r;
    here[t] = base + t * kBlock + threadIdx.x < a.lanes && p[t] < a.pieces;
    e[t] = piece_start<V>(p[t], a.dim, &skip[t]);
    raw[t] = {};
    if (here[t]) raw[t] = raw_load<T, V>(a.x.p + row[t] * a.x.stride + e[t] * (int64_t)sizeof(T));
  }
#pragma unroll
  for (int t = 0; t < kRowSteps; ++t) {
    float v[V];
    to_f32<T, V>(raw[t], v);
    const uint32_t top = lanes_max(here[t] ? magnitude<V>(v, skip[t]) : 0u, 1 << a.group_lanes_log);
    if (!here[t]) continue;
    const float scale = scale_of(__uint_as_float(top));
    const Quotient by(scale);
    if ((p[t] & ((1 << a.group_lanes_log) - 1)) == 0)
      ((float*)(a.q.scales + row[t] * a.q.sstride))[(p[t] * V) >> a.group_log] = scale;
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = by(v[k]);
    char* to = a.q.p + row[t] * a.q.stride + e[t];
    if (skip[t] == 0) {
      row_store<e4m3, V>(to, v, a.stream);
    } else {
      // the skipped elements have their own piece's scale
#pragma unroll
      for (int k = 0; k < V; ++k) {
        const float one[1] = {v[k]};
        if (k >= skip[t]) row_store<e4m3, 1>(to + k, one);
      }
    }
  }
}

// One scale for a row of more pieces than a wave: a block per row.  A lane keeps
// its first pieces in registers and reads those behind them again.
constexpr int kKeep = 4;

template <typename T, int V>
__global__ void __launch_bounds__(1024) k_wide_codes(RowsArgs a) {
  __shared__ uint32_t lds[1024 / kWave];
  const int64_t row = block_index();
  if (row >= a.n) return;      // (a grid of two dimensions is rounded up)
  const char* x = a.x.p + row * a.x.stride;
  const int32_t lanes = (int32_t)blockDim.x, l = (int32_t)threadIdx.x;
  typename Raw<T, V>::vec raw[kKeep];
  uint32_t top = 0;
#pragma unroll
  for (int t = 0; t < kKeep; ++t) {
    // lanes behind the last piece repeat it
    int32_t skip;
    const int32_t e = piece_start<V>(min(t * lanes + l, a.pieces - 1), a.dim, &skip);
    raw[t] = raw_load<T, V>(x + e * (int64_t)sizeof(T));
  }
#pragma unroll
  for (int t = 0; t < kKeep; ++t) {
    float v[V];
    to_f32<T, V>(raw[t], v);
    top = max(top, magnitude<V>(v, 0));
  }
#pragma unroll 4
  for (int32_t p = kKeep * lanes + l; p < a.pieces; p += lanes) {
    int32_t skip;
    float v[V];
    row_load<T, V>(x + piece_start<V>(p, a.dim, &skip) * (int64_t)sizeof(T), v);
    top = max(top, magnitude<V>(v, 0));
  }
  top = lanes_max(top, kWave);
  if (lane_id() == 0) lds[threadIdx.x / kWave] = top;
  __syncthreads();
  for (int i = 0; i < lanes / kWave; ++i) top = max(top, lds[i]);
  const float scale = scale_of(__uint_as_float(top));
  const Quotient by(scale);
  if (l == 0) *(float*)(a.q.scales + row * a.q.sstride) = scale;
  // (with one scale the overlap of the last two pieces is written twice alike)
  const auto write = [&](int32_t p, float (&v)[V]) {
    int32_t skip;
    const int32_t e = piece_start<V>(p, a.dim, &skip);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = by(v[k]);
    row_store<e4m3, V>(a.q.p + row * a.q.stride + e, v, a.stream);
  };
#pragma unroll
  for (int t = 0; t < kKeep; ++t)
    if (t * lanes + l < a.pieces) {
      float v[V];
      to_f32<T, V>(raw[t], v);
      write(t * lanes + l, v);
    }
#pragma unroll 4
  for (int32_t p = kKeep * lanes + l; p < a.pieces; p += lanes) {
    int32_t skip;
    float v[V];
    row_load<T, V>(x + piece_start<V>(p, a.dim, &skip) * (int64_t)sizeof(T), v);
    write(p, v);
  }
}

template <typename T>
int launch_rows(RowsArgs& a, hipStream_t stream) {
  constexpr int V = kVec<T>;
  const bool wide = a.dim >= V;
  const int vec = wide ? V : 1;
  const int32_t group = a.q.group && a.q.group < a.dim ? a.q.group : 0;
  a.pieces = (int32_t)cdiv(a.dim, vec);
  a.stream = a.n * a.dim > kStreamBytes;
  if (!group && a.pieces > kWave) {
    int threads = 128;
    while (threads < 1024 && threads * kKeep < a.pieces) threads *= 2;
    hipLaunchKernelGGL((k_wide_codes<T, V>), grid_of(a.n), dim3(threads), 0, stream, a);
    GG_LAUNCH_CHECK("k_wide_codes");
    return GG_OK;
  }
  a.group_log = 31;
  a.group_lanes_log = 0;
  if (group) {
    a.group_log = __builtin_ctz((unsigned)group);
    a.group_lanes_log = a.group_log - __builtin_ctz((unsigned)vec);
  } else {
    while ((1 << a.group_lanes_log) < a.pieces) ++a.group_lanes_log;
  }
  a.row_lanes = (int32_t)cdiv(a.pieces, 1 << a.group_lanes_log) << a.group_lanes_log;
  a.lanes = a.n * a.row_lanes;
  const dim3 grid = grid_of(cdiv(a.lanes, kBlock * kRowSteps));
  if (wide)
    hipLaunchKernelGGL((k_rows_codes<T, V>), grid, dim3(kBlock), 0, stream, a);
  else
    hipLaunchKernelGGL((k_rows_codes<T, 1>), grid, dim3(kBlock), 0, stream, a);
  GG_LAUNCH_CHECK("k_rows_codes");
  return GG_OK;
}

// ---------------------------------------------------------------------------
// Weights.
// ---------------------------------------------------------------------------
struct BlocksArgs {
  KRows x;
  KBlocks q, qt;               // p == nullptr: absent
  int64_t rows, cols;
  int32_t down, across;        // blocks
  bool shared;                 // a cache line holds codes or numbers of two blocks
};

// A workgroup per 128 x 128 elements, which stay in registers between the largest
// magnitude and the codes; the transposed codes go through LDS, four by four bytes
// at a time.  Bound by memory: 16,384 x 4,096 fp32, both ways, 83 us, 4.9 TB/s.  Blocks
// whose edges lie inside cache lines are dealt in bands of rows to the XCDs, or else
// lines go to memory in parts (8,191 x 4,095 bf16 36 us, in the order of rows 57; 8,192 x
// 4,096 24 in that order, 26 in bands).
template <typename T>
__global__ void __launch_bounds__(kBlock) k_blocks_codes(BlocksArgs a) {
  constexpr int V = kVec<T>, kLanes = kScaleBlock / V, kStep = kBlock / kLanes,
                kSteps = kScaleBlock / kStep, kPitch = kScaleBlock + 4;
  __shared__ uint32_t tile[kScaleBlock * kPitch / 4];
  __shared__ uint32_t tops[kBlock / kWave];
  // Neighbours that share lines run on one XCD, at about one time.
  const int64_t b = block_index();
  int32_t rb = (int32_t)(b / a.across), cb = (int32_t)(b - (int64_t)rb * a.across);
  if (rb >= a.down) return;    // (a grid of two dimensions is rounded up)
  if (a.shared) tile_place(a.down, a.across, &rb, &cb);
  const int64_t r0 = (int64_t)rb * kScaleBlock, c0 = (int64_t)cb * kScaleBlock;
  const int32_t nr = (int32_t)min((int64_t)kScaleBlock, a.rows - r0),
                nc = (int32_t)min((int64_t)kScaleBlock, a.cols - c0);
  const int32_t c = (int32_t)threadIdx.x % kLanes * V, r = (int32_t)threadIdx.x / kLanes;
  const char* x = a.x.p + r0 * a.x.stride + (c0 + c) * (int64_t)sizeof(T);
  float v[kSteps][V];
  uint32_t top = 0;
  // (the lanes whose piece the last column cuts read it by elements)
  typename Raw<T, V>::vec raw[kSteps] = {};
  const bool cut = c < nc && c + V > nc;
  if (c + V <= nc) {
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
      if (t * kStep + r < nr) raw[t] = raw_load<T, V>(x + (t * kStep + r) * a.x.stride);
  }
#pragma unroll
  for (int t = 0; t < kSteps; ++t) to_f32<T, V>(raw[t], v[t]);
  if (cut) {
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int k = 0; k < V; ++k) {
        float one[1] = {0.0f};
        if (t * kStep + r < nr && c + k < nc)
          row_load<T, 1>(x + (t * kStep + r) * a.x.stride + k * (int64_t)sizeof(T), one);
        v[t][k] = one[0];
      }
  }
#pragma unroll
  for (int t = 0; t < kSteps; ++t) top = max(top, magnitude<V>(v[t], 0));
  top = lanes_max(top, kWave);
  if (lane_id() == 0) tops[threadIdx.x / kWave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kBlock / kWave; ++i) top = max(top, tops[i]);
  const float scale = scale_of(__uint_as_float(top));
  const Quotient by(scale);
  if (threadIdx.x == 0) {
    if (a.q.p) ((float*)(a.q.scales + rb * a.q.sstride))[cb] = scale;
    if (a.qt.p) ((float*)(a.qt.scales + cb * a.qt.sstride))[rb] = scale;
  }
#pragma unroll
  for (int t = 0; t < kSteps; ++t) {
#pragma unroll
    for (int k = 0; k < V; ++k) v[t][k] = by(v[t][k]);
    const int32_t at = t * kStep + r;
    if (a.q.p && at < nr) {
      char* to = a.q.p + (r0 + at) * a.q.stride + c0 + c;
      if (c + V <= nc) {
        row_store<e4m3, V>(to, v[t]);
      } else {
#pragma unroll
        for (int k = 0; k < V; ++k) {
          const float one[1] = {v[t][k]};
          if (c + k < nc) row_store<e4m3, 1>(to + k, one);
        }
      }
    }
    if (a.qt.p) {
#pragma unroll
      for (int k = 0; k < V; k += 4)
        tile[(at * kPitch + c + k) / 4] = to_codes(v[t][k], v[t][k + 1], v[t][k + 2], v[t][k + 3]);
    }
  }
  if (!a.qt.p) return;
  __syncthreads();
  // Four rows by four columns a lane: a half wave's lanes lie along the rows, so
  // that they write 128 bytes of a transposed row.
#pragma unroll
  for (int t = 0; t < kScaleBlock * kScaleBlock / (16 * kBlock); ++t) {
    const int32_t i = t * kBlock + (int32_t)threadIdx.x;
    const int32_t tr = i % 32 * 4, tc = i / 32 * 4;
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = tile[((tr + k) * kPitch + tc) / 4];
    const uint32_t ab0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400),   // a0 b0 a1 b1
        ab1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602),
        cd0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400),
        cd1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602);
    const uint32_t o[4] = {__builtin_amdgcn_perm(cd0, ab0, 0x05040100),
                           __builtin_amdgcn_perm(cd0, ab0, 0x07060302),
                           __builtin_amdgcn_perm(cd1, ab1, 0x05040100),
                           __builtin_amdgcn_perm(cd1, ab1, 0x07060302)};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (tc + k >= nc) continue;
      char* to = a.qt.p + (c0 + tc + k) * a.qt.stride + r0 + tr;
      typedef uint32_t mem __attribute__((aligned(1)));
      if (tr + 4 <= nr) {
        *(GG_GLOBAL mem*)to = o[k];
      } else {
        for (int32_t j = 0; tr + j < nr; ++j) *(GG_GLOBAL uint8_t*)(to + j) = (uint8_t)(o[k] >> 8 * j);
      }
    }
  }
}

}  // namespace

int pack_blocks(const gg_blocks_t* b, const char* name, int64_t rows, int64_t cols, bool written,
                KBlocks* out) {
  GG_REQUIRE(b != nullptr, "%s: no blocks given", name);
  GG_REQUIRE(b->data != nullptr && b->scales != nullptr, "%s: data or scales are NULL", name);
  GG_REQUIRE(rows <= 1 || (b->stride >= 0 && (!written || b->stride >= cols)),
             "%s: stride %lld invalid for rows of %lld bytes", name, (long long)b->stride,
             (long long)cols);
  GG_REQUIRE((uintptr_t)b->scales % 4 == 0 && b->scales_stride % 4 == 0,
             "%s: scales are not 4-byte aligned", name);
  GG_REQUIRE(rows <= kScaleBlock || (b->scales_stride >= 0 &&
                                     (!written || b->scales_stride >= 4 * cdiv(cols, kScaleBlock))),
             "%s: scales' stride %lld invalid", name, (long long)b->scales_stride);
  out->p = (char*)b->data;
  out->stride = b->stride;
  out->scales = (char*)b->scales;
  out->sstride = b->scales_stride;
  return GG_OK;
}

}  // namespace gg

using namespace gg;

extern "C" int gg_quantise_rows(const gg_rows_t* x, int64_t n, int64_t dim, const gg_rows_t* q,
                                hipStream_t stream) {
  GG_REQUIRE(dim >= 1 && dim <= GG_QUANTISE_MAX_DIM, "dim %lld outside 1..%d", (long long)dim,
             GG_QUANTISE_MAX_DIM);
  GG_REQUIRE(n >= 0 && n <= GG_NORM_MAX_ROWS, "n = %lld unsupported", (long long)n);
  RowsArgs a = {};
  int rc = pack_rows(x, "x", n, dim, kBitFloats, false, &a.x);
  if (rc == GG_OK) rc = pack_rows(q, "q", n, dim, kBitE4M3, true, &a.q);
  if (rc != GG_OK || n == 0) return rc;
  a.n = n;
  a.dim = (int32_t)dim;
  GG_FOR_FLOAT(x->dtype, T, return launch_rows<T>(a, stream));
}

extern "C" int gg_quantise_blocks(const gg_rows_t* w, int64_t rows, int64_t cols,
                                  const gg_blocks_t* q, const gg_blocks_t* qt, hipStream_t stream) {
  GG_REQUIRE(rows >= 1 && rows <= GG_QUANTISE_MAX_DIM, "rows %lld outside 1..%d", (long long)rows,
             GG_QUANTISE_MAX_DIM);
  GG_REQUIRE(cols >= 1 && cols <= GG_QUANTISE_MAX_DIM, "cols %lld outside 1..%d", (long long)cols,
             GG_QUANTISE_MAX_DIM);
  GG_REQUIRE(q || qt, "no output asked for");
  BlocksArgs a = {};
  int rc = pack_rows(w, "w", rows, cols, kBitFloats, false, &a.x);
  if (rc == GG_OK && q) rc = pack_blocks(q, "q", rows, cols, true, &a.q);
  if (rc == GG_OK && qt) rc = pack_blocks(qt, "qt", cols, rows, true, &a.qt);
  if (rc != GG_OK) return rc;
  a.rows = rows;
  a.cols = cols;
  a.across = (int32_t)cdiv(cols, kScaleBlock);
  a.down = (int32_t)cdiv(rows, kScaleBlock);
  const dim3 grid = grid_of((int64_t)a.down * a.across);
  a.shared = grid.y == 1 && ((uintptr_t)a.x.p | (uintptr_t)a.x.stride | (uintptr_t)a.q.p | (uintptr_t)a.q.stride |
                             (uintptr_t)a.qt.p | (uintptr_t)a.qt.stride) % kScaleBlock != 0;
  GG_FOR_FLOAT(w->dtype, T, {
    hipLaunchKernelGGL((k_blocks_codes<T>), grid, dim3(kBlock), 0, stream, a);
  });
  GG_LAUNCH_CHECK("k_blocks_codes");
  return GG_OK;
}
