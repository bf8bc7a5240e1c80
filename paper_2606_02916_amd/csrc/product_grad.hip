// The gradient of 8-bit weights from the 8-bit rows that the forward product took:
//   dw[j][c] = sum_i dz[i][j] a[i][c],   a[i][c] = code[i][c] * scale[i][c / 128].
#include "product.hpp"

namespace gg {
namespace {

typedef short v4s __attribute__((ext_vector_type(4)));

struct GradArgs {
  KRows a, dz, dw;
  int64_t n, chunk;            // rows, and those of a split
  int32_t k, m;
  int32_t per_row;             // a has one scale a row
  int32_t add;
  int32_t tiles_k, tiles_j, splits;
  float* part;                 // [splits][m][k] where there are several
};

constexpr int32_t kTileK = kScaleBlock;    // columns of a tile: one scale of each row
constexpr int32_t kTileI = 32;             // rows of a step

// Scaled gradients as bf16 numbers that add up to them.  The codes are bf16 numbers
// themselves, so products are exact and sums fp32.  One part for bf16 results (2^-8 of a
// term at most, the rounding that the result itself gets, and less of a sum of many), two for
// fp16 (2^-15), three for fp32, which are the fp32 number.
// An infinity or a NaN is whole in the first part, and the parts behind an infinity are those
// of the largest number of its sign, which cannot cancel it.
template <int PARTS>
__device__ __forceinline__ void split(float x, float y, uint32_t (&p)[PARTS]) {
  const auto rounded = [](float a, float b) {
    const v2bf v = {(bf16)a, (bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  };
  const auto upper = [](float a, float b) {
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302);
  };
  const auto lower = [](float a) { return a - __uint_as_float(__float_as_uint(a) & 0xffff0000u); };
  if constexpr (PARTS == 1) {
    p[0] = rounded(x, y);
  } else {
    p[0] = upper(x, y);
    x = lower(__builtin_amdgcn_fmed3f(x, -kLargest, kLargest));
    y = lower(__builtin_amdgcn_fmed3f(y, -kLargest, kLargest));
    if constexpr (PARTS == 2) {
      p[1] = rounded(x, y);
    } else {
      p[1] = upper(x, y);
      p[2] = upper(lower(x), lower(y));
    }
  }
}

// Four columns of a row of fp32 sums, and what dw holds there: with `add` read before, all of a
// wave's that can be under way together (1 row of 8,960 x 19,904 fp32 added 331 us, 622 when
// each was read before it was written).
template <typename O>
__device__ __forceinline__ void load_old(const GradArgs& a, int32_t j, int32_t c, float (&v)[4]) {
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = 0.0f;
  if (!a.add) return;
  const char* from = a.dw.p + j * a.dw.stride + c * (int64_t)sizeof(O);
  if (c + 4 <= a.k) {
    row_load<O, 4>(from, v);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      float one[1] = {};
      if (c + r < a.k) row_load<O, 1>(from + r * sizeof(O), one);
      v[r] = one[0];
    }
  }
}

template <typename O>
__device__ __forceinline__ void store_sums(const GradArgs& a, int32_t j, int32_t c, const float (&f)[4],
                                           const float (&old)[4]) {
  char* to = a.dw.p + j * a.dw.stride + c * (int64_t)sizeof(O);
  float v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = old[r] + f[r];
  if (c + 4 <= a.k) {
    row_store<O, 4>(to, v);
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float one[1] = {v[r]};
      if (c + r < a.k) row_store<O, 1>(to + r * sizeof(O), one);
    }
  }
}

// A wave's sums into dw, or into its split's.
template <typename O, int TK, int TJ>
__device__ __forceinline__ void store_tile(const GradArgs& a, int32_t part, int32_t c0, int32_t j0,
                                           int32_t l, const v4f (&acc)[TK][TJ]) {
#pragma unroll
  for (int t = 0; t < TJ; ++t) {
    const int32_t j = j0 + t * 16 + l % 16;
    if (j >= a.m) continue;
    float old[TK][4];
    if (!a.part) {
#pragma unroll
      for (int u = 0; u < TK; ++u) {
        const int32_t c = c0 + u * 16 + l / 16 * 4;
        if (c < a.k) load_old<O>(a, j, c, old[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < TK; ++u) {
      const int32_t c = c0 + u * 16 + l / 16 * 4;
      if (c >= a.k) continue;
      const float f[4] = {acc[u][t][0], acc[u][t][1], acc[u][t][2], acc[u][t][3]};
      if (a.part) {
        float* to = a.part + ((int64_t)part * a.m + j) * a.k + c;
        if (c + 4 <= a.k) {
          row_store<float, 4>((char*)to, f);
        } else {
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (c + r < a.k) to[r] = f[r];
        }
      } else {
        store_sums<O>(a, j, c, f, old[u]);
      }
    }
  }
}

// The transposing read: 16 lanes' four elements of 8 bytes, lanes 4 r .. 4 r + 3 at row r's
// 16 columns; lane c of them gets column c of the four rows.
__device__ __forceinline__ v4s read_across(const void* p) {
  typedef __attribute__((address_space(3))) v4s* at;
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)p);
}

__device__ __forceinline__ v8bf both(v4s lo, v4s hi) {
  return __builtin_bit_cast(v8bf, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// bf16 gradients into bf16 weights' gradients: tiles of 256 columns of a by 256 of dz, 64
// rows at a time.  The gradients go to LDS as they are, without a register between; codes
// times their scales are rounded to bf16 on the way (2^-8 of a term at most, as the
// result itself, of which the sum over 16,384 rows is 2.3e-3 off instead of 1.7e-3, root mean
// squares), which is a quarter of the matrix unit's time in other operations, where
// scaled gradients, a version for each 128 columns, are more than all of it.  LDS holds
// rows of 512 bytes, unit u of 32 bytes in place u ^ (row & 7), so that the eight rows
// that half a wave reads across meet all banks.  Wave (wk, wj) has 128 x 64 of the tile.
constexpr int32_t kWideK = 256, kWideJ = 256, kWideI = 64;

__global__ void __launch_bounds__(512) k_product_grad_wide(GradArgs a) {
  constexpr int TK = 8, TJ = 4, kRowBytes = 512;
  __shared__ __attribute__((aligned(16))) char la[2][kWideI * kRowBytes], lz[2][kWideI * kRowBytes];
  const int32_t tid = (int32_t)threadIdx.x, l = lane_id(),
                wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t wk = wave % 2, wj = wave / 2;
  int32_t tk0, tj0;
  tile_place(a.tiles_k, a.tiles_j, &tk0, &tj0);
  const int32_t c0 = tk0 * kWideK, j0 = tj0 * kWideJ;
  const int64_t first = blockIdx.y * a.chunk, end = min(a.n, first + a.chunk);

  // Codes: 16 of a row, of two rows, a lane; a unit of LDS each.  Columns behind the last
  // ones may hold anything, they are columns of no result; the piece that holds the last
  // one is read from 16 before the row's end and moved down.
  const int32_t ra = tid / 16, ua = tid % 16, ca = c0 + ua * 16, cl = min(ca, a.k - 16);
  const bool edge = c0 + kWideK > a.k;
  const int32_t scale_col = a.per_row ? 0 : min(ca, a.k - 1) / kScaleBlock * 4;
  const char* code_at = a.a.p + (first + ra) * a.a.stride + cl;
  const char* scale_at = a.a.scales + (first + ra) * a.a.sstride + scale_col;
  const int64_t code_half = 32 * a.a.stride, scale_half = 32 * a.a.sstride;
  v4i codes[2];
  float scale[2];
  // Gradients: a wave's load brings two rows, 16 bytes a lane; columns behind the last ones
  // repeat them.
  const char* zp = a.dz.p + (first + wave * 2) * a.dz.stride;
  const int32_t uz = l % 32 / 2, hz = l % 2;
  uint32_t z_off[4];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const int32_t r = t * 16 + wave * 2 + l / 32;
    const int32_t j = min(j0 + ((uz ^ (r & 7)) * 2 + hz) * 8, a.m - 8);
    z_off[t] = (uint32_t)(t * 16 + l / 32) * (uint32_t)a.dz.stride + (uint32_t)j * 2;
  }
  const auto put = [&](v4i code, float scale, int32_t r, int buf) {
    if (edge) code = move_down(code, ca - cl);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(code[i], false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(code[i], true);
      const v2bf p = {(bf16)(lo[0] * scale), (bf16)(lo[1] * scale)},
                 q = {(bf16)(hi[0] * scale), (bf16)(hi[1] * scale)};
      w[2 * i] = __builtin_bit_cast(uint32_t, p);
      w[2 * i + 1] = __builtin_bit_cast(uint32_t, q);
    }
    v4i* to = (v4i*)&la[buf][r * kRowBytes + (ua ^ (r & 7)) * 32];
    to[0] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    to[1] = v4i{(int)w[4], (int)w[5], (int)w[6], (int)w[7]};
  };
  typedef v4i mem __attribute__((aligned(1)));
  // a step of 64 rows: gradients to LDS, codes to registers
  const auto bring = [&](int buf) {
#pragma unroll
    for (int t = 0; t < 4; ++t)
      load_to_lds16(zp, z_off[t], lds_at(&lz[buf][(t * 16 + wave * 2) * kRowBytes]));
    zp += kWideI * a.dz.stride;
  };
  const auto fetch = [&] {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      codes[t] = *(const GG_GLOBAL mem*)(code_at + t * code_half);
      scale[t] = *(const GG_GLOBAL float*)(scale_at + t * scale_half);
    }
  };
  const auto next_codes = [&] {
    code_at += 2 * code_half;
    scale_at += 2 * scale_half;
  };
  // fewer rows, with zeros behind them
  const auto fetch_last = [&](int32_t rows, int buf) {
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
      const bool here = t * 32 + ra < rows;
      v4i code = {};
      if (here) code = *(const GG_GLOBAL mem*)(code_at + t * code_half);
      put(code, here ? *(const GG_GLOBAL float*)(scale_at + t * scale_half) : 0.0f, t * 32 + ra, buf);
    }
#pragma unroll 1
    for (int t = 0; t < 4; ++t) {
      const int32_t r = t * 16 + wave * 2 + l / 32;
      const int32_t j = min(j0 + ((uz ^ (r & 7)) * 2 + hz) * 8, a.m - 8);
      v4i v = {};
      if (r < rows) v = *(const GG_GLOBAL v4i*)(zp + (t * 16 + l / 32) * a.dz.stride + j * 2LL);
      *(v4i*)&lz[buf][(t * 16 + wave * 2) * kRowBytes + l * 16] = v;
    }
  };
  // A unit's 16 columns of rows 4 q .. 4 q + 3 for lanes 16 q .. 16 q + 15 and of the rows 16
  // behind them.
  const int32_t tr = l % 16 / 4 + l / 16 * 4;
  const auto operand = [&](const char* rows, int32_t unit) {
    const char* p = rows + tr * kRowBytes + ((unit ^ (tr & 7)) * 32 + l % 4 * 8);
    return both(read_across(p), read_across(p + 16 * kRowBytes));
  };
  v4f acc[TK][TJ] = {};
  // A step's products; `more`: the next step's codes, which are in registers, go to LDS
  // meanwhile, and those after it are read.  In this order: the operand of the next products
  // before these, and other operations between products.
  const auto add = [&](int buf, bool more, auto then) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const char *pa = la[buf] + h * 32 * kRowBytes, *pz = lz[buf] + h * 32 * kRowBytes;
      v8bf x[TK], z[2];
      z[0] = operand(pz, wj * TJ);
#pragma unroll
      for (int u = 0; u < TK; ++u) x[u] = operand(pa, wk * TK + u);
#pragma unroll
      for (int t = 0; t < TJ; ++t) {
        if (t + 1 < TJ) z[t + 1 & 1] = operand(pz, wj * TJ + t + 1);
#pragma unroll
        for (int u = 0; u < TK; ++u)
          acc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u], z[t & 1], acc[u][t], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        if (h == 0 && more && t < 2) put(codes[t], scale[t], t * 32 + ra, buf ^ 1);
        if (h == 0 && more && t == 2) then();
      }
    }
  };
  const auto nothing = [] {};
  const int64_t rows = max(end - first, (int64_t)0);
  const int32_t steps = (int32_t)(rows / kWideI), rest = (int32_t)(rows % kWideI);
  int buf = 0;
  if (steps) {
    bring(0);
    fetch();
    next_codes();
#pragma unroll
    for (int t = 0; t < 2; ++t) put(codes[t], scale[t], t * 32 + ra, 0);
    if (steps > 1) fetch();
    for (int32_t s = 1; s < steps; ++s) {
      // All of a step's loads are there.  (Leaving those of codes under way, whose number the
      // compiler chooses, takes 912 us instead of 916 of 16,384 rows, 4,096 x 8,192.)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
      add(buf, true, [&] {
        // (behind the codes' use: the compiler's wait for them would be one for these too)
        bring(buf ^ 1);
        next_codes();
        if (s + 1 < steps) fetch();
      });
      buf ^= 1;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    add(buf, false, nothing);
    buf ^= 1;
  }
  if (rest) {
    fetch_last(rest, buf);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    add(buf, false, nothing);
  }
  store_tile<bf16, TK, TJ>(a, blockIdx.y, c0 + wk * TK * 16, j0 + wj * TJ * 16, l, acc);
}

// Every other gradient: a tile of 128 columns of a by BJ of dz, 32 rows at a time through
// LDS.  Both operands of the MFMA run along the rows, which lie across both matrices: LDS
// keeps them as they come, and the transposing reads hand a lane four rows' elements of
// its column.  A row of the tile is 32 bytes longer than its elements, so that the 4 x 32
// bytes of such a read meet different banks.  Codes are turned into bf16 and gradients
// scaled and split once, on the way into LDS, two steps after they were asked for.
// Wave (wk, wj) has 64 x BJ/2 of the tile.  Columns behind the last ones may hold anything,
// they are columns of no result; the piece that holds the last one is read from its own
// length before the row's end and moved down, but with TINY, for rows shorter than a
// piece, which are read by elements.
template <typename Z, typename O, int PARTS, int BJ, bool TINY>
__global__ void __launch_bounds__(kBlock, 2) k_product_grad(GradArgs a) {
  constexpr int TK = 4, TJ = BJ / 32, V = kVec<Z>;
  constexpr int kPitchA = kTileK + 16, kPitchZ = BJ + 16;
  constexpr int kLanesZ = BJ / V, kStepZ = kBlock / kLanesZ, kLoadsZ = kTileI / kStepZ;
  static_assert(kTileI * kTileK == kBlock * 16 && kTileI % kStepZ == 0, "a step's loads");
  __shared__ __attribute__((aligned(16))) short la[2][kTileI * kPitchA];
  __shared__ __attribute__((aligned(16))) short lz[2][PARTS][kTileI * kPitchZ];
  const int32_t tid = (int32_t)threadIdx.x, l = lane_id(),
                wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t wk = wave % 2, wj = wave / 2;
  // the tiles of a split, which read the same rows, next to each other on one XCD
  const uint32_t place = xcd_turn(blockIdx.y * gridDim.x + blockIdx.x, gridDim.x * gridDim.y);
  const int32_t part = (int32_t)(place / gridDim.x), tile = (int32_t)(place % gridDim.x);
  const int32_t c0 = tile % a.tiles_k * kTileK, j0 = tile / a.tiles_k * BJ;
  const int64_t first = part * a.chunk, end = min(a.n, first + a.chunk);

  // a step's loads: 16 codes a lane, and kLoadsZ pieces of gradients with their rows' scales
  typedef v4i mem __attribute__((aligned(1)));
  const int32_t ra = tid / 8, ca = c0 + tid % 8 * 16, rz = tid / kLanesZ, cz = j0 + tid % kLanesZ * V;
  const int32_t cl = TINY ? ca : min(ca, a.k - 16), zl = TINY ? cz : min(cz, a.m - V);
  const bool edge_a = c0 + kTileK > a.k, edge_z = j0 + BJ > a.m;
  const char* code_at = a.a.p + (first + ra) * a.a.stride + cl;
  const char* z_at = a.dz.p + (first + rz) * a.dz.stride + zl * (int64_t)sizeof(Z);
  const char* scale_at =
      a.a.scales + (first + rz) * a.a.sstride + (a.per_row ? 0 : c0 / kScaleBlock * 4LL);
  struct Step {
    v4i codes, z[kLoadsZ];
    float scale[kLoadsZ];
  };
  // `rows`: as many of the step's are there (all of them but for a last step); then on by
  // `by` rows
  const auto fetch = [&](Step& s, auto whole, int32_t rows, int32_t by) {
    const bool here = whole || ra < rows;
    s.codes = {};
    if constexpr (TINY) {
      if (here) s.codes = load_codes(code_at - cl, cl, a.k);
    } else if (here) {
      s.codes = *(const GG_GLOBAL mem*)code_at;
    }
#pragma unroll
    for (int t = 0; t < kLoadsZ; ++t) {
      s.z[t] = {};
      s.scale[t] = 0.0f;
      const char* p = z_at + t * kStepZ * a.dz.stride;
      if (whole || t * kStepZ + rz < rows) {
        s.scale[t] = *(const GG_GLOBAL float*)(scale_at + t * kStepZ * a.a.sstride);
        if constexpr (TINY) {
          typename Raw<Z, V>::vec v = {};
#pragma unroll
          for (int x = 0; x < V; ++x)
            if (cz + x < a.m) v[x] = raw_load<Z, 1>(p + x * sizeof(Z));
          s.z[t] = __builtin_bit_cast(v4i, v);
        } else {
          s.z[t] = *(const GG_GLOBAL mem*)p;
        }
      }
    }
    code_at += by * a.a.stride;
    z_at += by * a.dz.stride;
    scale_at += by * a.a.sstride;
  };
  const auto keep = [&](const Step& s, int buf) {
    const v4i codes = !TINY && edge_a ? move_down(s.codes, ca - cl) : s.codes;
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      w[2 * i] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[i], 1.0f, false));
      w[2 * i + 1] = __builtin_bit_cast(
          uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[i], 1.0f, true));
    }
    v4i* to = (v4i*)&la[buf][ra * kPitchA + (ca - c0)];
    to[0] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    to[1] = v4i{(int)w[4], (int)w[5], (int)w[6], (int)w[7]};
#pragma unroll
    for (int t = 0; t < kLoadsZ; ++t) {
      const v4i z = !TINY && edge_z ? move_down(s.z[t], (cz - zl) * (int32_t)sizeof(Z)) : s.z[t];
      float v[V];
      to_f32<Z, V>(__builtin_bit_cast(typename Raw<Z, V>::vec, z), v);
      uint32_t p[V / 2][PARTS];
#pragma unroll
      for (int x = 0; x < V / 2; ++x)
        split<PARTS>(v[2 * x] * s.scale[t], v[2 * x + 1] * s.scale[t], p[x]);
#pragma unroll
      for (int q = 0; q < PARTS; ++q) {
        uint32_t* at = (uint32_t*)&lz[buf][q][(t * kStepZ + rz) * kPitchZ + (cz - j0)];
#pragma unroll
        for (int x = 0; x < V / 2; ++x) at[x] = p[x][q];
      }
    }
  };
  // rows 4 q .. 4 q + 3 and 16 + them for lanes 16 q .. 16 q + 15, a column each
  const int32_t tr = l % 16 / 4 + l / 16 * 4, tc = l % 4 * 4;
  const auto operand = [&](const short* tile, int pitch, int32_t col) {
    const short* p = tile + tr * pitch + col + tc;
    return both(read_across(p), read_across(p + 16 * pitch));
  };
  v4f acc[TK][TJ] = {};
  const auto add = [&](int buf) {
    v8bf x[TK];
#pragma unroll
    for (int u = 0; u < TK; ++u) x[u] = operand(la[buf], kPitchA, (wk * TK + u) * 16);
#pragma unroll
    for (int t = 0; t < TJ; ++t)
#pragma unroll
      for (int q = PARTS - 1; q >= 0; --q) {
        const v8bf z = operand(lz[buf][q], kPitchZ, (wj * TJ + t) * 16);
#pragma unroll
        for (int u = 0; u < TK; ++u)
          acc[u][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[u], z, acc[u][t], 0, 0, 0);
      }
  };
  const int64_t rows = max(end - first, (int64_t)0);
  const int32_t steps = (int32_t)(rows / kTileI), rest = (int32_t)(rows % kTileI);
  const std::true_type whole;
  Step s[2];
  int32_t i = 0;
  // step i's rows are in LDS and step i + 1's on their way; behind the last whole step its
  // rows are read again
  const auto step = [&](Step& now, const Step& next) {
    __syncthreads();
    fetch(now, whole, 0, i + 3 < steps ? kTileI : 0);
    add(i & 1);
    keep(next, ~i & 1);
    ++i;
  };
  if (steps) {
    fetch(s[0], whole, 0, steps > 1 ? kTileI : 0);
    fetch(s[1], whole, 0, steps > 2 ? kTileI : 0);
    keep(s[0], 0);
    while (i + 2 < steps) {
      step(s[0], s[1]);
      step(s[1], s[0]);
    }
    if (i + 1 < steps) step(s[0], s[1]);
    __syncthreads();
    add(i & 1);
    ++i;
  }
  if (rest) {
    // (the pointers are at the last whole step's rows)
    if (steps) {
      code_at += kTileI * a.a.stride;
      z_at += kTileI * a.dz.stride;
      scale_at += kTileI * a.a.sstride;
    }
    fetch(s[0], std::false_type(), rest, 0);
    keep(s[0], i & 1);
    __syncthreads();
    add(i & 1);
  }
  store_tile<O, TK, TJ>(a, part, c0 + wk * TK * 16, j0 + wj * TJ * 16, l, acc);
}

// The splits' sums, in an order that depends on their number: a block's waves take them in
// turn and are added up in theirs.  64 x 4 columns a block.
constexpr int kJoinWaves = 16;

template <typename O>
__global__ void __launch_bounds__(kJoinWaves* kWave) k_product_join(GradArgs a) {
  __shared__ v4f lds[kJoinWaves][kWave];
  const int32_t across = (a.k + 3) / 4, l = lane_id(), wave = (int32_t)threadIdx.x / kWave,
                waves = (int32_t)blockDim.x / kWave;
  const int64_t i = (int64_t)blockIdx.x * kWave + l;
  const bool here = i < (int64_t)a.m * across;
  const int32_t j = here ? (int32_t)(i / across) : 0, c = here ? (int32_t)(i - (int64_t)j * across) * 4 : 0;
  const float* p = a.part + (int64_t)j * a.k + c;
  const int64_t step = (int64_t)a.m * a.k;
  v4f f = {};
  if (here && c + 4 <= a.k) {
#pragma unroll 4
    for (int32_t s = wave; s < a.splits; s += waves) {
      float v[4];
      row_load<float, 4>((const char*)(p + s * step), v);
#pragma unroll
      for (int r = 0; r < 4; ++r) f[r] += v[r];
    }
  } else if (here) {
    for (int32_t s = wave; s < a.splits; s += waves)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (c + r < a.k) f[r] += p[s * step + r];
  }
  lds[wave][l] = f;
  __syncthreads();
  if (wave || !here) return;
  for (int32_t w = 1; w < waves; ++w) f += lds[w][l];
  const float sums[4] = {f[0], f[1], f[2], f[3]};
  float old[4];
  load_old<O>(a, j, c, old);
  store_sums<O>(a, j, c, sums, old);
}

// Which kernel and how many splits of the rows: the least of a sum of measured
// microseconds, with as many splits as fill the chip or a power of two, whose blocks
// go evenly to its parts.  A step of 32 rows takes a block of 128 x 128 alone on its CU 0.5,
// 0.8 and 1.15 with one, two and three parts, a block of 64 columns of dz 0.38, 0.55 and 0.73;
// two on a CU take 1.35 and three 1.85 times as long for each.  The wide kernel, one block
// on a CU, takes 1.4 for 64 rows while half the chip has none and 1.75 behind that, and 8 more
// to begin and end.  Splits cost a second launch, 4, and their sums' way to memory and
// back at 6.5 MB/us.  (bf16, 1,024 rows: 4,096 x 4,096 45 us wide, 50 in tiles of 128; 2,048
// x 2,048 22 in tiles of 128 of all rows, 34 in two splits or wide; 512 rows of
// 1,024 x 1,024 9 in tiles of 64, 12 of 128, 21 wide.  233,000 rows of 602 x 41 fp32 78 with 768 blocks, 81 with 512.)
struct GradShape {
  int bj;                      // kWideJ: the wide kernel
  int64_t tiles_k, tiles_j, splits;
  float cost;
};

GradShape tiles_of(int64_t k, int64_t m, int bj) {
  return {bj, cdiv(k, bj == kWideJ ? kWideK : kTileK), cdiv(m, bj), 0, 0.0f};
}

int blocks_on_a_cu(int bj) { return bj == kWideJ ? 1 : bj == 128 ? 2 : 3; }

// as many as fill the chip's 256 CUs, of 64 rows at least
int64_t most_splits(const GradShape& s, int64_t n) {
  const int64_t blocks = 256 * blocks_on_a_cu(s.bj);
  return std::max<int64_t>(1, std::min(blocks / (s.tiles_k * s.tiles_j), cdiv(n, kWideI)));
}

GradShape shape_of(int64_t n, int64_t k, int64_t m, int parts, int bj) {
  static constexpr float kStep[2][3] = {{0.38f, 0.55f, 0.73f}, {0.5f, 0.8f, 1.15f}},
                         kShared[4] = {0.0f, 1.0f, 1.35f, 1.85f};
  GradShape best = tiles_of(k, m, bj);
  const int64_t tiles = best.tiles_k * best.tiles_j, held = blocks_on_a_cu(bj);
  for (int64_t s = most_splits(best, n), next = 1; s; s = next / 2) {
    for (next = 1; next < s;) next *= 2;
    const int64_t blocks = tiles * s, chunk = cdiv(n, s), rounds = blocks / (256 * held),
                  rest = blocks % (256 * held);
    float cost;
    if (bj == kWideJ)
      cost = 8 + (rounds + (rest > 0)) * cdiv(chunk, kWideI) * (blocks <= 128 ? 1.4f : 1.75f);
    else
      cost = (rounds * kShared[held] + kShared[cdiv(rest, 256)]) * cdiv(chunk, kTileI) *
             kStep[bj == 128][parts - 1];
    if (s > 1) cost += 4 + (float)s * m * k * (8 / 6.5e6f);
    if (best.splits && cost >= best.cost) continue;
    best.splits = s;
    best.cost = cost;
  }
  return best;
}

template <typename Z, typename O, int PARTS>
int launch_grad(GradArgs& a, hipStream_t stream) {
  GradShape s = shape_of(a.n, a.k, a.m, PARTS, 64);
  const auto or_else = [&](int bj) {
    const GradShape t = shape_of(a.n, a.k, a.m, PARTS, bj);
    if (t.cost < s.cost) s = t;
  };
  if (a.m > 64 && a.k >= 16) or_else(128);
  // (the wide kernel moves whole pieces of 16 bytes of the gradients, with offsets of 32 bits)
  if (std::is_same<Z, bf16>::value && std::is_same<O, bf16>::value && a.m % 8 == 0 && a.m >= 128 &&
      a.k >= 128 && a.n >= 128 && aligned16(a.dz.p) && a.dz.stride % 16 == 0 && a.dz.stride <= 1 << 25)
    or_else(kWideJ);
  a.tiles_k = (int32_t)s.tiles_k;
  a.tiles_j = (int32_t)s.tiles_j;
  a.splits = (int32_t)s.splits;
  a.chunk = align_up(cdiv(a.n, s.splits), kWideI);
  if (s.splits == 1) a.part = nullptr;
  const dim3 grid((unsigned)(s.tiles_k * s.tiles_j), (unsigned)s.splits);
  if (s.bj == kWideJ)
    hipLaunchKernelGGL(k_product_grad_wide, grid, dim3(512), 0, stream, a);
  else if (a.m < kVec<Z> || a.k < 16)
    hipLaunchKernelGGL((k_product_grad<Z, O, PARTS, 64, true>), grid, dim3(kBlock), 0, stream, a);
  else if (s.bj == 64)
    hipLaunchKernelGGL((k_product_grad<Z, O, PARTS, 64, false>), grid, dim3(kBlock), 0, stream, a);
  else
    hipLaunchKernelGGL((k_product_grad<Z, O, PARTS, 128, false>), grid, dim3(kBlock), 0, stream, a);
  GG_LAUNCH_CHECK("k_product_grad");
  if (a.part) {
    int waves = 1;
    while (waves < kJoinWaves && waves < a.splits) waves *= 2;
    hipLaunchKernelGGL((k_product_join<O>), dim3((unsigned)cdiv(a.m * cdiv(a.k, 4), kWave)),
                       dim3(waves * kWave), 0, stream, a);
    GG_LAUNCH_CHECK("k_product_join");
  }
  return GG_OK;
}

}  // namespace
}  // namespace gg

using namespace gg;

static bool grad_sizes(int64_t n, int64_t k, int64_t m) {
  return n >= 0 && n <= GG_PRODUCT_MAX_ROWS && k >= 1 && k <= GG_PRODUCT_MAX_DIM && m >= 1 &&
         m <= GG_PRODUCT_MAX_DIM;
}

extern "C" size_t gg_ws_product(int64_t n, int64_t k, int64_t m) {
  if (!grad_sizes(n, k, m)) return 0;
  // (whichever tiles are taken)
  int64_t splits = 1;
  for (const int bj : {64, 128, kWideJ}) splits = std::max(splits, most_splits(tiles_of(k, m, bj), n));
  return splits > 1 ? align_up((size_t)splits * m * k * sizeof(float), 256) : 0;
}

extern "C" int gg_product_backward(const gg_rows_t* a, int64_t n, int64_t k, const gg_rows_t* dz,
                                   int64_t m, const gg_rows_t* dw, int32_t flags, void* ws,
                                   size_t ws_bytes, hipStream_t stream) {
  GG_REQUIRE(n >= 0 && n <= GG_PRODUCT_MAX_ROWS, "n = %lld unsupported", (long long)n);
  GG_REQUIRE(k >= 1 && k <= GG_PRODUCT_MAX_DIM, "k %lld outside 1..%d", (long long)k,
             GG_PRODUCT_MAX_DIM);
  GG_REQUIRE(m >= 1 && m <= GG_PRODUCT_MAX_DIM, "m %lld outside 1..%d", (long long)m,
             GG_PRODUCT_MAX_DIM);
  GG_REQUIRE((flags & ~GG_PRODUCT_ADD) == 0, "unknown flags %d", flags);
  GradArgs p = {};
  int rc = pack_rows(a, "a", n, k, kBitE4M3, false, &p.a);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(p.a.group == 0 || p.a.group == kScaleBlock, "a: group %d is neither 0 nor %d", p.a.group,
             kScaleBlock);
  rc = pack_rows(dz, "dz", n, m, kBitFloats, false, &p.dz);
  if (rc == GG_OK) rc = pack_rows(dw, "dw", m, k, (1u << dz->dtype) | kBitF32, true, &p.dw);
  if (rc != GG_OK) return rc;
  const size_t need = gg_ws_product(n, k, m);
  GG_REQUIRE(need == 0 || (ws && (uintptr_t)ws % 16 == 0 && ws_bytes >= need),
             "workspace of %zu bytes < %zu, or not aligned", ws_bytes, need);
  GG_REQUIRE(cdiv(k, kTileK) * cdiv(m, 64) <= kGridX * 4, "%lld x %lld: too many tiles", (long long)m,
             (long long)k);
  p.n = n;
  p.k = (int32_t)k;
  p.m = (int32_t)m;
  p.per_row = p.a.group == 0;
  p.add = flags & GG_PRODUCT_ADD;
  p.part = (float*)ws;
  if (n == 0 && p.add) return GG_OK;
  GG_FOR_FLOAT(dz->dtype, Z, {
    if (dw->dtype == GG_F32) return launch_grad<Z, float, 3>(p, stream);
    if constexpr (sizeof(Z) == 2) return launch_grad<Z, Z, std::is_same<Z, f16>::value ? 2 : 1>(p, stream);
    return GG_ERR_UNSUPPORTED;
  });
}
