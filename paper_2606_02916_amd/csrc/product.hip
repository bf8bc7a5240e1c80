// The product of 8-bit rows with 8-bit weights:
//   out[i][j] = sum_g sa[i][g] sb[j / 128][g] sum_{k in block g} a[i][k] b[j][k],
// codes multiplied by matrix instructions over a block of 128, each block's sum scaled
// and added in fp32.
#include "product.hpp"

namespace gg {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int32_t kBlockK = kScaleBlock;   // bytes of a row in a step

struct ProductArgs {
  KRows a, out;
  KBlocks b;
  int64_t n;
  int32_t k, m, kb;            // kb: blocks of k
  int32_t per_row;             // a has one scale a row
  int32_t scales16;            // four blocks' scales of a row, and of weights, are aligned, and
                               // k is whole fours of blocks
  int32_t tiles_i, tiles_j;
};

// A lane's 32 codes as the operand of a product of 16 rows by 16 rows over 128
// columns.  Which columns a lane has does not matter, both operands agree on it.
//
// The 8-bit matrix instructions add eight products at a time (a lane's codes 8 c .. 8 c +
// 7) and drop, towards zero, what lies below 2^-13 of the largest one's power of two:
// 2^-16 of the result where codes are normally distributed, 2^-14 where they are spread
// over many powers of two.  That is well below the rounding of a 16-bit output (2^-9,
// 2^-12) and not of a 32-bit one, whose codes are multiplied as bf16: exact products,
// added in fp32, at half the rate.
//
// Weights are multiplied with the power of two of their scale on the way (`power`, its
// exponent with fp32's bias): the 8-bit instructions take one, and so does the conversion to
// bf16, exactly.  (8,191 x 4,096 to 16,384 523 us, without 515: the instruction is longer.)
constexpr int32_t kNoPower = 127;

template <bool EXACT>
struct Codes {
  v8i v;
  __device__ __forceinline__ void set(v4i lo, v4i hi, int32_t power = kNoPower) {
    v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
};
template <>
struct Codes<true> {
  v8bf v[4];
  __device__ __forceinline__ void set(v4i lo, v4i hi, int32_t power = kNoPower) {
    const float two = __uint_as_float((uint32_t)power << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int w0 = i < 2 ? lo[2 * i] : hi[2 * i - 4], w1 = i < 2 ? lo[2 * i + 1] : hi[2 * i - 3];
      const v2bf p[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w0, two, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w0, two, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w1, two, false),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)w1, two, true)};
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = p[j / 2][j % 2];
    }
  }
};

__device__ __forceinline__ v4f multiply(const Codes<false>& weights, const Codes<false>& rows, int32_t power) {
  // e4m3 by e4m3
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(weights.v, rows.v, v4f{}, 0, 0, 0, power, 0,
                                                          kNoPower);
}
__device__ __forceinline__ v4f multiply(const Codes<true>& a, const Codes<true>& b, int32_t) {
  v4f d = {};
#pragma unroll
  for (int i = 0; i < 4; ++i) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], d, 0, 0, 0);
  return d;
}

// A scale of weights in two factors, 2^(power - 127) and the rest.  The product of two scales
// may pass fp32's range where the result, a block's sum of up to 2^25 and down to 2^-18 times
// it, does not (rows of gradients of 1e-35): the power goes to the codes, and a row's scale times
// the rest is as far from the range's ends as the row's scale.  The power itself is kept from
// taking a block's sum out of the range; then one of both scales is so small or large that the
// result is out of it too.
struct Scale {
  int32_t power;
  float rest;
  __device__ __forceinline__ explicit Scale(float s) {
    power = min(max((int32_t)(__float_as_uint(s) >> 23 & 255), kNoPower - 108), kNoPower + 102);
    rest = __builtin_amdgcn_ldexpf(s, kNoPower - power);
  }
};

// Which of a wave's weights' rows a lane multiplies: of each 16 G rows, G products take four of
// every 4 G, so that a lane ends with 4 G columns side by side of a row of the output, and a
// row's four lanes with 16 G: whole cache lines in 16 bits with G = 4 (8,191 x 4,096 to 16,384
// 527 us, with G = 1 553; 10,610 of 128 to 36,776 204 and 232).
template <typename O, int TJ>
constexpr int kSide = sizeof(O) == 4 ? 1 : TJ < 4 ? TJ : 4;

template <int G>
__device__ __forceinline__ int32_t lane_row(int32_t l) {
  return l % 16 / 4 * (4 * G) + l % 4;
}
template <int G>
__device__ __forceinline__ constexpr int32_t product_row(int u) {
  return u / G * (16 * G) + u % G * 4;
}
// Where a row's pieces are in LDS: piece c in place c ^ key.  The sixteen rows of a product have
// each key twice, in rows of 128 bytes of either half of the banks.
template <int G>
__device__ __forceinline__ int32_t row_key(int32_t r) {
  return (r >> 1 & 1) | (r / (4 * G) & 3) << 1;
}

// A lane's codes of a row in LDS: its pieces q and q + 4, q = l / 16.  Its rows have one key,
// l / 2 & 7.  The sixteen lanes that LDS serves at a time are 0-3, 12-15, 20-23 and 24-27,
// and their like: eight rows' piece q and the other eight's piece q ^ 1, all in different
// banks.  (With pieces 2 q and 2 q + 1 the same reads take twice as long.)
template <typename C>
__device__ __forceinline__ C operand(const v4i* row, int32_t l, int32_t power = kNoPower) {
  const int32_t c = l / 16 ^ (l >> 1 & 7);
  C v;
  v.set(row[c], row[c ^ 4], power);
  return v;
}

// Codes at any byte.  The memory reads 16 bytes that begin inside a word in 2.8 times
// the time of 16 that begin with one (1 row of 4,096 to 16,384 37 us and 13.5), and so
// the whole words that hold a piece's bytes are read, and moved down to its place p.
__device__ __forceinline__ v4i words_from(const v4i& w, int32_t next, uint32_t p) {
  const uint32_t skip = p & 3;
  return v4i{(int)__builtin_amdgcn_alignbyte(w[1], w[0], skip), (int)__builtin_amdgcn_alignbyte(w[2], w[1], skip),
             (int)__builtin_amdgcn_alignbyte(w[3], w[2], skip), (int)__builtin_amdgcn_alignbyte(next, w[3], skip)};
}
typedef v4i words4 __attribute__((aligned(4)));

// A lane's codes of a row in LDS whose words begin `skip` bytes before the row: the words
// behind pieces q and q + 4 are the next pieces' first ones, and behind the last one, `end`.
template <typename C>
__device__ __forceinline__ C operand_of_words(const v4i* row, const int32_t* end, uint32_t skip, int32_t l,
                                              int32_t power = kNoPower) {
  const int32_t q = l / 16, turn = l >> 1 & 7, c = q ^ turn;
  const int32_t next = row[q + 1 ^ turn][0];
  const int32_t* far = q == 3 ? end : (const int32_t*)(row + (q + 5 ^ turn));
  C v;
  v.set(words_from(row[c], next, skip), words_from(row[c ^ 4], *far, skip), power);
  return v;
}

// The products of a wave's TJ x TI operands from LDS, added to acc with the scales of
// its rows.  A product's sum is scaled kLag products later, when the matrix unit has it,
// and the weights of the next 16 rows are read before this one's products; kept in
// this order for many products and for fp32 results (10,610 rows of 128 to 36,776 bf16 204 us, 207
// otherwise; 8,191 of 4,096 to 16,384 fp32 1,028 and 1,053).  Of few the compiler's order hides more
// of what comes before the first, the weights' power (300 rows of 8,192 to 1,024 bf16 16.6 us, in
// this one 17.6).  weights(r) and rows(r): the operands of this lane's row r; `power`: the weights'.
template <int TJ, int TI, typename C, typename W, typename R>
__device__ __forceinline__ void multiply_step(const float (&scale)[TI], int32_t power, v4f (&acc)[TJ][TI],
                                              W weights, R rows) {
  constexpr int N = TJ * TI, kLag = N > 3 ? 3 : N - 1;
  constexpr bool kOrdered = N >= 16 || std::is_same<C, Codes<true>>::value;
  C r[TI], w[2];
  v4f d[N];
  w[0] = weights(0);
#pragma unroll
  for (int t = 0; t < TI; ++t) r[t] = rows(t * 16);
#pragma unroll
  for (int x = 0; x < N + kLag; ++x) {
    const int u = x / TI, t = x % TI, y = x - kLag;
    if (x < N) {
      if (t == 0 && u + 1 < TJ) w[u + 1 & 1] = weights((u + 1) * 16);
      d[x] = multiply(w[u & 1], r[t], power);
    }
    if (y >= 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        acc[y / TI][y % TI][i] = __builtin_fmaf(d[y][i], scale[y % TI], acc[y / TI][y % TI][i]);
    }
    if constexpr (kOrdered) __builtin_amdgcn_sched_barrier(0);
  }
}

// Sixteen numbers of two bytes to any multiple of two: stores of 16 bytes that begin inside a
// word are split by the memory, and so between a first and a last number go words
// (10,239 rows of 114 to 53,277 fp16 450 us, 531 without).
template <typename O>
__device__ __forceinline__ void store_run(char* to, const float (&f)[16]) {
  typedef uint32_t w4 __attribute__((ext_vector_type(4), aligned(4)));
  typedef uint32_t w3 __attribute__((ext_vector_type(3), aligned(4)));
  typedef O two __attribute__((ext_vector_type(2)));
  uint32_t w[8];
#pragma unroll
  for (int x = 0; x < 8; ++x) w[x] = __builtin_bit_cast(uint32_t, two{(O)f[2 * x], (O)f[2 * x + 1]});
  if ((uintptr_t)to & 2) {
    uint32_t v[7];
#pragma unroll
    for (int x = 0; x < 7; ++x) v[x] = __builtin_amdgcn_alignbyte(w[x + 1], w[x], 2);
    *(GG_GLOBAL uint16_t*)to = (uint16_t)w[0];
    *(GG_GLOBAL w4*)(to + 2) = w4{v[0], v[1], v[2], v[3]};
    *(GG_GLOBAL w3*)(to + 18) = w3{v[4], v[5], v[6]};
    *(GG_GLOBAL uint16_t*)(to + 30) = (uint16_t)(w[7] >> 16);
  } else {
    *(GG_GLOBAL w4*)to = w4{w[0], w[1], w[2], w[3]};
    *(GG_GLOBAL w4*)(to + 16) = w4{w[4], w[5], w[6], w[7]};
  }
}

// A wave's sums, G products' columns side by side.
template <typename O, int G, int TJ, int TI>
__device__ __forceinline__ void store_tile(const ProductArgs& a, int64_t i0, int32_t j0, int32_t l,
                                           const v4f (&acc)[TJ][TI], int64_t first = 0) {
  constexpr int kRun = 4 * G;                    // columns of a lane
#pragma unroll
  for (int t = 0; t < TI; ++t) {
    const int64_t i = i0 + t * 16 + l % 16;
    if (i < first || i >= a.n) continue;
    char* const row = a.out.p + i * a.out.stride;
#pragma unroll
    for (int u = 0; u < TJ; u += G) {
      const int32_t j = j0 + product_row<G>(u) + l / 16 * kRun;
      float f[kRun];
#pragma unroll
      for (int x = 0; x < kRun; ++x) f[x] = acc[u + x / 4][t][x % 4];
      if (j + kRun <= a.m) {
        if constexpr (kRun == 16)
          store_run<O>(row + j * (int64_t)sizeof(O), f);
        else
          row_store<O, kRun>(row + j * (int64_t)sizeof(O), f);
      } else {
#pragma unroll
        for (int x = 0; x < kRun; ++x) {
          const float one[1] = {f[x]};
          if (j + x < a.m) row_store<O, 1>(row + (j + x) * (int64_t)sizeof(O), one);
        }
      }
    }
  }
}

// A tile of BJ weights' rows by BI rows of a, blocks of 128 bytes of k at a time
// through LDS.  A row of a block is eight pieces of 16 bytes, placed by its key.  Wave (wj,
// wi) has BJ/WJ x BI/WI of the tile, weights as the rows of the MFMA's result, so that a
// lane has one row's scale to apply and neighbours to store.
//
// Pieces of whole words go from memory to LDS without a register between, STAGES - 1 steps
// ahead, and the scales with them, so that the wait for a step can count the loads behind it.  A step has WK blocks of k, each for WJ x WI waves, whose
// sums are added at the end: few rows' steps are short, and so there are half as
// many.  A step at k's end that is not whole comes through registers, with zeros
// behind the end.  BYTES: rows may begin inside a word; the words that hold a row's block
// are brought, with one more for each row, and moved down as operands are read (8,191 x
// 4,096 to 16,384 bf16 with weights one byte off 870 us, through registers with 16 bytes from any
// place 1,470; rows 4,097 apart 990).
template <typename O, int BJ, int BI, int WJ, int WI, int WK, int STAGES, bool BYTES>
__global__ void __launch_bounds__(WJ* WI* WK* kWave, BI > 32 ? 2 : 1) k_product_pipe(ProductArgs a) {
  constexpr int kThreads = WJ * WI * WK * kWave, kGroup = kThreads / WK, kPieces = (BJ + BI) * 8,
                kLoads = kPieces * WK / kThreads, kBlocksJ = (BJ + kScaleBlock - 1) / kScaleBlock;
  constexpr int TJ = BJ / WJ / 16, TI = BI / WI / 16, G = kSide<O, TJ>;
  static_assert(kPieces % kGroup == 0, "whole loads");
  static_assert(BJ / WJ <= kScaleBlock && kScaleBlock % (BJ / WJ) == 0, "one block of weights a wave");
  static_assert(BI + kBlocksJ <= kGroup, "a lane for each scale");
  static_assert(!BYTES || BJ + BI <= kGroup, "a lane for each row");
  constexpr int kBehind = (kLoads + 1 + BYTES) * (STAGES - 2);   // loads that may be under way
  static_assert(kBehind < 64, "the counter of loads");
  typedef Codes<sizeof(O) == 4> C;
  __shared__ v4i lds[STAGES][WK][kPieces];
  __shared__ float scales[STAGES][kThreads];
  __shared__ int32_t ends[BYTES ? STAGES : 1][BYTES ? kThreads : 1];
  const int32_t l = lane_id(),
                wave_all = __builtin_amdgcn_readfirstlane((int32_t)threadIdx.x / kWave);
  // a group of waves brings its own block of a step and multiplies it
  const int32_t wk = wave_all / (WJ * WI), wave = wave_all % (WJ * WI), tid = wave * kWave + l;
  const int32_t wj = wave % WJ, wi = wave / WJ;
  int32_t ti0, tj0;
  tile_place(a.tiles_i, a.tiles_j, &ti0, &tj0);
  const int64_t i0 = (int64_t)ti0 * BI;
  const int32_t j0 = tj0 * BJ;

  // the pieces that this lane brings: rows behind the last one repeat it
  const char* const jbase = a.b.p + j0 * a.b.stride;
  const char* const ibase = a.a.p + i0 * a.a.stride;
  const int32_t jlast = min(a.m - j0, BJ) - 1, ilast = (int32_t)min(a.n - i0, (int64_t)BI) - 1;
  const auto piece_of = [&](int32_t r) { return (tid % 8 ^ (r < BJ ? row_key<G>(r) : row_key<1>(r))) * 16; };
  const auto row_of = [&](int t, int64_t* off) {
    const int32_t r = (t * kGroup + tid) / 8;
    *off = r < BJ ? min(r, jlast) * a.b.stride : min(r - BJ, ilast) * a.a.stride;
    return r;
  };
  // (BYTES: whole words, from the one with a row's first byte on)
  const uint32_t jskip = BYTES ? (uintptr_t)jbase & 3 : 0, iskip = BYTES ? (uintptr_t)ibase & 3 : 0;
  uint32_t from[kLoads];
#pragma unroll
  for (int t = 0; t < kLoads; ++t) {
    int64_t off;
    const int32_t r = row_of(t, &off);
    from[t] = ((uint32_t)off + (r < BJ ? jskip : iskip) & (BYTES ? ~3u : ~0u)) + piece_of(r);
  }
  // and of row tid the word with the last byte of a block
  const char* end_from = nullptr;
  if constexpr (BYTES) {
    const char* p = tid < BJ ? jbase + min(tid, jlast) * a.b.stride : ibase + min(tid - BJ, ilast) * a.a.stride;
    end_from = (const char*)((uintptr_t)(p + kBlockK - 1) & ~(uintptr_t)3);
  }
  // its scale: a row's, or behind them a block's of weights
  const char* scale_from;
  int32_t scale_step = a.per_row ? 0 : 4;
  if (tid < BI) {
    scale_from = a.a.scales + (i0 + min(tid, ilast)) * a.a.sstride;
  } else {
    scale_from = a.b.scales + min(j0 + min(tid - BI, kBlocksJ - 1) * kScaleBlock, a.m - 1) /
                                  kScaleBlock * a.b.sstride;
    scale_step = 4;
  }
  const int32_t whole = a.k / (kBlockK * WK), steps = (a.kb + WK - 1) / WK;
  const auto bring = [&](int32_t s, int slot) {
    const int32_t g = s * WK + wk;
    v4i* const to = lds[slot][wk];
    if (s < whole) {
      const char *jp = jbase - jskip + (int64_t)g * kBlockK, *ip = ibase - iskip + (int64_t)g * kBlockK;
#pragma unroll
      for (int t = 0; t < kLoads; ++t) {
        // (a load's 64 lanes are of one matrix: BJ is a multiple of 8)
        const bool weights = (t * kGroup + wave * kWave) / 8 < BJ;
        load_to_lds16(weights ? jp : ip, from[t], lds_at(to + t * kGroup + wave * kWave));
      }
      if constexpr (BYTES)
        load_to_lds4(end_from + (int64_t)g * kBlockK, lds_at(&ends[slot][wave_all * kWave]));
    } else {
      v4i got[kLoads];
#pragma unroll
      for (int t = 0; t < kLoads; ++t) {
        int64_t off;
        const int32_t r = row_of(t, &off);
        got[t] = codes_read((r < BJ ? jbase : ibase) + off, g * kBlockK + piece_of(r), a.k);
      }
#pragma unroll
      for (int t = 0; t < kLoads; ++t) {
        const int32_t r = (t * kGroup + tid) / 8;
        to[t * kGroup + tid] = codes_moved(got[t], g * kBlockK + piece_of(r), a.k);
      }
    }
    load_to_lds4(scale_from + (int64_t)min(g, a.kb - 1) * scale_step,
                 lds_at(&scales[slot][wave_all * kWave]));
  };

  // bytes before this lane's rows, the same for all of them, which are fours apart
  const int32_t wrow = wj * TJ * 16 + lane_row<G>(l), rrow = wi * TI * 16 + l % 16;
  const uint32_t wskip = jskip + (uint32_t)wrow * (uint32_t)a.b.stride,
                 rskip = iskip + (uint32_t)rrow * (uint32_t)a.a.stride;
  v4f acc[TJ][TI] = {};
#pragma unroll
  for (int s = 0; s < STAGES - 1; ++s)
    if (s < steps) bring(s, s);
  int slot = 0;
  for (int32_t s = 0; s < steps; ++s) {
    // step s is here, in all waves' parts, and step s - 1 has been read
    if (s + STAGES - 2 < whole)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kBehind) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (s + STAGES - 1 < steps) bring(s + STAGES - 1, slot ? slot - 1 : STAGES - 1);
    if (WK == 1 || s * WK + wk < a.kb) {
      const float* sc = scales[slot] + wk * kGroup;
      const Scale sb(sc[BI + wj * TJ * 16 / kScaleBlock]);
      float scale[TI];
#pragma unroll
      for (int t = 0; t < TI; ++t) scale[t] = sc[(wi * TI + t) * 16 + l % 16] * sb.rest;
      const v4i *w = lds[slot][wk] + wrow * 8, *r = lds[slot][wk] + (BJ + rrow) * 8;
      if constexpr (BYTES) {
        const int32_t *we = ends[slot] + wk * kGroup + wrow, *re = ends[slot] + wk * kGroup + BJ + rrow;
        // (a step at k's end has its codes in place)
        const uint32_t ws = s < whole ? wskip : 0, rs = s < whole ? rskip : 0;
        multiply_step<TJ, TI, C>(scale, sb.power, acc,
                                 [&](int x) { return operand_of_words<C>(w + product_row<G>(x / 16) * 8, we + product_row<G>(x / 16), ws, l, sb.power); },
                                 [&](int x) { return operand_of_words<C>(r + x * 8, re + x, rs, l); });
      } else {
        multiply_step<TJ, TI, C>(scale, sb.power, acc,
                                 [&](int x) { return operand<C>(w + product_row<G>(x / 16) * 8, l, sb.power); },
                                 [&](int x) { return operand<C>(r + x * 8, l); });
      }
    }
    slot = slot + 1 < STAGES ? slot + 1 : 0;
  }
  if constexpr (WK > 1) {
    // the groups' sums, in order
    typedef v4f Sums[TJ * TI][kWave];
    static_assert(sizeof(Sums) * WJ * WI <= sizeof(lds), "room for a group's sums");
    Sums* sums = (Sums*)&lds[0][0][0] + wave;
#pragma unroll
    for (int x = 1; x < WK; ++x) {
      __syncthreads();
      if (wk == x)
#pragma unroll
        for (int y = 0; y < TJ * TI; ++y) (*sums)[y][l] = acc[y / TI][y % TI];
      __syncthreads();
      if (wk == 0)
#pragma unroll
        for (int y = 0; y < TJ * TI; ++y) acc[y / TI][y % TI] += (*sums)[y][l];
    }
    if (wk) return;
  }
  store_tile<O, G, TJ, TI>(a, i0 + wi * TI * 16, j0 + wj * TJ * 16, l, acc);
}

// Tiles of 256 x 256 of rows that begin with words, two blocks of k in LDS.  One wait a block, before its last quarter of
// products: the next block has been on its way since the same place in the block before,
// and its first operands are read into the registers that the last products leave.
// 8,191 x 4,096 to 16,384 bf16 take 524 us, 2,100 TFLOP/s (515 to 545 on different cards).
// Of 535 432 are left without the loads, 370 without the scaling too: products, their scaling
// and LDS's reads do not quite overlap (a wave's products alone would be 240), and the loads'
// requests come on top.
template <typename O>
__global__ void __launch_bounds__(512, 2) k_product_wide(ProductArgs a) {
  constexpr int BJ = 256, BI = 256, WJ = 2, WI = 4, TJ = BJ / WJ / 16, TI = BI / WI / 16, G = kSide<O, TJ>, kThreads = 512;
  typedef Codes<false> C;
  __shared__ v4i lds[2][(BJ + BI) * 8];
  __shared__ v4f scales[2][kThreads];
  const int32_t tid = (int32_t)threadIdx.x, l = lane_id(),
                wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t wj = wave % WJ, wi = wave / WJ;
  int32_t ti0, tj0;
  tile_place(a.tiles_i, a.tiles_j, &ti0, &tj0);
  // the last tile of rows reaches back instead of over their end
  const int64_t i0 = min((int64_t)ti0 * BI, a.n - BI);
  const int32_t skip = (int32_t)((int64_t)ti0 * BI - i0);
  const int32_t j0 = tj0 * BJ;

  // The pieces that this lane brings: of row tid / 8 and those 64, 128 and 192 behind it, of
  // weights and of a; weights' rows behind the last one repeat it.
  const char* const jbase = a.b.p + j0 * a.b.stride;
  const char* const ibase = a.a.p + i0 * a.a.stride;
  const int32_t jlast = min(a.m - j0, BJ) - 1;
  // (rows 64 apart have one key)
  const int32_t jpiece = (tid % 8 ^ row_key<G>(tid / 8)) * 16, ipiece = (tid % 8 ^ row_key<1>(tid / 8)) * 16;
  uint32_t jfrom[4];
#pragma unroll
  for (int t = 0; t < 4; ++t)
    jfrom[t] = (uint32_t)min(t * 64 + tid / 8, jlast) * (uint32_t)a.b.stride + jpiece;
  const uint32_t ifrom = (uint32_t)(tid / 8) * (uint32_t)a.a.stride + ipiece;
  // its scale: a row's, or behind them a block's of weights
  const bool of_row = tid < BI;
  const char* const scale_from =
      of_row ? a.a.scales + (i0 + tid) * a.a.sstride
             : a.b.scales + min(j0 + min(tid - BI, 1) * kScaleBlock, a.m - 1) / kScaleBlock * a.b.sstride;
  const int32_t scale_step = of_row && a.per_row ? 0 : 4;
  // Scales come for four blocks at a time where they lie on 16-byte boundaries (each
  // lane's is in a line of its own: one for each block takes 547 us instead of 529, 8,191 x
  // 4,096 to 16,384), for one at a time elsewhere.
  const bool fours = a.scales16;
  const int32_t whole = a.k / kBlockK;
  // Each XCD's blocks begin at another block of k, so that rows a power of two apart do
  // not all ask the same part of memory (529 us instead of 550).
  const int32_t turn = (int32_t)(blockIdx.x % kXcds) * whole / kXcds / 4 * 4;
  const auto at = [&](int32_t g) {
    const int32_t x = g + turn;
    return x >= whole ? x - whole : x;
  };
  const auto bring_scale = [&](int32_t g, int slot) {
    load_to_lds4(scale_from + g * scale_step, lds_at((float*)scales[slot] + wave * kWave));
  };
  const auto bring_scales = [&](int32_t g) {
    if (!fours)
      bring_scale(at(g), g & 1);
    else if (g % 4 == 0)
      load_to_lds16_at(scale_from + at(g) * 4, lds_at(scales[g / 4 & 1] + wave * kWave));
  };
  const auto bring = [&](int32_t g, int slot) {
    const char *jp = jbase + (int64_t)at(g) * kBlockK, *ip = ibase + (int64_t)at(g) * kBlockK;
    const uint32_t to = lds_at(lds[slot] + wave * kWave);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      load_to_lds16(jp, jfrom[t], to + t * kThreads * 16);
      load_to_lds16(ip + t * 64 * a.a.stride, ifrom, to + (t + 4) * kThreads * 16);
    }
    bring_scales(g);
  };

  const auto wait = [] { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
  constexpr int kEarly = TJ - 2;      // 16-row pieces of weights before the wait
  v4f acc[TJ][TI] = {};
  C rows[TI], w[4];
  float scale[TI], held[2] = {};
  int32_t power = kNoPower;           // of this block's weights
  v4f d[3] = {};                      // products whose sums are not scaled yet
  const auto weights = [&](int buf, int u) {
    return operand<C>(lds[buf] + (wj * TJ * 16 + lane_row<G>(l) + product_row<G>(u)) * 8, l);
  };
  const auto row = [&](int buf, int t) {
    return operand<C>(lds[buf] + (BJ + wi * TI * 16 + l % 16) * 8 + t * 128, l);
  };
  const auto add = [&](int u, int t, const v4f& x, float s) {
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[u][t][i] = __builtin_fmaf(x[i], s, acc[u][t][i]);
    // (here, not behind the wait, where all of them would have to be held for)
    asm volatile("" : "+v"(acc[u][t]));
  };
  const auto product = [&](const C& x, const C& y) {
    v4f z = multiply(x, y, power);
    // (here, not where its sum is scaled, which may be behind the wait or the next block's scales)
    asm volatile("" : "+v"(z));
    return z;
  };
  const int32_t held_log = fours ? 2 : 0;
  const auto scale_at = [&](int32_t g) {
    return (const float*)scales[g >> held_log & 1] + (g & (1 << held_log) - 1);
  };
  const int32_t apart = fours ? 4 : 1, of_weights = (BI + wj) * apart, of_rows = (wi * TI * 16 + l % 16) * apart;
  const auto read_scales = [&](const float* sc, const Scale& sb) {
    power = sb.power;
#pragma unroll
    for (int t = 0; t < TI; ++t) scale[t] = sc[of_rows + t * 16 * apart] * sb.rest;
  };
  if (whole) {
    bring(0, 0);
    wait();
    if (whole > 1) bring(1, 1);
    read_scales(scale_at(0), Scale(scale_at(0)[of_weights]));
    w[0] = weights(0, 0);
    w[1] = weights(0, 1);
#pragma unroll
    for (int t = 0; t < TI; ++t) rows[t] = row(0, t);
  }
  for (int32_t g = 0; g < whole; ++g) {
    const int buf = g & 1;
#pragma unroll
    for (int x = 0; x < kEarly * TI; ++x) {
      const int u = x / TI, t = x % TI;
      if (t == 0) w[(u + 2) % 4] = weights(buf, u + 2);
      const v4f z = product(w[u % 4], rows[t]);
      if (x == 0) add(TJ - 1, 2, d[0], held[0]);
      if (x == 1) add(TJ - 2, 3, d[1], held[1]);
      if (x == 2) add(TJ - 1, 3, d[2], held[1]);
      if (x >= 3) add((x - 3) / TI, (x - 3) % TI, d[x % 3], scale[(x - 3) % TI]);
      d[x % 3] = z;
      __builtin_amdgcn_sched_barrier(0);
    }
    // the next block is here, and this one has been read; what is read of the next one
    // meets the rest of this one's products
    wait();
    if (g + 2 < whole) bring(g + 2, buf);
    // (its products wait for this one)
    const float next = scale_at(g + 1)[of_weights];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int y = 0; y < 2 * TI; ++y) {
      const int x = kEarly * TI + y, u = kEarly + y % 2, t = y / 2;
      const v4f z = product(w[u % 4], rows[t]);
      // (the tile three products before)
      const int v = y - 3;
      if (v < 0)
        add((x - 3) / TI, (x - 3) % TI, d[x % 3], scale[(x - 3) % TI]);
      else
        add(kEarly + v % 2, v / 2, d[x % 3], scale[v / 2]);
      d[x % 3] = z;
      if (y % 2) rows[t] = row(buf ^ 1, t);
      if (y < 2) w[y] = weights(buf ^ 1, y);
      __builtin_amdgcn_sched_barrier(0);
    }
    held[0] = scale[2];
    held[1] = scale[3];
    read_scales(scale_at(g + 1), Scale(next));
    static_assert(TI == 4 && (kEarly * TI + 2 * TI) % 3 == 2 && TJ % 4 == 0, "the order of d and w");
    const v4f z = d[2];
    d[2] = d[1];
    d[1] = d[0];
    d[0] = z;
  }
  add(TJ - 1, 2, d[0], held[0]);
  add(TJ - 2, 3, d[1], held[1]);
  add(TJ - 1, 3, d[2], held[1]);
  if (whole < a.kb) {
    // the block at k's end, zeros behind it (the empty statement keeps what is needed here
    // only from being computed before the loop, whose registers are all taken)
    int32_t lane = tid;
    asm volatile("" : "+v"(lane));
    __syncthreads();
    bring_scale(whole, 0);
    const auto column_of = [&](int t) {
      return whole * kBlockK + (lane % 8 ^ (t < 4 ? row_key<G>(lane / 8) : row_key<1>(lane / 8))) * 16;
    };
    v4i got[8];
#pragma unroll
    for (int t = 0; t < 8; ++t) {
      const int32_t r = t % 4 * 64 + lane / 8;
      got[t] = codes_read(t < 4 ? jbase + min(r, jlast) * a.b.stride : ibase + r * a.a.stride, column_of(t), a.k);
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) lds[0][t * kThreads + lane] = codes_moved(got[t], column_of(t), a.k);
    wait();
    const float* sc = (const float*)scales[0];
    const Scale end(sc[BI + wj]);
    power = end.power;
#pragma unroll
    for (int t = 0; t < TI; ++t) scale[t] = sc[(wi * TI + t) * 16 + l % 16] * end.rest;
    multiply_step<TJ, TI, C>(scale, power, acc, [&](int x) { return weights(0, x / 16); },
                             [&](int x) { return row(0, x / 16); });
  }
  store_tile<O, G, TJ, TI>(a, i0 + wi * TI * 16, j0 + wj * TJ * 16, l, acc, i0 + skip);
}

// Tiles of matrices with more than 2^23 bytes from a row to the next: blocks come through
// registers.
template <typename O, int BJ, int BI, int WJ, int WI>
__global__ void __launch_bounds__(WJ* WI* kWave, sizeof(O) == 4 ? 1 : 2) k_product_tile(ProductArgs a) {
  constexpr int kThreads = WJ * WI * kWave, kRows = kThreads / 8, kLoads = (BJ + BI) / kRows,
                kLoadsJ = BJ / kRows;
  constexpr int TJ = BJ / WJ / 16, TI = BI / WI / 16;
  static_assert(BJ % kRows == 0 && BI % kRows == 0 && BJ / WJ <= kScaleBlock, "tile");
  typedef Codes<sizeof(O) == 4> C;
  __shared__ v4i lds[2][(BJ + BI) * 8];
  const int32_t tid = (int32_t)threadIdx.x, l = lane_id(),
                wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int32_t wj = wave % WJ, wi = wave / WJ;
  int32_t ti0, tj0;
  tile_place(a.tiles_i, a.tiles_j, &ti0, &tj0);
  const int64_t i0 = (int64_t)ti0 * BI;
  const int32_t j0 = tj0 * BJ;

  // the rows of this lane's pieces: those behind the last one repeat it
  const int32_t slot = tid % 8;
  const char* row[kLoads];
#pragma unroll
  for (int t = 0; t < kLoads; ++t) {
    const int32_t r = t * kRows + tid / 8;
    row[t] = t < kLoadsJ ? a.b.p + min(j0 + r, a.m - 1) * a.b.stride
                         : a.a.p + min(i0 + (r - BJ), a.n - 1) * a.a.stride;
  }
  v4i got[kLoads];
  const auto fetch = [&](int32_t g) {
#pragma unroll
    for (int t = 0; t < kLoads; ++t)
      got[t] = load_codes(row[t], g * kBlockK + (slot ^ ((t * kRows + tid / 8) >> 1 & 7)) * 16, a.k);
  };
  const auto keep = [&](int buf) {
#pragma unroll
    for (int t = 0; t < kLoads; ++t) lds[buf][t * kThreads + tid] = got[t];
  };
  // scales: of this lane's rows, and of the wave's block of weights
  const char* row_scale[TI];
#pragma unroll
  for (int t = 0; t < TI; ++t)
    row_scale[t] = a.a.scales + min(i0 + (wi * TI + t) * 16 + l % 16, a.n - 1) * a.a.sstride;
  const char* block_scale =
      a.b.scales + min(j0 + wj * TJ * 16, a.m - 1) / kScaleBlock * a.b.sstride;
  float sa[TI], sb;
  const auto scales = [&](int32_t g) {
    sb = *(const float*)(block_scale + 4 * g);
#pragma unroll
    for (int t = 0; t < TI; ++t) sa[t] = *(const GG_GLOBAL float*)(row_scale[t] + (a.per_row ? 0 : 4 * g));
  };

  v4f acc[TJ][TI] = {};
  fetch(0);
  scales(0);
  keep(0);
  for (int32_t g = 0; g < a.kb; ++g) {
    const int buf = g & 1;
    __syncthreads();
    const Scale of_weights(sb);
    float scale[TI];
#pragma unroll
    for (int t = 0; t < TI; ++t) scale[t] = sa[t] * of_weights.rest;
    const bool more = g + 1 < a.kb;
    if (more) {
      fetch(g + 1);
      scales(g + 1);
    }
    const v4i *w = lds[buf] + (wj * TJ * 16 + l % 16) * 8, *r = lds[buf] + (BJ + wi * TI * 16 + l % 16) * 8;
    multiply_step<TJ, TI, C>(scale, of_weights.power, acc,
                             [&](int x) { return operand<C>(w + x * 8, l, of_weights.power); },
                             [&](int x) { return operand<C>(r + x * 8, l); });
    if (more) keep(buf ^ 1);
  }
  store_tile<O, 1, TJ, TI>(a, i0 + wi * TI * 16, j0 + wj * TJ * 16, l, acc);
}

// Few rows: operands go from memory to registers, without LDS.  A block has 16 weights' rows
// and 16 rows of a; its waves take the blocks of k in turn, with no wait for each
// other, the next two's operands loaded before these two's products, and their sums are
// added in the order of the waves' halves.  Bound by the weights' bytes (1 row of
// 4,096 to 16,384 bf16 12.9 us, 5.2 TB/s), and for more rows by those of a, which every block
// reads from the caches.  BYTES: rows may begin inside a word.
constexpr int kFewWaves = 8;

template <typename O, bool BYTES>
__global__ void __launch_bounds__(kFewWaves* kWave, 2) k_product_few(ProductArgs a) {
  constexpr int kAhead = 2;                      // blocks of k in a step
  typedef Codes<sizeof(O) == 4> C;
  __shared__ v4f lds[kFewWaves / 2][kWave];
  const int32_t l = lane_id(),
                wave = __builtin_amdgcn_readfirstlane((int32_t)threadIdx.x / kWave),
                waves = (int32_t)blockDim.x / kWave;
  int32_t ti0, tj0;
  tile_place(a.tiles_i, a.tiles_j, &ti0, &tj0);
  const int32_t j0 = tj0 * 16;
  const int64_t i0 = (int64_t)ti0 * 16;
  // rows behind the last one repeat it
  const char* const wbase = a.b.p + j0 * a.b.stride;
  const char* const rbase = a.a.p + i0 * a.a.stride;
  const char* const sbase = a.a.scales + i0 * a.a.sstride;
  const char* const wscale = a.b.scales + j0 / kScaleBlock * a.b.sstride;
  const int32_t r = (int32_t)min(a.n - i0 - 1, (int64_t)(l % 16));
  const uint32_t w_off = (uint32_t)min(l % 16, a.m - j0 - 1) * (uint32_t)a.b.stride,
                 r_off = (uint32_t)r * (uint32_t)a.a.stride, s_off = (uint32_t)r * (uint32_t)a.a.sstride;
  const int32_t whole = a.k / kBlockK, lane_c = l / 16 * 32;
  // 32 codes of a row, and with BYTES the word with the last one
  struct Piece {
    v4i w[2];
    int32_t last;
    __device__ __forceinline__ void load(const char* base, uint32_t off) {
      const uint32_t skip = BYTES ? (uint32_t)(uintptr_t)base + off & 3 : 0;
      const uintptr_t p = (uintptr_t)base + off - skip;
#pragma unroll
      for (int x = 0; x < 2; ++x) w[x] = *(const GG_GLOBAL words4*)(p + 16 * x);
      if (BYTES) last = *(const GG_GLOBAL int32_t*)(p + (skip ? 32 : 28));
    }
    __device__ __forceinline__ C codes(const char* base, uint32_t off, int32_t power = kNoPower) const {
      C c;
      if constexpr (BYTES) {
        const uint32_t p = (uint32_t)(uintptr_t)base + off;
        c.set(words_from(w[0], w[1][0], p), words_from(w[1], last, p), power);
      } else {
        c.set(w[0], w[1], power);
      }
      return c;
    }
  };
  struct Step {
    Piece w[kAhead], r[kAhead];
    float sb[kAhead], sa[kAhead];
  };
  const auto load_scales = [&](int32_t g, int h, Step& s) {
    s.sb[h] = *(const float*)(wscale + 4LL * g);
    s.sa[h] = *(const GG_GLOBAL float*)(sbase + (a.per_row ? 0 : 4LL * g) + s_off);
  };
  const auto load = [&](int32_t g0, Step& s) {
#pragma unroll
    for (int h = 0; h < kAhead; ++h) {
      const int32_t g = g0 + h * waves;
      if (g >= whole) break;
      load_scales(g, h, s);
      s.w[h].load(wbase + (int64_t)g * kBlockK, w_off + lane_c);
      s.r[h].load(rbase + (int64_t)g * kBlockK, r_off + lane_c);
    }
  };
  v4f acc[1][1] = {};
  const auto add = [&](const C& w, const C& r, int32_t power, float scale) {
    const v4f d = multiply(w, r, power);
#pragma unroll
    for (int x = 0; x < 4; ++x) acc[0][0][x] = __builtin_fmaf(d[x], scale, acc[0][0][x]);
  };
  const auto add_all = [&](int32_t g0, const Step& s) {
#pragma unroll
    for (int h = 0; h < kAhead; ++h) {
      if (g0 + h * waves >= whole) break;
      const Scale sb(s.sb[h]);
      add(s.w[h].codes(wbase, w_off, sb.power), s.r[h].codes(rbase, r_off), sb.power, s.sa[h] * sb.rest);
    }
  };
  Step s[2];
  const int32_t step = waves * kAhead;
  load(wave, s[0]);
  for (int32_t g = wave; g < whole; g += 2 * step) {
    load(g + step, s[1]);
    add_all(g, s[0]);
    if (g + step >= whole) break;
    load(g + 2 * step, s[0]);
    add_all(g + step, s[1]);
  }
  if (whole < a.kb && whole % waves == wave) {   // the block at k's end
    load_scales(whole, 0, s[0]);
    const auto end_of = [&](const char* row, int32_t power = kNoPower) {
      const int32_t c = whole * kBlockK + lane_c;
      C codes;
      codes.set(load_codes(row, c, a.k), load_codes(row, c + 16, a.k), power);
      return codes;
    };
    const Scale sb(s[0].sb[0]);
    add(end_of(wbase + w_off, sb.power), end_of(rbase + r_off), sb.power, s[0].sa[0] * sb.rest);
  }
  for (int32_t half = waves / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (wave >= half && wave < 2 * half) lds[wave - half][l] = acc[0][0];
    __syncthreads();
    if (wave < half) acc[0][0] += lds[wave][l];
  }
  if (wave == 0) store_tile<O, 1, 1, 1>(a, i0, j0, l, acc);
}

int tiles_of(ProductArgs& a, int bj, int bi) {
  a.tiles_i = (int32_t)cdiv(a.n, bi);
  a.tiles_j = (int32_t)cdiv(a.m, bj);
  GG_REQUIRE((int64_t)a.tiles_i * a.tiles_j <= kGridX * 4, "%lld x %d: too many tiles", (long long)a.n, a.m);
  return GG_OK;
}

// Both matrices' rows begin with a word.
bool in_words(const ProductArgs& a) {
  return ((uintptr_t)a.a.p | (uintptr_t)a.b.p | (uintptr_t)a.a.stride | (uintptr_t)a.b.stride) % 4 == 0;
}

template <typename O>
int launch_few(ProductArgs& a, hipStream_t stream) {
  const int rc = tiles_of(a, 16, 16);
  if (rc != GG_OK) return rc;
  int waves = 1;
  while (waves < kFewWaves && waves < a.kb) waves *= 2;
  const dim3 grid((unsigned)a.tiles_i * a.tiles_j), block(waves * kWave);
  if (in_words(a))
    hipLaunchKernelGGL((k_product_few<O, false>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((k_product_few<O, true>), grid, block, 0, stream, a);
  GG_LAUNCH_CHECK("k_product_few");
  return GG_OK;
}

template <typename O, int BJ, int BI, int WJ, int WI, int WK, int STAGES>
int launch_pipe(ProductArgs& a, hipStream_t stream) {
  const int rc = tiles_of(a, BJ, BI);
  if (rc != GG_OK) return rc;
  const dim3 grid((unsigned)a.tiles_i * a.tiles_j), block(WJ * WI * WK * kWave);
  if (in_words(a))
    hipLaunchKernelGGL((k_product_pipe<O, BJ, BI, WJ, WI, WK, STAGES, false>), grid, block, 0, stream, a);
  else
    hipLaunchKernelGGL((k_product_pipe<O, BJ, BI, WJ, WI, WK, STAGES, true>), grid, block, 0, stream, a);
  GG_LAUNCH_CHECK("k_product_pipe");
  return GG_OK;
}

template <typename O>
int launch_wide(ProductArgs& a, hipStream_t stream) {
  const int rc = tiles_of(a, 256, 256);
  if (rc != GG_OK) return rc;
  hipLaunchKernelGGL((k_product_wide<O>), dim3((unsigned)a.tiles_i * a.tiles_j), dim3(512), 0, stream, a);
  GG_LAUNCH_CHECK("k_product_wide");
  return GG_OK;
}

template <typename O, int BJ, int BI, int WJ, int WI>
int launch_tile(ProductArgs& a, hipStream_t stream) {
  const int rc = tiles_of(a, BJ, BI);
  if (rc != GG_OK) return rc;
  hipLaunchKernelGGL((k_product_tile<O, BJ, BI, WJ, WI>), dim3((unsigned)a.tiles_i * a.tiles_j),
                     dim3(WJ * WI * kWave), 0, stream, a);
  GG_LAUNCH_CHECK("k_product_tile");
  return GG_OK;
}

// Which kernel: microseconds measured beside the next best, bf16 results.  (fp32 results, whose
// products take twice as long, go by the same rule, without the largest tiles.)
template <typename O>
int launch_product(ProductArgs& a, hipStream_t stream) {
  // offsets in a tile are of 32 bits
  const bool near = std::max({a.a.stride, a.b.stride, a.a.sstride}) <= 1 << 23;
  const bool words = in_words(a);
  const auto tiles = [&](int bj, int bi) { return cdiv(a.n, bi) * cdiv(a.m, bj); };
  if (!near) return launch_tile<O, 128, 128, 2, 2>(a, stream);
  // Few rows, or rows and weights that are few together: without LDS, which gathers rows
  // badly (16 rows of 4,096 to 4,096 7.6 us, through LDS 8.7; of 8,192 to 8,192 20.5 and 15.1;
  // 64 rows of 4,096 to 1,024 7.3 and 8.6, to 4,096 20.5 and 9.0).
  if (a.n <= 4 || tiles(16, 16) * a.kb <= 8192) return launch_few<O>(a, stream);
  // The smallest tiles of which there is one for each CU, or that hold all rows (steps of 32 x 32
  // take 0.33 us, of 32 x 64 0.4, of 32 x 96 and beyond 0.6; 1,076 rows of 7,808 to 384 16.8 us in
  // 32 x 64, 22.9 in 32 x 128; 256 rows of 4,096 to 4,096 15.1 in 32 x 128, 26.1 in 128 x 128).
  const auto fits = [&](int bj, int bi) { return a.n <= bi || tiles(bj, bi) <= 256; };
  if (fits(32, 32)) return launch_pipe<O, 32, 32, 1, 2, 2, 5>(a, stream);
  if (fits(32, 64)) return launch_pipe<O, 32, 64, 1, 4, 2, 5>(a, stream);
  if (fits(32, 96)) return launch_pipe<O, 32, 96, 2, 2, 2, 3>(a, stream);
  if (tiles(32, 128) <= 256) return launch_pipe<O, 32, 128, 1, 4, 2, 3>(a, stream);
  if (tiles(64, 128) <= 256) return launch_pipe<O, 64, 128, 2, 2, 2, 3>(a, stream);
  if (tiles(128, 128) <= 256) return launch_pipe<O, 128, 128, 2, 2, 2, 2>(a, stream);
  // A round of 256 of 256 x 256 takes 1.4 to 1.85 times one of 512 of 128 x 128 (8,192 and 2,048
  // columns), and does twice as much.  Of few blocks of k its stores, with no other block on
  // the CU, are waited for (10,239 rows to 53,277, k 512: 621 and 567, 1,024: 858 and 855).
  if constexpr (sizeof(O) == 2)
    if (words && a.kb > 4 && a.n >= 256 && cdiv(tiles(256, 256), 256) * 8 <= cdiv(tiles(128, 128), 512) * 5)
      return launch_wide<O>(a, stream);
  return launch_pipe<O, 128, 128, 2, 2, 1, 2>(a, stream);
}

}  // namespace
}  // namespace gg

using namespace gg;

extern "C" int gg_product_forward(const gg_rows_t* a, int64_t n, int64_t k, const gg_blocks_t* b,
                                  int64_t m, const gg_rows_t* out, hipStream_t stream) {
  GG_REQUIRE(n >= 0 && n <= GG_PRODUCT_MAX_ROWS, "n = %lld unsupported", (long long)n);
  GG_REQUIRE(k >= 1 && k <= GG_PRODUCT_MAX_DIM, "k %lld outside 1..%d", (long long)k,
             GG_PRODUCT_MAX_DIM);
  GG_REQUIRE(m >= 1 && m <= GG_PRODUCT_MAX_DIM, "m %lld outside 1..%d", (long long)m,
             GG_PRODUCT_MAX_DIM);
  ProductArgs p = {};
  int rc = pack_rows(a, "a", n, k, kBitE4M3, false, &p.a);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(p.a.group == 0 || p.a.group == kScaleBlock, "a: group %d is neither 0 nor %d", p.a.group,
             kScaleBlock);
  rc = pack_blocks(b, "b", m, k, false, &p.b);
  if (rc == GG_OK) rc = pack_rows(out, "out", n, m, kBitFloats, true, &p.out);
  if (rc != GG_OK || n == 0) return rc;
  p.n = n;
  p.k = (int32_t)k;
  p.m = (int32_t)m;
  p.kb = (int32_t)cdiv(k, kBlockK);
  p.per_row = p.a.group == 0;
  p.scales16 = !p.per_row && k % (4 * kBlockK) == 0 && aligned16(p.a.scales) && aligned16(p.b.scales) &&
               p.a.sstride % 16 == 0 && p.b.sstride % 16 == 0;
  GG_FOR_FLOAT(out->dtype, O, return launch_product<O>(p, stream));
}
