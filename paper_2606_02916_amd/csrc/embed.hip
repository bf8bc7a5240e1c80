// Embedding lookup with scaling, and its gradient by sorted ids.
#include "rows.hpp"

namespace gg {
namespace {

__device__ __forceinline__ int64_t id_at(const void* ids, int32_t bits, int64_t i) {
  return bits == 64 ? ((const int64_t*)ids)[i] : (int64_t)((const int32_t*)ids)[i];
}

// ---------------------------------------------------------------------------
// Lookup: out[i] = scale * table[ids[i]].
//
// Nothing is used twice, so the call is bound by memory: the rows read and the
// rows written.  The output is one run of n * pieces pieces of 16 bytes (of
// the wider type), dealt to the lanes in order: every store covers a
// contiguous run, rows of any width fill the waves, and one wide row spreads
// over as many waves as it has.  A lane has U pieces in flight.  1.5M rows of
// 100 fp32 take 210 us, 5.0 TB/s if each distinct row counts once, a 1 GiB copy's
// rate; 400,000 rows of 128 codes to fp16 30 us, 5.1; one row 2.2 us, an empty
// launch's time.
// ---------------------------------------------------------------------------
struct LookupArgs {
  KRows table, out;
  const void* ids;
  int32_t id_bits;
  int32_t dim;
  int64_t rows, n;
  float scale;
  uint32_t pieces, pmagic;
  bool stream;        // the output goes past the caches
  int32_t glog;       // log2 of the elements per scale; 31: one scale per row
  int32_t* status;
};

template <typename TI, typename TO, int V, int U>
__global__ void __launch_bounds__(kBlock) k_embed_rows(LookupArgs a) {
  // The block's first row and piece (the same for all lanes).
  // (below the number of pieces, which is 2^32 at most)
  const uint32_t base = blockIdx.x * (uint32_t)(kBlock * U);
  const uint32_t row0 = base / a.pieces, rem = base - row0 * a.pieces;
  // All ids, then all rows: a lane waits twice, whatever U is.
  typename Raw<TI, V>::vec raw[U];
  float mul[U], mul2[U];
  int64_t row[U], id[U];
  int32_t e[U];
  bool ok[U];
  bool bad = false;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const uint32_t o = rem + (uint32_t)(j * kBlock + threadIdx.x);
    const uint32_t r = chunk_row(o, a.pmagic);
    int32_t skip;
    e[j] = piece_start<V>((int32_t)(o - r * a.pieces), a.dim, &skip);
    row[j] = (int64_t)row0 + r;
    ok[j] = row[j] < a.n;
    id[j] = min(row[j], a.n - 1);
  }
  if (a.ids) {
#pragma unroll
    for (int j = 0; j < U; ++j) id[j] = id_at(a.ids, a.id_bits, id[j]);
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    raw[j] = {};
    mul[j] = mul2[j] = 0.0f;
    if (ok[j]) {
      if ((uint64_t)id[j] < (uint64_t)a.rows) {
        raw[j] = raw_load<TI, V>(a.table.p + id[j] * a.table.stride + e[j] * (int64_t)sizeof(TI));
        mul[j] = mul2[j] = 1.0f;
        if constexpr (sizeof(TI) == 1) {
          // The row's last piece may lie in two groups (never in more).
          const float* sc = (const float*)(a.table.scales + id[j] * a.table.sstride);
          mul[j] = sc[e[j] >> a.glog];
          mul2[j] = sc[(e[j] + V - 1) >> a.glog];
        }
      } else {
        bad |= id[j] != -1;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    if (!ok[j]) continue;
    if ((uint64_t)id[j] < (uint64_t)a.rows) {
      mul[j] *= a.scale;
      mul2[j] *= a.scale;
    }
    float v[V];
    to_f32<TI, V>(raw[j], v);
#pragma unroll
    for (int k = 0; k < V; ++k)
      v[k] *= sizeof(TI) == 1 && ((e[j] ^ (e[j] + k)) >> a.glog) ? mul2[j] : mul[j];
    row_store<TO, V>(a.out.p + (int64_t)row[j] * a.out.stride + e[j] * (int64_t)sizeof(TO), v,
                     a.stream);
  }
  if (bad) set_status(a.status, GG_DEV_BAD_ID);
}

// ---------------------------------------------------------------------------
// Sorting the ids: pairs (key, position) by key, positions ascending within a
// key.  A key is its id, or num_rows for an id that adds nothing; the radix
// passes take the low digit first and keep the order of equal digits, so the
// result depends on the ids alone.
//
// A tile of pairs belongs to a block; wave w of it holds the pairs
// [w * kTileWave, (w + 1) * kTileWave) of the tile, 64 neighbouring ones at a
// time.  Lanes whose digits agree find each other by one ballot per digit bit,
// so equal digits are counted and ranked without atomics.
//
// Each launch waits more than it works: 200,003 ids take four of 5, 13, 5 and 13
// us, of which reading and writing the pairs at a copy's rate would be half a
// microsecond each.  What they cost is the way through one tile: its load, the
// counters of all tiles, the scan, LDS and the store.  Every tile reads every
// tile's counters, 1 KB each: up to 2^24 ids those stay in an XCD's cache (1M ids
// of 8 fp16 92 us for the whole call, 4.2M 236, 16.8M 1.1 ms), beyond they are the
// call (33.6M 9.6 ms, 67M 19).
// ---------------------------------------------------------------------------
// Up to this many pairs find their places by counting, in a single launch.
constexpr int kRankBlock = 1024;
constexpr int kRankMost = 16384;
// Beyond, tiles of 2,048 pairs spread the instructions over the chip, two pairs a
// lane, so that a SIMD has several waves to take them from (eight pairs a lane in
// blocks of 4 waves: 60,000 ids of 64 fp32 60 us instead of 50, 524,000 of 16 66
// instead of 62; four in 8 waves 52 and 66).  Every tile reads the counters of all,
// so many ids have tiles of 8,192, with digits of 8 bits instead of 9.
constexpr int kSmallThreads = 1024, kSmallKeys = 2;     // pairs per lane
constexpr int kLargeThreads = 1024, kLargeKeys = 8;
constexpr int kSmallTile = kSmallThreads * kSmallKeys, kLargeTile = kLargeThreads * kLargeKeys;
constexpr int kSmallSortTiles = 256;                    // most small tiles
constexpr int digit_limit(int tile) { return tile == kSmallTile ? 9 : 8; }

// Rows to be cleared by the sort's launches, in blocks behind its own: the sort
// waits for memory more than it uses it.  Rows that lie back to back are one
// run of 16-byte pieces, which a block clears 8 pieces a lane in one place: past
// the caches, so that what the sort and the sums read stays there (32,768 ids
// and 128,000 x 2,048 bf16 rows 140 us, through the caches 164; one piece a lane
// in one place 151).
constexpr int kFillRun = 8;

struct FillArgs {
  char* p;
  int64_t stride;
  int64_t r0, r1;          // rows of this launch
  int32_t row_bytes, pieces, lanes_log;
};

template <int NT>
__device__ void fill_rows_with_zeros(const FillArgs& f, uint32_t block, uint32_t blocks) {
  typedef Raw<f16, 8>::vec vec;
  typedef Raw<f16, 8>::mem mem;
  if (f.stride == f.row_bytes) {
    char* p = f.p + f.r0 * f.stride;
    const int64_t bytes = (f.r1 - f.r0) * f.stride, n = bytes / 16;
    constexpr int kRun = NT * kFillRun;      // pieces that a block clears in one place
    for (int64_t i0 = (int64_t)block * kRun; i0 < n; i0 += (int64_t)blocks * kRun)
#pragma unroll
      for (int u = 0; u < kFillRun; ++u) {
        const int64_t i = i0 + u * NT + threadIdx.x;
        if (i < n) __builtin_nontemporal_store(vec{}, (GG_GLOBAL mem*)(p + i * 16));
      }
    if (block == 0 && threadIdx.x < (bytes - n * 16) / 2)
      *(GG_GLOBAL uint16_t*)(p + n * 16 + threadIdx.x * 2) = 0;
    return;
  }
  const int groups = NT >> f.lanes_log, lanes = 1 << f.lanes_log;
  const int g = threadIdx.x >> f.lanes_log, l = threadIdx.x & (lanes - 1);
  for (int64_t r = f.r0 + (int64_t)block * groups + g; r < f.r1; r += (int64_t)blocks * groups) {
    char* p = f.p + r * f.stride;
    for (int32_t c = l; c < f.pieces; c += lanes) {
      if (f.row_bytes >= 16)
        *(GG_GLOBAL mem*)(p + min(c * 16, f.row_bytes - 16)) = vec{};
      else
        *(GG_GLOBAL uint16_t*)(p + 2 * c) = 0;
    }
  }
}

struct Keys {
  const void* ids;       // first pass: the ids; later passes: key and pos
  int32_t id_bits;
  const uint32_t* key;
  const uint32_t* pos;
  int64_t n;
  uint32_t rows;         // num_rows
  int32_t shift, bits;   // the pass's digit
  int32_t* status;
};

// A lane's keys of the pairs first + lane, first + 64 + lane, .. below `left`,
// all loads in flight together (places past the end repeat the last pair).
template <int K>
__device__ __forceinline__ void load_keys(const Keys& a, int64_t first, int left,
                                          uint32_t (&key)[K]) {
  int64_t at[K];
#pragma unroll
  for (int j = 0; j < K; ++j) at[j] = min(first + j * kWave + lane_id(), a.n - 1);
  if (!a.ids) {
#pragma unroll
    for (int j = 0; j < K; ++j) key[j] = a.key[at[j]];
    return;
  }
  int64_t id[K];
  if (a.id_bits == 64) {
#pragma unroll
    for (int j = 0; j < K; ++j) id[j] = ((const int64_t*)a.ids)[at[j]];
  } else {
#pragma unroll
    for (int j = 0; j < K; ++j) id[j] = ((const int32_t*)a.ids)[at[j]];
  }
  bool bad = false;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const bool in = (uint64_t)id[j] < (uint64_t)a.rows;
    key[j] = in ? (uint32_t)id[j] : a.rows;
    bad |= !in && id[j] != -1 && j * kWave + lane_id() < left;
  }
  if (bad) set_status(a.status, GG_DEV_BAD_ID);
}

// Lanes with this lane's digit, among the valid ones: four instructions a bit.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, int bits, bool valid) {
  uint64_t m = __ballot(valid);
  uint32_t lo = (uint32_t)m, hi = (uint32_t)(m >> 32);
  for (int b = 0; b < bits; ++b) {
    const uint32_t t = (uint32_t)__builtin_amdgcn_sbfe((int)d, (uint32_t)b, 1u);   // 0 or ~0
    const uint64_t one = __ballot(t != 0);
    lo &= ~((uint32_t)one ^ t);
    hi &= ~((uint32_t)(one >> 32) ^ t);
  }
  return (uint64_t)hi << 32 | lo;
}

// Ranks a wave's pairs: cnt[d] ends as their number with digit d, rank[j] as the
// number of earlier ones.
// (The counters go by LDS addresses: through generic ones, volatile accesses
// become flat ones, with a wait for global memory at each.)
template <int K>
__device__ __forceinline__ void rank_tile(const uint32_t (&key)[K], int shift, int bits, int left,
                                          uint16_t* cnt, uint16_t (&rank)[K]) {
  const uint32_t mask = (1u << bits) - 1u;
  const int lane = lane_id();
  auto* c = (__attribute__((address_space(3))) volatile uint16_t*)cnt;
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const uint32_t d = (key[j] >> shift) & mask;
    const bool valid = j * kWave + lane < left;
    const uint64_t m = same_digit(d, bits, valid);
    // A wave's LDS accesses run in order: all its lanes read before one writes.
    const uint32_t before = c[d];
    const int below = lanes_below(m);
    rank[j] = (uint16_t)(before + below);
    if (valid && below == 0) c[d] = (uint16_t)(before + __popcll(m));
  }
}

// Digit counts of each tile: hist[tile][digit].
template <int NT, int K>
__global__ void __launch_bounds__(NT) k_sort_count(Keys a, int32_t* hist, int tiles,
                                                   FillArgs f) {
  if ((int)blockIdx.x >= tiles)
    return fill_rows_with_zeros<NT>(f, blockIdx.x - tiles, gridDim.x - tiles);
  constexpr int kSortWaves = NT / kWave, kTile = NT * K, kTileWave = kWave * K;
  __shared__ uint16_t cnt[kSortWaves << digit_limit(kTile)];
  const int digits = 1 << a.bits, w = threadIdx.x / kWave;
  for (int i = threadIdx.x; i < kSortWaves * digits; i += NT) cnt[i] = 0;
  const int64_t first = (int64_t)blockIdx.x * kTile + w * kTileWave;
  const int left = (int)min((int64_t)kTileWave, max((int64_t)0, a.n - first));
  uint32_t key[K];
  uint16_t rank[K];
  load_keys(a, first, left, key);
  __syncthreads();
  rank_tile(key, a.shift, a.bits, left, cnt + w * digits, rank);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += NT) {
    int32_t s = 0;
#pragma unroll
    for (int v = 0; v < kSortWaves; ++v) s += cnt[v * digits + d];
    hist[(int64_t)blockIdx.x * digits + d] = s;
  }
}

// Moves a tile's pairs to their places: those of smaller digits come first,
// then those of earlier tiles with the same digit, as the counts of all tiles
// (hist) tell.
template <int NT, int K>
__global__ void __launch_bounds__(NT) k_sort_scatter(Keys a, const int32_t* hist, int tiles,
                                                     uint32_t* key_out, uint32_t* pos_out,
                                                     FillArgs f) {
  if ((int)blockIdx.x >= tiles)
    return fill_rows_with_zeros<NT>(f, blockIdx.x - tiles, gridDim.x - tiles);
  constexpr int kSortWaves = NT / kWave, kTile = NT * K, kTileWave = kWave * K;
  __shared__ uint16_t cnt[kSortWaves << digit_limit(kTile)];
  __shared__ int32_t base[1 << digit_limit(kTile)];
  __shared__ uint16_t local[1 << digit_limit(kTile)];     // first place of a digit in the tile
  __shared__ uint32_t s_key[kTile], s_pos[kTile];
  __shared__ int2 s_mine[NT], s_all[NT];
  __shared__ uint64_t s_scan[kSortWaves];
  const int tid = threadIdx.x, digits = 1 << a.bits, w = tid / kWave;
  for (int i = tid; i < kSortWaves * digits; i += NT) cnt[i] = 0;
  const int64_t first = (int64_t)blockIdx.x * kTile + w * kTileWave;
  const int left = (int)min((int64_t)kTileWave, max((int64_t)0, a.n - first));
  uint32_t key[K], pos[K];
  uint16_t rank[K];
#pragma unroll
  for (int j = 0; j < K; ++j) pos[j] = (uint32_t)(first + j * kWave + lane_id());
  if (!a.ids) {
#pragma unroll
    for (int j = 0; j < K; ++j) pos[j] = a.pos[min((int64_t)pos[j], a.n - 1)];
  }
  load_keys(a, first, left, key);
  // A lane adds up two neighbouring digits over a share of the tiles.
  const int cols = digits / 2, groups = NT / cols, c = tid & (cols - 1), g = tid / cols;
  const int per = (tiles + groups - 1) / groups, t1 = min(tiles, (g + 1) * per);
  int2 mine = {0, 0}, all = {0, 0};
#pragma unroll 16
  for (int t = g * per; t < t1; ++t) {
    const int2 v = ((const int2*)hist)[(int64_t)t * cols + c];
    const bool before = t < (int)blockIdx.x;
    all.x += v.x;
    all.y += v.y;
    mine.x += before ? v.x : 0;
    mine.y += before ? v.y : 0;
  }
  s_mine[tid] = mine;
  s_all[tid] = all;
  __syncthreads();
  rank_tile(key, a.shift, a.bits, left, cnt + w * digits, rank);
  __syncthreads();
  // The digits' totals over all tiles and in this one, scanned together.
  mine = all = {0, 0};
  int32_t in[2] = {0, 0};
  if (tid < cols) {
    for (int x = 0; x < groups; ++x) {
      mine.x += s_mine[x * cols + tid].x;
      mine.y += s_mine[x * cols + tid].y;
      all.x += s_all[x * cols + tid].x;
      all.y += s_all[x * cols + tid].y;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int v = 0; v < kSortWaves; ++v) {
        const uint16_t n = cnt[v * digits + 2 * tid + h];
        cnt[v * digits + 2 * tid + h] = (uint16_t)in[h];     // of earlier waves
        in[h] += n;
      }
  }
  uint64_t total;
  const uint64_t before = block_excl_scan<NT>(
      (uint64_t)(uint32_t)(all.x + all.y) << 32 | (uint32_t)(in[0] + in[1]), s_scan, &total);
  if (tid < cols) {
    const int32_t b = (int32_t)(before >> 32), l = (int32_t)(before & 0xffffffffu);
    base[2 * tid] = b + mine.x;
    base[2 * tid + 1] = b + all.x + mine.y;
    local[2 * tid] = (uint16_t)l;
    local[2 * tid + 1] = (uint16_t)(l + in[0]);
  }
  __syncthreads();
  // The tile in order in LDS, so that a digit's pairs leave in one run.
#pragma unroll
  for (int j = 0; j < K; ++j) {
    if (j * kWave + lane_id() >= left) continue;
    const uint32_t d = (key[j] >> a.shift) & (digits - 1);
    const uint32_t to = (uint32_t)local[d] + cnt[w * digits + d] + rank[j];
    s_key[to] = key[j];
    s_pos[to] = pos[j];
  }
  __syncthreads();
  const int size = (int)min((int64_t)kTile, a.n - (int64_t)blockIdx.x * kTile);
#pragma unroll
  for (int j = 0; j < K; ++j) {
    const int i = j * NT + tid;
    if (i >= size) continue;
    const uint32_t k = s_key[i], d = (k >> a.shift) & (digits - 1);
    const uint32_t to = (uint32_t)base[d] + (uint32_t)(i - (int)local[d]);
    key_out[to] = k;
    pos_out[to] = s_pos[i];
  }
}

// Few pairs: a pair's place is the number of smaller keys, and of equal ones
// before it.  A block has 64 pairs, one per lane, and its waves compare them
// with a share of all keys each, which they read from LDS four at a time.  That
// is n^2 comparisons, but on the whole chip and in one launch.  Comparisons bound
// it: rows of 64 fp32 added into 233,000, the whole call with this sort and with
// four launches of the other kernels: 4,000 ids 16 and 26 us, 8,000 22 and 28,
// 12,000 27 and 30, 14,298 29 both, 16,384 32 and 30.
__global__ void __launch_bounds__(kRankBlock) k_sort_rank(Keys a, int blocks, uint32_t* key_out,
                                                          uint32_t* pos_out, FillArgs f) {
  if ((int)blockIdx.x >= blocks)
    return fill_rows_with_zeros<kRankBlock>(f, blockIdx.x - blocks, gridDim.x - blocks);
  constexpr int kWaves = kRankBlock / kWave;
  __shared__ uint4 s_key[kWaves][kWave / 4];
  __shared__ uint32_t s_count[kWaves][kWave];
  const int n = (int)a.n, w = threadIdx.x / kWave, lane = lane_id();
  const int i0 = (int)blockIdx.x * kWave;
  uint32_t own[1];
  // (the ids out of range are reported once)
  load_keys(a, i0, w == 0 ? n - i0 : 0, own);
  const uint32_t k = own[0];
  const int chunks = (n + kWave - 1) / kWave, per = (chunks + kWaves - 1) / kWaves;
  const int c1 = min(chunks, (w + 1) * per);
  uint32_t count = 0;
  uint32_t next[1];
  if (w * per < c1) load_keys(a, (int64_t)w * per * kWave, 0, next);
  for (int c = w * per; c < c1; ++c) {
    // a place past the end counts for nobody
    const uint32_t mine = c * kWave + lane < n ? next[0] : ~0u;
    if (c + 1 < c1) load_keys(a, (int64_t)(c + 1) * kWave, 0, next);
    ((uint32_t*)s_key[w])[lane] = mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (c < (int)blockIdx.x) {
#pragma unroll
      for (int j = 0; j < kWave / 4; ++j) {
        const uint4 v = s_key[w][j];
        count += (v.x <= k) + (v.y <= k) + (v.z <= k) + (v.w <= k);
      }
    } else if (c > (int)blockIdx.x) {
#pragma unroll
      for (int j = 0; j < kWave / 4; ++j) {
        const uint4 v = s_key[w][j];
        count += (v.x < k) + (v.y < k) + (v.z < k) + (v.w < k);
      }
    } else {
      for (int j = 0; j < kWave; ++j) {
        const uint32_t v = ((const uint32_t*)s_key[w])[j];
        count += v < k || (v == k && j < lane);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  s_count[w][lane] = count;
  __syncthreads();
  if (w == 0 && i0 + lane < n) {
#pragma unroll
    for (int x = 1; x < kWaves; ++x) count += s_count[x][lane];
    key_out[count] = k;
    pos_out[count] = (uint32_t)(i0 + lane);
  }
}

// ---------------------------------------------------------------------------
// Sums of the sorted rows.
//
// A run is the positions of one id.  k_grad_rows gives a block `per` rows of
// the gradient (or, when rows are added to, the runs that start in `per` sorted
// positions), so that every row is written once, zeros included, and the
// gradient needs no pass that clears it.  Short runs are summed by a group of
// `lanes` lanes each, longer ones by the block's groups together.  Runs of
// more than `chunk` positions are cut at multiples of it: the launch's first
// blocks sum their parts, a block per chunk, so that an id that fills the whole
// call still spreads over the chip, and k_grad_long joins them.
//
// Bound by memory: dy's rows are read once in the order of the ids, the
// gradient's written once.  200,003 x 602 fp32 rows into 233,000 take 222 us, 4.7
// TB/s; 32,768 x 2,048 bf16 rows, ids by a power law, 49.
// ---------------------------------------------------------------------------
constexpr int kGradRows = 256;       // most entries of a block
constexpr int kGroupRun = 32;        // longest run that one group sums (4, 8 and 16: 2,468
                                     // ids of 1,253 rows 43, 33 and 34 us, 32 takes 28)
constexpr int kPosCache = 1024;
constexpr int kLongUnroll = 8;       // rows in flight in a longer run
template <int V>
constexpr int kItems = 16 / V < 4 ? 16 / V : 4;     // short runs summed together
template <int V>
constexpr uint32_t kTerms = 8 / kItems<V>;           // rows of each in flight

struct GradArgs {
  const uint32_t* key;     // sorted
  const uint32_t* pos;
  uint32_t n, rows;
  int32_t dim;
  int32_t pieces;          // column pieces of a row
  int32_t lanes_log;       // lanes of a group (a power of two up to 64)
  int32_t tiles;           // column tiles of a group
  int32_t shift;           // column tiles start at piece -shift
  uint32_t tmagic;         // div_magic(tiles)
  uint32_t per;            // rows (or positions) of a block
  uint32_t chunk;
  int32_t add;
  int32_t by_position;     // blocks have positions, not rows: rows are added to, or were cleared
  uint32_t part_blocks;
  float scale;
  KRows dy, grad;
  float* part;             // [chunk][2][dim]: a run from before the chunk, one into the next
};

// First i in [lo, hi) with k[i] >= v, or hi.  All lanes of a wave together: 64
// probes a step.
__device__ uint32_t wave_lower_bound(const uint32_t* k, uint32_t lo, uint32_t hi, uint32_t v) {
  const uint32_t lane = lane_id();
  while (hi - lo > kWave) {
    const uint32_t step = (hi - lo + kWave - 1) / kWave;
    const uint64_t i = (uint64_t)lo + (uint64_t)(lane + 1) * step - 1;
    const uint32_t c = (uint32_t)__popcll(__ballot(i < hi && k[i] < v));
    lo += c * step;
    hi = min(hi, lo + step);
  }
  return lo + (uint32_t)__popcll(__ballot(lo + lane < hi && k[lo + lane] < v));
}

// The piece of lane l of a group in a column tile; `in`: it has one (lanes
// without one get another's).  A row's last piece and the one before it, which it
// overlaps, are always of one tile (shift, below): a wave reads both before it
// writes either, so that what is added to is added to once.
__device__ __forceinline__ int32_t piece_of(const GradArgs& a, int32_t tile, int32_t l, bool* in) {
  const int32_t p = (tile << a.lanes_log) + l - a.shift;
  *in = (uint32_t)p < (uint32_t)a.pieces;
  return min(max(p, 0), a.pieces - 1);
}

// Adds the rows dy[pos[p]], p = p0, p0 + step, .. < p1, to acc.
template <typename TD, int V>
__device__ __forceinline__ void add_rows(const GradArgs& a, uint32_t p0, uint32_t p1, uint32_t step,
                                         int32_t e, float (&acc)[V]) {
  const char* base = a.dy.p + e * (int64_t)sizeof(TD);
  for (uint64_t p = p0; p < p1; p += (uint64_t)step * kLongUnroll) {
    // Several rows in flight; places past the end repeat the first row and add 0.
    typename Raw<TD, V>::vec raw[kLongUnroll];
    uint32_t at[kLongUnroll];
#pragma unroll
    for (int u = 0; u < kLongUnroll; ++u) {
      const uint64_t q = p + (uint64_t)u * step;
      at[u] = a.pos[q < p1 ? q : p];
    }
#pragma unroll
    for (int u = 0; u < kLongUnroll; ++u)
      raw[u] = raw_load<TD, V>(base + (int64_t)at[u] * a.dy.stride);
#pragma unroll
    for (int u = 0; u < kLongUnroll; ++u) {
      const bool in = p + (uint64_t)u * step < p1;
      float v[V];
      to_f32<TD, V>(raw[u], v);
#pragma unroll
      for (int k = 0; k < V; ++k) acc[k] += in ? v[k] : 0.0f;
    }
  }
}

// As add_rows, over the parts of run [beg, end) that sum_parts left.
template <int V>
__device__ __forceinline__ void add_parts(const GradArgs& a, uint32_t beg, uint32_t end,
                                          uint32_t first, uint32_t step, int32_t e,
                                          float (&acc)[V]) {
  const uint32_t c0 = beg / a.chunk, c1 = (end - 1) / a.chunk;
#pragma unroll 4
  for (uint32_t c = c0 + first; c <= c1; c += step) {
    // the chunk where the run starts holds a part that leads into the next one
    const float* p = a.part + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * a.dim + e;
    float v[V];
    row_load<float, V>((const char*)p, v);
#pragma unroll
    for (int k = 0; k < V; ++k) acc[k] += v[k];
  }
}

// Sums the groups' accumulators into group 0's, in the order of the groups.
template <int V>
__device__ __forceinline__ void join_groups(float (&acc)[V], float* lds, int lanes, int groups) {
  const int tid = threadIdx.x;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < V; ++k) lds[k * kBlock + tid] = acc[k];
  __syncthreads();
  if (tid < lanes)
    for (int g = 1; g < groups; ++g)
#pragma unroll
      for (int k = 0; k < V; ++k) acc[k] += lds[k * kBlock + g * lanes + tid];
}

// One column tile of a chunk's parts of long runs.
template <typename TD, int V>
__device__ __forceinline__ void sum_parts(const GradArgs& a, uint32_t c, int32_t tile, float* lds,
                                          uint32_t (*s_run)[2]) {
  const uint32_t c0 = c * a.chunk;
  const uint32_t c1 = (uint32_t)min((uint64_t)a.n, (uint64_t)c0 + a.chunk);
  const uint32_t kb = a.key[c0], ke = a.key[c1 - 1];
  const bool from = c0 > 0 && a.key[c0 - 1] == kb && kb < a.rows;
  const bool into = c1 < a.n && a.key[c1] == ke && ke < a.rows && !(from && ke == kb);
  if (!from && !into) return;
  const int w = threadIdx.x / kWave;
  // Each run's positions in this chunk, none if the run is not a long one: a run
  // that ends at h began more than a chunk earlier if the position a chunk
  // before its last holds it too.
  if (w == 0) {
    const uint32_t h = from ? wave_lower_bound(a.key, c0, c1, kb + 1) : c0;
    const bool is_long = from && ((h == c1 && c1 < a.n && a.key[c1] == kb) ||
                                  (h > a.chunk && a.key[h - 1 - a.chunk] == kb));
    if (lane_id() == 0) {
      s_run[0][0] = c0;
      s_run[0][1] = is_long ? h : c0;
    }
  } else if (w == 1) {
    const uint32_t b = into ? wave_lower_bound(a.key, c0, c1, ke) : c1;
    const bool is_long = into && (uint64_t)b + a.chunk < a.n && a.key[b + a.chunk] == ke;
    if (lane_id() == 0) {
      s_run[1][0] = is_long ? b : c1;
      s_run[1][1] = c1;
    }
  }
  __syncthreads();
  const int lanes = 1 << a.lanes_log, groups = kBlock >> a.lanes_log;
  const int g = threadIdx.x >> a.lanes_log, l = threadIdx.x & (lanes - 1);
  int32_t skip;
  bool in;
  const int32_t e = piece_start<V>(piece_of(a, tile, l, &in), a.dim, &skip);
  for (int s = 0; s < 2; ++s) {
    const uint32_t p0 = s_run[s][0], p1 = s_run[s][1];
    if (p0 >= p1) continue;
    float acc[V] = {};
    add_rows<TD, V>(a, p0 + g, p1, groups, e, acc);
    join_groups<V>(acc, lds, lanes, groups);
    if (g == 0 && in)
      row_store<float, V>((char*)(a.part + ((int64_t)c * 2 + s) * a.dim + e), acc);
  }
}

template <typename TG, int V>
__device__ __forceinline__ void put_row(const GradArgs& a, uint32_t row, int32_t e,
                                        float (&acc)[V]) {
  char* p = a.grad.p + (int64_t)row * a.grad.stride + e * (int64_t)sizeof(TG);
#pragma unroll
  for (int k = 0; k < V; ++k) acc[k] *= a.scale;
  if (a.add) {
    float old[V];
    row_load<TG, V>(p, old);
#pragma unroll
    for (int k = 0; k < V; ++k) acc[k] += old[k];
  }
  row_store<TG, V>(p, acc);
}

// The runs of up to kGroupRun positions.  Items are (entry, column tile); a
// group sums kItems of them at a time, kTerms rows of each in flight, so that
// runs of one or two rows, as most are, cost one wait.  What is left of longer ones
// is summed an item at a time, kLongUnroll rows in flight, where kItems are four
// (200,003 fp32 rows of 256 into 100,000, ids by a power law, 111 us instead of
// 124); with two, of four rows each, all go on together (32,768 bf16 rows of
// 1,024 into 64,000 61 us, 64 the other way).  CACHED: the positions are in LDS.
template <typename TD, typename TG, int V, bool CACHED, bool ADD>
__device__ __forceinline__ void sum_short_runs(const GradArgs& a, uint32_t entries,
                                               const uint32_t* s_row, const uint32_t* s_beg,
                                               const uint32_t* s_end, const uint32_t* s_pos,
                                               uint32_t p0, uint32_t* many) {
  const int groups = kBlock >> a.lanes_log;
  const int g = threadIdx.x >> a.lanes_log, l = threadIdx.x & ((1 << a.lanes_log) - 1);
  const uint32_t items = entries * (uint32_t)a.tiles;
  for (uint32_t i0 = 0; i0 < items; i0 += groups * kItems<V>) {
    uint32_t x[kItems<V>], cnt[kItems<V>], most = 0;
    int32_t e[kItems<V>];
    typename Raw<TG, V>::vec old[kItems<V>];
    float acc[kItems<V>][V];
#pragma unroll
    for (int u = 0; u < kItems<V>; ++u) {
      const uint32_t item = i0 + u * groups + g;
      x[u] = item < items ? chunk_row(item, a.tmagic) : 0u;
      int32_t skip;
      const int32_t piece = ((int32_t)(item - x[u] * a.tiles) << a.lanes_log) + l - a.shift;
      const bool mine = item < items && (uint32_t)piece < (uint32_t)a.pieces;
      e[u] = mine ? piece_start<V>(piece, a.dim, &skip) : -1;
      cnt[u] = s_end[x[u]] - s_beg[x[u]];
      if (cnt[u] > kGroupRun) {
        *many = 1;
        e[u] = -1;
      }
      if (e[u] < 0) cnt[u] = 0;
      most = max(most, cnt[u]);
      if (ADD && e[u] >= 0)
        old[u] = raw_load<TG, V>(a.grad.p + (int64_t)s_row[x[u]] * a.grad.stride +
                                 e[u] * (int64_t)sizeof(TG));
#pragma unroll
      for (int k = 0; k < V; ++k) acc[u][k] = 0.0f;
    }
    constexpr bool kOneByOne = kItems<V> == 4;
    const uint32_t together = kOneByOne ? min(most, kTerms<V>) : most;
    for (uint32_t r = 0; r < together; r += kTerms<V>) {
      typename Raw<TD, V>::vec raw[kItems<V>][kTerms<V>];
#pragma unroll
      for (int u = 0; u < kItems<V>; ++u)
#pragma unroll
        for (uint32_t t = 0; t < kTerms<V>; ++t) {
          raw[u][t] = {};
          if (r + t < cnt[u]) {
            const uint32_t p = s_beg[x[u]] + r + t;
            const uint32_t at = CACHED ? s_pos[p - p0] : a.pos[p];
            raw[u][t] = raw_load<TD, V>(a.dy.p + (int64_t)at * a.dy.stride +
                                        e[u] * (int64_t)sizeof(TD));
          }
        }
#pragma unroll
      for (int u = 0; u < kItems<V>; ++u)
#pragma unroll
        for (uint32_t t = 0; t < kTerms<V>; ++t) {
          float v[V];
          to_f32<TD, V>(raw[u][t], v);
#pragma unroll
          for (int k = 0; k < V; ++k) acc[u][k] += v[k];
        }
    }
    if (kOneByOne && most > kTerms<V>) {
#pragma unroll
      for (int u = 0; u < kItems<V>; ++u)
        for (uint32_t r = kTerms<V>; r < cnt[u]; r += kLongUnroll) {
          typename Raw<TD, V>::vec raw[kLongUnroll];
#pragma unroll
          for (uint32_t t = 0; t < kLongUnroll; ++t) {
            raw[t] = {};
            if (r + t < cnt[u]) {
              const uint32_t p = s_beg[x[u]] + r + t;
              const uint32_t at = CACHED ? s_pos[p - p0] : a.pos[p];
              raw[t] = raw_load<TD, V>(a.dy.p + (int64_t)at * a.dy.stride +
                                       e[u] * (int64_t)sizeof(TD));
            }
          }
#pragma unroll
          for (uint32_t t = 0; t < kLongUnroll; ++t) {
            float v[V];
            to_f32<TD, V>(raw[t], v);
#pragma unroll
            for (int k = 0; k < V; ++k) acc[u][k] += v[k];
          }
        }
    }
#pragma unroll
    for (int u = 0; u < kItems<V>; ++u) {
      if (e[u] < 0) continue;
#pragma unroll
      for (int k = 0; k < V; ++k) acc[u][k] *= a.scale;
      if constexpr (ADD) {
        float was[V];
        to_f32<TG, V>(old[u], was);
#pragma unroll
        for (int k = 0; k < V; ++k) acc[u][k] += was[k];
      }
      row_store<TG, V>(a.grad.p + (int64_t)s_row[x[u]] * a.grad.stride +
                           e[u] * (int64_t)sizeof(TG), acc[u]);
    }
  }
}

// The first blocks sum the chunks' parts of long runs, a column tile each; the
// others have rows of the gradient.
// ADD: rows are added to.  (A kernel of its own: what the rows hold takes
// registers, and 96 leave five waves a SIMD; in one kernel for both, 104, 1.5M
// rows of 100 fp32 into 2.45M took 462 us and now take 420.)
template <typename TD, typename TG, int V, bool ADD>
__global__ void __launch_bounds__(kBlock) __attribute__((amdgpu_waves_per_eu(5)))
k_grad_rows(GradArgs a) {
  __shared__ float lds[V * kBlock];
  __shared__ uint32_t s_run[2][2];
  if (blockIdx.x < a.part_blocks) {
    const uint32_t c = blockIdx.x / (uint32_t)a.tiles;
    sum_parts<TD, V>(a, c, (int32_t)(blockIdx.x - c * a.tiles), lds, s_run);
    return;
  }
  const uint32_t block = blockIdx.x - a.part_blocks;
  __shared__ uint32_t s_row[kGradRows], s_beg[kGradRows], s_end[kGradRows];
  __shared__ uint32_t s_pos[kPosCache];      // pos of the block's positions [p0, p0 + cached)
  __shared__ uint32_t s_range[2], s_many;
  __shared__ int32_t s_heads[kBlock / kWave];
  const uint32_t tid = threadIdx.x, w = tid / kWave;
  uint32_t entries, p0, cached;
  if (tid == 0) s_many = 0;
  if (!a.by_position) {
    // Rows [v0, v0 + entries) and their runs.
    const uint32_t v0 = block * a.per;
    entries = min(a.per, a.rows - v0);
    if (w < 2) {
      const uint32_t r = wave_lower_bound(a.key, 0, a.n, w == 0 ? v0 : v0 + entries);
      if (lane_id() == 0) s_range[w] = r;
    }
    if (tid < entries) {
      s_row[tid] = v0 + tid;
      s_beg[tid] = s_end[tid] = 0u;
    }
    __syncthreads();
    const uint32_t p1 = s_range[1];
    p0 = s_range[0];
    cached = p1 - p0 <= kPosCache ? p1 - p0 : 0u;
    if (cached) {
      for (uint32_t p = p0 + tid; p < p1; p += kBlock) {
        const uint32_t k = a.key[p];
        s_pos[p - p0] = a.pos[p];
        if (p == p0 || a.key[p - 1] != k) s_beg[k - v0] = p;
        if (p + 1 == p1 || a.key[p + 1] != k) s_end[k - v0] = p + 1;
      }
    } else if (p1 > p0 && tid < entries) {
      uint32_t at[2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint32_t lo = p0, hi = p1;
        while (lo < hi) {
          const uint32_t mid = lo + (hi - lo) / 2;
          if (a.key[mid] < v0 + tid + x) lo = mid + 1;
          else hi = mid;
        }
        at[x] = lo;
      }
      s_beg[tid] = at[0];
      s_end[tid] = at[1];
    }
  } else {
    // Runs that start at positions [p0, p0 + per).
    // (a run may end up to kGroupRun positions behind them)
    p0 = block * a.per;
    const uint32_t p = p0 + tid, last = min(a.n, p0 + a.per);
    cached = min(a.n, p0 + a.per + kGroupRun) - p0;
    for (uint32_t i = tid; i < cached; i += kBlock) s_pos[i] = a.pos[p0 + i];
    const uint32_t k = p < last ? a.key[p] : a.rows;
    const bool head = k < a.rows && (p == 0 || a.key[p - 1] != k);
    const uint64_t m = __ballot(head);
    if (lane_id() == 0) s_heads[w] = __popcll(m);
    __syncthreads();
    uint32_t i = lanes_below(m);
    entries = 0;
    for (uint32_t x = 0; x < kBlock / kWave; ++x) {
      i += x < w ? s_heads[x] : 0;
      entries += s_heads[x];
    }
    if (entries == 0) return;
    if (head) {
      s_row[i] = k;
      s_beg[i] = p;
    }
    __syncthreads();
    if (tid + 1 < entries) s_end[tid] = s_beg[tid + 1];
    if (w == 0) {
      // The last run may go on behind the block's positions (ids that add
      // nothing may follow it within them).
      const uint32_t v = s_row[entries - 1];
      uint32_t end = wave_lower_bound(a.key, s_beg[entries - 1], last, v + 1);
      if (end == last && last < a.n && a.key[last] == v)
        end = wave_lower_bound(a.key, last, a.n, v + 1);
      if (lane_id() == 0) s_end[entries - 1] = end;
    }
  }
  __syncthreads();

  const int lanes = 1 << a.lanes_log, groups = kBlock >> a.lanes_log;
  const int g = tid >> a.lanes_log, l = tid & (lanes - 1);
  if (cached || entries == 0)
    sum_short_runs<TD, TG, V, true, ADD>(a, entries, s_row, s_beg, s_end, s_pos, p0, &s_many);
  else
    sum_short_runs<TD, TG, V, false, ADD>(a, entries, s_row, s_beg, s_end, s_pos, p0, &s_many);
  __syncthreads();
  if (!s_many) return;
  int32_t skip;
  for (uint32_t x = 0; x < entries; ++x) {
    const uint32_t beg = s_beg[x], end = s_end[x];
    if (end - beg <= kGroupRun || end - beg > a.chunk) continue;
    for (int32_t t = 0; t < a.tiles; ++t) {
      bool in;
      const int32_t e = piece_start<V>(piece_of(a, t, l, &in), a.dim, &skip);
      float acc[V] = {};
      add_rows<TD, V>(a, beg + g, end, groups, e, acc);
      join_groups<V>(acc, lds, lanes, groups);
      if (g == 0 && in) put_row<TG, V>(a, s_row[x], e, acc);
    }
  }
}

// The long runs that start in chunk blockIdx.x, which is at most one: its
// parts are added up in the order of the chunks.  5 to 7 us: an empty launch, a
// search for the run's ends and, for the longest run, its few hundred parts.
template <typename TG, int V>
__global__ void __launch_bounds__(kBlock) k_grad_long(GradArgs a) {
  __shared__ float lds[V * kBlock];
  const uint32_t c = blockIdx.x, c0 = c * a.chunk, c1 = c0 + a.chunk;   // c1 < n
  const uint32_t k = a.key[c1 - 1];
  if (k >= a.rows || a.key[c1] != k) return;
  const uint32_t beg = wave_lower_bound(a.key, c0, c1, k);
  if (beg == c0 && c0 > 0 && a.key[c0 - 1] == k) return;        // started earlier
  if ((uint64_t)beg + a.chunk >= a.n || a.key[beg + a.chunk] != k) return;
  const uint32_t end = wave_lower_bound(a.key, c1, a.n, k + 1);
  const int lanes = 1 << a.lanes_log, groups = kBlock >> a.lanes_log;
  const int g = threadIdx.x >> a.lanes_log, l = threadIdx.x & (lanes - 1);
  int32_t skip;
  bool in;
  const int32_t e = piece_start<V>(piece_of(a, (int32_t)blockIdx.y, l, &in), a.dim, &skip);
  float acc[V] = {};
  add_parts<V>(a, beg, end, g, groups, e, acc);
  join_groups<V>(acc, lds, lanes, groups);
  if (g == 0 && in) put_row<TG, V>(a, k, e, acc);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// Positions of a chunk: 1,024 chunks or fewer, unless they would be longer than
// kMaxChunk.
constexpr uint32_t kMinChunk = 64, kMaxChunk = 1024;

uint32_t grad_chunk(int64_t n) {
  uint32_t c = kMinChunk;
  while (c < kMaxChunk && (int64_t)c * 1024 < n) c *= 2;
  return c;
}

// The sort of n ids: by counting (tiles = 1), or by passes over tiles of a block
// each.
struct SortShape {
  int tiles, threads, digit;   // digit: most bits of one
  bool small;
};

SortShape sort_shape(int64_t n) {
  if (n <= kRankMost) return {n > 0 ? 1 : 0, kRankBlock, 0, true};
  const int64_t small = cdiv(n, kSmallTile);
  if (small <= kSmallSortTiles)
    return {(int)small, kSmallThreads, digit_limit(kSmallTile), true};
  return {(int)cdiv(n, kLargeTile), kLargeThreads, digit_limit(kLargeTile), false};
}

struct EmbedWs {
  uint32_t *key[2], *pos[2];
  int32_t* hist;
  float* part;
};

size_t embed_ws_layout(int64_t n, int32_t dim, char* base, EmbedWs* out) {
  Carve c{base, 0, 0};
  EmbedWs w;
  // The most that any m <= n takes, so that a workspace serves smaller calls.
  const int64_t counters =
      std::max(std::min<int64_t>(cdiv(n, kSmallTile), kSmallSortTiles) << digit_limit(kSmallTile),
               cdiv(n, kLargeTile) << digit_limit(kLargeTile));
  const int64_t chunks =
      std::max(std::min<int64_t>(cdiv(n, kMinChunk), 1024), cdiv(n, kMaxChunk));
  for (int i = 0; i < 2; ++i) {
    w.key[i] = c.take<uint32_t>((size_t)n);
    w.pos[i] = c.take<uint32_t>((size_t)n);
  }
  w.hist = c.take<int32_t>((size_t)counters);
  w.part = c.take<float>((size_t)chunks * 2 * dim);
  if (out) *out = w;
  return align_up(c.used, 256);
}

constexpr int kFillLanes = 1024 * 1024;      // most lanes that clear rows in a launch
constexpr int64_t kClearBytes = 320LL << 20;

struct Lanes {
  int32_t pieces, lanes_log, tiles;
};

Lanes lanes_of(int32_t dim, int vec) {
  Lanes r;
  r.pieces = (int32_t)cdiv(dim, vec);
  r.lanes_log = 0;
  while (r.lanes_log < 6 && (1 << r.lanes_log) < r.pieces) ++r.lanes_log;
  r.tiles = (int32_t)cdiv(r.pieces, 1 << r.lanes_log);
  return r;
}

template <typename TI, typename TO>
int launch_lookup(LookupArgs& a, hipStream_t stream) {
  // The wider type's pieces are 16 bytes.
  constexpr int V = sizeof(TI) > sizeof(TO) ? kVec<TI> : kVec<TO>;
  const bool wide = a.dim >= V;
  a.pieces = (uint32_t)cdiv(a.dim, wide ? V : 1);
  a.pmagic = div_magic(a.pieces);
  const uint64_t total = (uint64_t)a.n * a.pieces;
  GG_REQUIRE(total <= 1ULL << 32, "%lld rows of %d elements are too many for one call",
             (long long)a.n, a.dim);
  a.stream = (int64_t)sizeof(TO) * a.n * a.dim > kStreamBytes;
  // One piece per lane while that leaves lanes idle, two in flight after (four
  // and eight: 1.5M rows of 100 fp32 221 and 229 us, two 216).
  const int u = total < 256 * 1024 ? 1 : 2;
  const dim3 grid((unsigned)((total + kBlock * u - 1) / (kBlock * u)));
  if (!wide)
    hipLaunchKernelGGL((k_embed_rows<TI, TO, 1, 2>),
                       dim3((unsigned)((total + kBlock * 2 - 1) / (kBlock * 2))), dim3(kBlock), 0,
                       stream, a);
  else if (u == 1)
    hipLaunchKernelGGL((k_embed_rows<TI, TO, V, 1>), grid, dim3(kBlock), 0, stream, a);
  else
    hipLaunchKernelGGL((k_embed_rows<TI, TO, V, 2>), grid, dim3(kBlock), 0, stream, a);
  GG_LAUNCH_CHECK("k_embed_rows");
  return GG_OK;
}

template <typename TD, typename TG, int V>
int launch_grad(GradArgs& a, hipStream_t stream) {
  const int64_t chunks = cdiv(a.n, a.chunk);
  a.part_blocks = chunks > 1 ? (uint32_t)(chunks * a.tiles) : 0u;
  const int64_t blocks = a.part_blocks + cdiv(a.by_position ? a.n : a.rows, a.per);
  if (blocks > 0) {
    if (a.add)
      hipLaunchKernelGGL((k_grad_rows<TD, TG, V, true>), dim3((unsigned)blocks), dim3(kBlock), 0,
                         stream, a);
    else
      hipLaunchKernelGGL((k_grad_rows<TD, TG, V, false>), dim3((unsigned)blocks), dim3(kBlock), 0,
                         stream, a);
    GG_LAUNCH_CHECK("k_grad_rows");
  }
  if (chunks > 1) {
    hipLaunchKernelGGL((k_grad_long<TG, V>), dim3((unsigned)chunks - 1, (unsigned)a.tiles),
                       dim3(kBlock), 0, stream, a);
    GG_LAUNCH_CHECK("k_grad_long");
  }
  return GG_OK;
}

}  // namespace
}  // namespace gg

using namespace gg;

extern "C" int gg_embed_forward(const gg_rows_t* table, int64_t num_rows, int32_t dim,
                                const void* ids_d, int32_t id_bits, int64_t n, float scale,
                                const gg_rows_t* out, int32_t* status_d, hipStream_t stream) {
  GG_REQUIRE(status_d, "status is NULL");
  GG_REQUIRE(dim >= 1 && dim <= GG_EMBED_MAX_DIM, "dim %d outside 1..%d", dim, GG_EMBED_MAX_DIM);
  GG_REQUIRE(num_rows >= 0 && n >= 0 && n <= 1LL << 33, "num_rows %lld or n %lld invalid",
             (long long)num_rows, (long long)n);
  GG_REQUIRE(id_bits == 32 || id_bits == 64, "ids of %d bits", id_bits);
  GG_REQUIRE((uintptr_t)ids_d % (id_bits / 8) == 0, "ids are not aligned");
  LookupArgs a = {};
  int rc = pack_rows(table, "table", num_rows, dim, kBitFloats | kBitE4M3, false, &a.table);
  if (rc == GG_OK) rc = pack_rows(out, "out", n, dim, kBitFloats, true, &a.out);
  if (rc != GG_OK || n == 0) return rc;
  a.ids = ids_d;
  a.id_bits = id_bits;
  a.dim = dim;
  a.rows = num_rows;
  a.n = n;
  a.scale = scale;
  a.glog = a.table.group ? __builtin_ctz((unsigned)a.table.group) : 31;
  a.status = status_d;
  GG_FOR_FLOAT(out->dtype, TO, {
    if (table->dtype == GG_E4M3) return launch_lookup<e4m3, TO>(a, stream);
    GG_FOR_FLOAT(table->dtype, TI, { return launch_lookup<TI, TO>(a, stream); });
  });
}

extern "C" size_t gg_ws_embed(int64_t n, int64_t num_rows, int32_t dim) {
  if (n < 0 || n > INT32_MAX - 1 || num_rows < 0 || num_rows > INT32_MAX - 1 || dim < 1 ||
      dim > GG_EMBED_MAX_DIM)
    return 0;
  return embed_ws_layout(n, dim, nullptr, nullptr);
}

extern "C" int gg_embed_backward(const gg_rows_t* dy, const void* ids_d, int32_t id_bits, int64_t n,
                                 int64_t num_rows, int32_t dim, float scale, const gg_rows_t* grad,
                                 int32_t flags, int32_t* status_d, void* ws, size_t ws_bytes,
                                 hipStream_t stream) {
  GG_REQUIRE(status_d, "status is NULL");
  GG_REQUIRE(dim >= 1 && dim <= GG_EMBED_MAX_DIM, "dim %d outside 1..%d", dim, GG_EMBED_MAX_DIM);
  GG_REQUIRE(n >= 0 && n <= INT32_MAX - 1, "n = %lld unsupported", (long long)n);
  GG_REQUIRE(num_rows >= 0 && num_rows <= INT32_MAX - 1, "num_rows %lld unsupported",
             (long long)num_rows);
  GG_REQUIRE(id_bits == 32 || id_bits == 64, "ids of %d bits", id_bits);
  GG_REQUIRE(n == 0 || ids_d, "ids are NULL");
  GG_REQUIRE((uintptr_t)ids_d % (id_bits / 8) == 0, "ids are not aligned");
  GG_REQUIRE((flags & ~GG_EMBED_ADD) == 0, "unknown flags %d", flags);
  GradArgs a = {};
  int rc = pack_rows(dy, "dy", n, dim, kBitFloats, false, &a.dy);
  if (rc == GG_OK) rc = pack_rows(grad, "grad", num_rows, dim, kBitFloats, true, &a.grad);
  if (rc != GG_OK) return rc;
  const size_t need = embed_ws_layout(n, dim, nullptr, nullptr);
  GG_REQUIRE(n == 0 || (ws && (uintptr_t)ws % 8 == 0 && ws_bytes >= need),
             "workspace of %zu bytes < %zu, or not aligned", ws_bytes, need);
  a.add = flags & GG_EMBED_ADD;
  if (n == 0 && (a.add || num_rows == 0)) return GG_OK;      // (ids are looked at in any case)
  EmbedWs w = {};
  if (n > 0) embed_ws_layout(n, dim, (char*)ws, &w);

  // The sort, of as many passes as the ids' width needs.
  Keys k = {};
  k.ids = ids_d;
  k.id_bits = id_bits;
  k.n = n;
  k.rows = (uint32_t)num_rows;
  k.status = status_d;
  const int key_bits = 32 - __builtin_clz((unsigned)std::max<int64_t>(num_rows, 1));
  const SortShape sh = sort_shape(n);
  const int tiles = sh.tiles, most = sh.digit;
  const int passes = most ? (int)cdiv(key_bits, most) : 1, digit = (int)cdiv(key_bits, passes);
  // Either the sort's launches clear all rows beside their own work and only rows
  // that occur are written after it, or the pass after it goes over all rows.
  // Clearing is faster where ids reach few of the rows (from one id per two rows
  // on their first stores count twice), and where the sort's launches hide
  // all of it, up to kClearBytes (fp32 rows into 200,000, 200,003 ids of a window:
  // of 256 115 us, 120 by rows; of 384 161, 162; of 512 207, 199; of 602 294, 262;
  // ids by a power law of 256 105, 138; one launch hides less: 16,000 bf16 rows
  // of 2,048 58, 50).  Many ids to a row leave nothing to clear: 1M in 5,000 95, 90.
  const int32_t row_bytes = dim * (int32_t)elem_bytes(grad->dtype);
  const bool hidden = tiles > 1 && n <= 8 * num_rows && num_rows * row_bytes <= kClearBytes;
  a.by_position = a.add || (n > 0 && (n * 2 <= num_rows || hidden));
  const bool clear = a.by_position && !a.add;
  FillArgs f = {};
  f.p = a.grad.p;
  f.stride = a.grad.stride;
  f.row_bytes = row_bytes;
  const Lanes fl = lanes_of(f.row_bytes, f.row_bytes >= 16 ? 16 : 2);
  f.pieces = fl.pieces;
  f.lanes_log = fl.lanes_log;
  const int launches = tiles == 1 ? 1 : 2 * passes;
  int launched = 0;
  // Blocks that clear the next launch's share of the rows.
  const auto fill_blocks = [&](int threads) {
    f.r0 = num_rows * launched / launches;
    f.r1 = num_rows * (launched + 1) / launches;
    ++launched;
    if (!clear) return 0;
    const int64_t want = cdiv((f.r1 - f.r0) << f.lanes_log, threads);
    return (int)std::min<int64_t>(want, kFillLanes / threads);
  };
  int at = 0;
  if (tiles == 1) {
    const int blocks = (int)cdiv(n, kWave);
    hipLaunchKernelGGL(k_sort_rank, dim3((unsigned)(blocks + fill_blocks(kRankBlock))),
                       dim3(kRankBlock), 0, stream, k, blocks, w.key[0], w.pos[0], f);
    GG_LAUNCH_CHECK("k_sort_rank");
  } else if (tiles > 1) {
    for (int p = 0; p < passes; ++p) {
      k.shift = p * digit;
      k.bits = std::min(digit, key_bits - k.shift);
      at = p & 1;
      const dim3 threads((unsigned)sh.threads);
      dim3 grid((unsigned)(tiles + fill_blocks(sh.threads)));
      if (sh.small)
        hipLaunchKernelGGL((k_sort_count<kSmallThreads, kSmallKeys>), grid, threads, 0, stream, k,
                           w.hist, tiles, f);
      else
        hipLaunchKernelGGL((k_sort_count<kLargeThreads, kLargeKeys>), grid, threads, 0, stream, k,
                           w.hist, tiles, f);
      GG_LAUNCH_CHECK("k_sort_count");
      grid.x = (unsigned)(tiles + fill_blocks(sh.threads));
      if (sh.small)
        hipLaunchKernelGGL((k_sort_scatter<kSmallThreads, kSmallKeys>), grid, threads, 0, stream, k,
                           w.hist, tiles, w.key[at], w.pos[at], f);
      else
        hipLaunchKernelGGL((k_sort_scatter<kLargeThreads, kLargeKeys>), grid, threads, 0, stream, k,
                           w.hist, tiles, w.key[at], w.pos[at], f);
      GG_LAUNCH_CHECK("k_sort_scatter");
      k.ids = nullptr;
      k.key = w.key[at];
      k.pos = w.pos[at];
    }
  }

  a.key = w.key[at];
  a.pos = w.pos[at];
  a.n = (uint32_t)n;
  a.rows = (uint32_t)num_rows;
  a.dim = dim;
  a.scale = scale;
  a.part = w.part;
  a.chunk = grad_chunk(n);
  GG_FOR_FLOAT(dy->dtype, TD, {
    constexpr int V = kVec<TD>;
    const Lanes l = lanes_of(dim, dim >= V ? V : 1);
    a.pieces = l.pieces;
    a.lanes_log = l.lanes_log;
    a.tiles = l.tiles;
    // A last piece alone in its tile gets the one before it beside it (there is
    // room: the tile has all other lanes free).
    a.shift = l.tiles > 1 && l.pieces % (1 << l.lanes_log) == 1 ? 1 : 0;
    a.tmagic = div_magic((uint32_t)l.tiles);
    // Rows of a block: what its groups take at a time, as far as these rows
    // have no more than 512 positions together, and more while that leaves 8,192
    // blocks.
    const int64_t all = a.by_position ? n : num_rows;
    const int64_t fill = (kBlock >> l.lanes_log) * kItems<V> / l.tiles;
    a.per = 1;
    while (a.per < kGradRows &&
           (a.per * 8192LL <= all ||
            (a.per * 2LL <= fill && (a.by_position || a.per * 2LL * n <= 512 * num_rows))))
      a.per *= 2;
    GG_FOR_FLOAT(grad->dtype, TG, {
      return dim >= V ? launch_grad<TD, TG, V>(a, stream) : launch_grad<TD, TG, 1>(a, stream);
    });
  });
}
