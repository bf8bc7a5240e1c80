// Distillation from a teacher's top logits, forward and backward.
//
// With T the temperature, p = softmax(t / T) over a row's entries and
// q = softmax(z / T) over the vocabulary:
//   loss = a T^2 sum_k p_k (log p_k - log q[id_k]),  a = weight * row_w
//   dz_j = a T (q_j - sum of p_k over the entries with id_k = j).
#include "rows.hpp"

namespace gg {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.69314718055994531f;

struct DistillArgs {
  KRows z, top, dz;
  const char* ids;             // row r's at ids + r * ids_stride
  int64_t ids_stride;
  int32_t ids64, k;
  int32_t kp;                  // k rounded up to 4: entries in LDS
  int32_t top_dtype;
  int32_t vocab;
  int64_t n;
  float temp, inv_temp;        // T, 1 / T
  float c2;                    // log2(e) / T
  float t_ln2;                 // T log(2)
  float weight;
  const float* row_w;          // nullptr: ones
  float* loss;
  float* lse;
  const float* lse_in;         // backward: as the forward call wrote it
  bool past;                   // the gradient goes past the caches
  int32_t lanes_log;
  int32_t splits;              // blocks of a row
  int32_t chunk;               // pieces of a split
  float2* part;                // [n][splits]: maximum of z, sum of exp((z - maximum) / T)
  float2* lesson;              // [n]: sum p (T log p - (z - pivot)); the pivot, -infinity
                               // where the row has no lesson
  int32_t* status;
};

// exp((z - m) / T) as 2^(z c2 - b), c2 = log2(e) / T and b = m c2: one fused
// multiply-add, rounded once, and the same b in a sum and in what is divided
// by it, so that b's own rounding, up to 2^6 where |b| is 2^31, cancels.  Beyond
// (all logits at -1e30 or the type's lowest value, say, or a tiny T) logits which
// differ at all differ by 2^7 at least, far too much to count, so c2 becomes a power
// of two under which m c2 is exact and the least difference is 2^10.
struct Soft {
  float m, c2, b;
  bool coarse;
};

__device__ __forceinline__ Soft soft_of(float m, float c2) {
  if (m == -INFINITY) return {m, c2, 0.0f, false};     // masked logits give 0
  const float b = m * c2;
  if (fabsf(b) > 0x1p31f && fabsf(m) <= 3.4028235e38f) {
    const uint32_t e = (__float_as_uint(m) >> 23) & 255u;
    const float c = __uint_as_float((254u + 34u - e) << 23);
    return {m, c, m * c, true};
  }
  return {m, c2, b, false};
}

__device__ __forceinline__ float exp_of(float z, const Soft& s) {
  return __builtin_amdgcn_exp2f(__builtin_fmaf(z, s.c2, -s.b));
}

// What a sum relative to a counts for relative to the larger maximum of t.
__device__ __forceinline__ float factor(const Soft& a, const Soft& t) {
  if (a.m == t.m) return 1.0f;
  return a.coarse || t.coarse || a.m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(a.b - t.b);
}

__device__ __forceinline__ float weight_of(const DistillArgs& a, int64_t row) {
  return a.row_w ? a.weight * a.row_w[row] : a.weight;
}

struct MaxSum {
  float m, s;     // largest logit; sum of exp((z - m) / T)
};

__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c2) {
  const Soft t = soft_of(fmaxf(a.m, b.m), c2);
  return {t.m, a.s * factor(soft_of(a.m, c2), t) + b.s * factor(soft_of(b.m, c2), t)};
}

// The statistics of `lanes` lanes, or of a block's waves, relative to their
// common maximum.
__device__ __forceinline__ MaxSum join_lanes(MaxSum st, int lanes, float c2) {
  const Soft t = soft_of(lanes_maxf(st.m, lanes), c2);
  return {t.m, lanes_sum(st.s * factor(soft_of(st.m, c2), t), lanes)};
}

__device__ __forceinline__ MaxSum join_waves(const float2* part, int waves, float c2) {
  float m = part[0].x, s = 0.0f;
#pragma unroll 1
  for (int w = 1; w < waves; ++w) m = fmaxf(m, part[w].x);
  const Soft t = soft_of(m, c2);
#pragma unroll 1
  for (int w = 0; w < waves; ++w) s += part[w].y * factor(soft_of(part[w].x, c2), t);
  return {m, s};
}

__device__ __forceinline__ float lse_of(const MaxSum& st, const Soft& t, float inv_temp) {
  const float l2 = __builtin_amdgcn_logf(st.s);       // -infinity for a row of none
  return t.coarse ? t.m * inv_temp + kLn2 * l2 : kLn2 * (t.b + l2);
}

// An lse from which the backward call does not take q: q's relative error is a few
// times |lse| 2^-24, and an lse beside a logit of -1e30 does not hold the number of
// logits that share it.  The row's statistics are computed again where that
// matters (2^-10 of q here; the gradient of a 16-bit row has 2^-9 at best).
constexpr float kFarLse = 4096.0f;

__device__ __forceinline__ bool is_far(float weight, float lse) {
  return weight != 0.0f && !(fabsf(lse) < kFarLse);
}

// T log q of a logit, from the distance to the largest one: the difference of z / T
// and an lse loses log q where both are large.  Beyond 2^40 units of the exponent it
// is the distance itself, which is a number where z / T may be none (the type's lowest
// value, or a tiny T): losses are summed in these units and then scaled by T once
// more, since T^2 may be 0 or infinite too.
__device__ __forceinline__ float t_log_q(const DistillArgs& a, float z, const MaxSum& st,
                                         const Soft& t) {
  const float l2 = __builtin_amdgcn_logf(st.s), d = __builtin_fmaf(z, t.c2, -t.b);
  return t.coarse || fabsf(d) > 0x1p40f ? (z - t.m) - a.t_ln2 * l2 : a.t_ln2 * (d - l2);
}

// ---------------------------------------------------------------------------
// A row's entries, up to kPerLane for each of `lanes` lanes of one wave.  Their
// loads are issued around the row's own: the ids before it, the logits at the
// ids behind it.  LDS holds, per entry, its id (-1: none), p summed over the
// entries with that id, log2 of its own p, and z[id].
// ---------------------------------------------------------------------------
constexpr int kEntryBytes = 16;
constexpr int kPerLane = 4;
static_assert(kPerLane * kWave >= GG_DISTILL_MAX_K, "a wave holds all entries");

struct Entries {
  int32_t* id;
  float *p, *lp, *z;
};

__device__ __forceinline__ Entries entries_at(char* lds, int group, int k) {
  char* at = lds + (size_t)group * k * kEntryBytes;
  return {(int32_t*)at, (float*)(at + 4 * k), (float*)(at + 8 * k), (float*)(at + 12 * k)};
}

template <typename T>
struct Held {
  uint32_t lo[kPerLane], hi[kPerLane];   // words of the id; the same word of 32 bits
  uint16_t tl[kPerLane], th[kPerLane];   // halves of the logit; the same one of 16 bits
  int32_t id[kPerLane];                  // -1: none
  float t[kPerLane];
  typename Raw<T, 1>::vec z[kPerLane];   // the row's own logit there
};

// Issues the loads of ids and logits of any width, without a branch that would
// wait for them; lanes behind the last entry repeat it.
template <typename T>
__device__ __forceinline__ void load_entries(const DistillArgs& a, int64_t row, int l, int lanes,
                                             Held<T>& h) {
  const auto* ids = (const GG_GLOBAL uint32_t*)(a.ids + row * a.ids_stride);
  const auto* tp = (const GG_GLOBAL uint16_t*)(a.top.p + row * a.top.stride);
  const int iw = a.ids64 ? 2 : 1, tw = a.top_dtype == GG_F32 ? 2 : 1;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    h.lo[u] = h.hi[u] = 0;
    h.tl[u] = h.th[u] = 0;
    if (u * lanes < a.k) {
      const int j = min(u * lanes + l, a.k - 1);
      h.lo[u] = ids[j * iw];
      h.hi[u] = ids[j * iw + iw - 1];
      h.tl[u] = tp[j * tw];
      h.th[u] = tp[j * tw + tw - 1];
    }
  }
}

// Their values, and the loads of the row's logits at them (of the first where
// there is no entry).
template <typename T>
__device__ __forceinline__ void take_entries(const DistillArgs& a, int64_t row, int l, int lanes,
                                             Held<T>& h) {
  const char* zp = a.z.p + row * a.z.stride;
  bool bad = false;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    h.id[u] = -1;
    h.t[u] = -INFINITY;
    h.z[u] = {};
    if (u * lanes < a.k) {
      const bool own = u * lanes + l < a.k;
      const bool in = h.lo[u] < (uint32_t)a.vocab && (!a.ids64 || h.hi[u] == 0);
      bad |= own && !in && (h.lo[u] & h.hi[u]) != ~0u;
      const float wide = __uint_as_float((uint32_t)h.th[u] << 16 |
                                         (a.top_dtype == GG_F32 ? h.tl[u] : 0u));
      const float half = (float)__builtin_bit_cast(f16, h.th[u]);
      if (own && in) {
        h.id[u] = (int32_t)h.lo[u];
        h.t[u] = a.top_dtype == GG_F16 ? half : wide;
      }
      h.z[u] = raw_load<T, 1>(zp + max(h.id[u], 0) * (int64_t)sizeof(T));
    }
  }
  if (bad) set_status(a.status, GG_DEV_BAD_ID);
}

// Whether the row has a lesson: an entry with a logit above -infinity, or a NaN
// (which a maximum passes over), and a weight.  SUM: p is summed over equal ids (for the gradient).
template <bool SUM, typename T>
__device__ __forceinline__ bool share_entries(const DistillArgs& a, float weight, int l, int lanes,
                                              const Held<T>& h, const Entries& en) {
  float tm = h.t[0];
#pragma unroll
  for (int u = 1; u < kPerLane; ++u) tm = fmaxf(tm, h.t[u]);
  const Soft f = soft_of(lanes_maxf(tm, lanes), a.c2);
  float total = 0.0f;
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) total += exp_of(h.t[u], f);
  total = lanes_sum(total, lanes);
  const float log_total = __builtin_amdgcn_logf(total);
#pragma unroll
  for (int u = 0; u < kPerLane; ++u) {
    const int j = u * lanes + l;
    if (j < a.kp) {
      const float lp = __builtin_fmaf(h.t[u], f.c2, -f.b) - log_total;
      en.id[j] = h.id[u];
      en.lp[j] = lp;
      en.p[j] = __builtin_amdgcn_exp2f(lp);
    }
  }
  if constexpr (SUM) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float p[kPerLane] = {};
#pragma unroll 4
    for (int x = 0; x < a.kp; x += 4) {
      const int4 id = *(const int4*)(en.id + x);
      const float4 px = *(const float4*)(en.p + x);
#pragma unroll
      for (int u = 0; u < kPerLane; ++u)
        if (u * lanes < a.k) {
          p[u] += h.id[u] == id.x ? px.x : 0.0f;
          p[u] += h.id[u] == id.y ? px.y : 0.0f;
          p[u] += h.id[u] == id.z ? px.z : 0.0f;
          p[u] += h.id[u] == id.w ? px.w : 0.0f;
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int u = 0; u < kPerLane; ++u)
      if (u * lanes + l < a.k) en.p[u * lanes + l] = p[u];
  }
  return !(total == 0.0f) && weight != 0.0f;
}

template <typename T>
__device__ __forceinline__ void share_logits(const DistillArgs& a, int l, int lanes,
                                             const Held<T>& h, const Entries& en) {
#pragma unroll
  for (int u = 0; u < kPerLane; ++u)
    if (u * lanes + l < a.k) en.z[u * lanes + l] = h.id[u] < 0 ? 0.0f : (float)h.z[u];
}

// sum_k p_k (T log p_k - t_log_qk(z_k)), by the same lanes.
template <typename F>
__device__ __forceinline__ float lesson_of(const DistillArgs& a, int l, int lanes,
                                           const Entries& en, F t_log_qk) {
  float v = 0.0f;
  for (int j = l; j < a.k; j += lanes) {
    const float p = en.id[j] < 0 ? 0.0f : __builtin_amdgcn_exp2f(en.lp[j]);
    if (p != 0.0f) v += p * (a.t_ln2 * en.lp[j] - t_log_qk(en.z[j]));
  }
  return lanes_sum(v, lanes);
}

// The gradient at the entries' own places in [lo, hi), after the rest of the
// row is stored.
template <typename T>
__device__ __forceinline__ void store_entries(const DistillArgs& a, int64_t row, int l, int lanes,
                                              const Entries& en, float c, float inv, const Soft& t,
                                              int32_t lo, int32_t hi) {
  for (int j = l; j < a.k; j += lanes) {
    const int32_t id = en.id[j];
    if (id < lo || id >= hi) continue;
    const float v[1] = {c * (inv * exp_of(en.z[j], t) - en.p[j])};
    row_store<T, 1>(a.dz.p + row * a.dz.stride + id * (int64_t)sizeof(T), v);
  }
}

// ---------------------------------------------------------------------------
// A row in registers: read once, written once.  The row's whole pieces are
// dealt to a group of lanes (part of a wave, or a block); its last elements,
// fewer than a piece, go to the first lanes, one each.
//
// Bound by memory where rows are long: 4,096 of 128,000 bf16, loss and gradient
// 400 us, 5.2 TB/s read and written; the loss alone 214, 4.9; of 50,000 x 1,500 fp32
// 49 us, 6.1.  Short rows are bound by what a row costs beside its logits, its
// entries' softmax and the reductions: 1M of 9 with 5 entries 55 us.  Rows that do
// not start at 16 bytes have single elements up to the first boundary: 4,096 of 128,001
// bf16 404 us, 5.2 TB/s (whole pieces from the row's start 506, every access of a wave
// touching one line more).
// ---------------------------------------------------------------------------
enum { kLossOnly = 0, kFused = 1, kBackward = 2 };

// Keeps the row in its own type between the passes over it: unseen by the
// compiler, which would hold the converted values, twice as large, as well.
template <typename R, int N>
__device__ __forceinline__ void keep_packed(R (&raw)[N]) {
#pragma unroll
  for (int t = 0; t < N; ++t)
    if constexpr (sizeof(R) == 16) {
      auto w = __builtin_bit_cast(u32x4, raw[t]);
      asm volatile("" : "+v"(w));
      raw[t] = __builtin_bit_cast(R, w);
    }
}

// How a row is cut: its elements up to the first 16-byte boundary, whole pieces
// from there, and what is left.  Single elements take a lane each, 14 at most, so
// rows that share a wave start with a piece, on the boundary or not.
struct Cut {
  int head, pieces;
  // The single element of lane l, where there is one.
  template <int V>
  __device__ __forceinline__ int single(int l) const {
    return l < head ? l : pieces * V + l;
  }
};

template <typename T, int V>
__device__ __forceinline__ Cut cut_of(const char* row, int vocab, int lanes) {
  const int head = V > 1 && lanes >= 16 && vocab >= 2 * V
                       ? (int)((0 - (uint32_t)(uintptr_t)row) & 15u) / (int)sizeof(T) : 0;
  return {head, (vocab - head) / V};
}

template <typename T, int V, int STEPS, bool BLK, int MODE>
__global__ void __launch_bounds__(BLK ? 1024 : kBlock) k_distill_rows(DistillArgs a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ float2 s_part[1024 / kWave];
  __shared__ int32_t s_has;
  const int lanes = BLK ? (int)blockDim.x : 1 << a.lanes_log;
  const int64_t row = BLK ? block_index() : (block_index() * kBlock + threadIdx.x) >> a.lanes_log;
  if (row >= a.n) return;
  const int l = BLK ? (int)threadIdx.x : (int)threadIdx.x & (lanes - 1);
  constexpr int kPiece = V * (int)sizeof(T);
  const char* zp = a.z.p + row * a.z.stride;
  const Cut cut = cut_of<T, V>(zp, a.vocab, lanes);
  const int pieces = cut.pieces, rest = a.vocab - pieces * V;
  const int single = cut.single<V>(l);

  const int el = BLK ? min(lanes, kWave) : lanes;     // lanes that read the entries
  const Entries en = entries_at(lds, BLK ? 0 : (int)threadIdx.x >> a.lanes_log, a.kp);
  Held<T> held;
  if (l < el) load_entries(a, row, l, el, held);
  const float weight = weight_of(a, row);
  // (lanes behind the last piece repeat it: a load in a branch would be waited for
  // with the entries)
  typename Raw<T, V>::vec raw[STEPS];
#pragma unroll
  for (int t = 0; t < STEPS; ++t)
    raw[t] = raw_load<T, V>(zp + cut.head * (int)sizeof(T) +
                            (int64_t)min(t * lanes + l, pieces - 1) * kPiece);
  const auto raw_last = raw_load<T, 1>(zp + min(single, a.vocab - 1) * (int64_t)sizeof(T));
  bool has = false;
  if (l < el) {
    take_entries(a, row, l, el, held);
    has = share_entries<MODE != kLossOnly>(a, weight, l, el, held, en);
    if (BLK && l == 0) s_has = has;
  }
  const float last[1] = {l < rest ? (float)raw_last : -INFINITY};

  // Softmax statistics: q_j = inv * exp_of(z_j, top).
  Soft top;
  float inv = 1.0f, lse = 0.0f;
  MaxSum all = {};
  bool empty, fresh = true;
  if constexpr (MODE == kBackward) {
    lse = a.lse_in[row];
    fresh = is_far(weight, lse);
    if (l < el) share_logits(a, l, el, held, en);
  }
  if (fresh) {
    float m = last[0];
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
      if (t * lanes + l < pieces) {
        float v[V];
        to_f32<T, V>(raw[t], v);
#pragma unroll
        for (int k = 0; k < V; ++k) m = fmaxf(m, v[k]);
      }
    keep_packed(raw);
    if (MODE != kBackward && l < el) share_logits(a, l, el, held, en);
    top = soft_of(lanes_maxf(m, min(lanes, kWave)), a.c2);
    float s = exp_of(last[0], top);
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
      if (t * lanes + l < pieces) {
        float v[V], sum = 0.0f;
        to_f32<T, V>(raw[t], v);
#pragma unroll
        for (int k = 0; k < V; ++k) sum += exp_of(v[k], top);
        s += sum;
      }
    if constexpr (MODE != kLossOnly) keep_packed(raw);
    all = {top.m, lanes_sum(s, min(lanes, kWave))};
    if constexpr (BLK) {
      if (lane_id() == 0) s_part[threadIdx.x / kWave] = make_float2(all.m, all.s);
      __syncthreads();
      all = join_waves(s_part, lanes / kWave, a.c2);
      top = soft_of(all.m, a.c2);
    }
    // Sums are about 1 at least, but for a row of which every logit is -infinity.
    empty = all.s == 0.0f;
    inv = 1.0f / all.s;
    lse = lse_of(all, top, a.inv_temp);
  } else {
    empty = lse == -INFINITY;
    top = soft_of(lse * a.temp, a.c2);
    if (BLK) __syncthreads();
  }
  if (BLK) has = s_has;
  has = has && !empty;
  if constexpr (MODE != kBackward) {
    if (l < el) {
      const float v =
          has ? lesson_of(a, l, el, en, [&](float z) { return t_log_q(a, z, all, top); }) : 0.0f;
      if (l == 0) {
        a.loss[row] = has ? weight * (a.temp * v) : 0.0f;
        if (a.lse) a.lse[row] = lse;
      }
    }
  }
  if constexpr (MODE == kLossOnly) return;

  char* d0 = a.dz.p + row * a.dz.stride;
  char* dp = d0 + cut.head * (int)sizeof(T);
  if (!has) {      // the same for the whole row
    const float zero[V] = {}, one[1] = {0.0f};
#pragma unroll
    for (int t = 0; t < STEPS; ++t)
      if (t * lanes + l < pieces) row_store<T, V>(dp + (int64_t)(t * lanes + l) * kPiece, zero);
    if (l < rest) row_store<T, 1>(d0 + single * (int64_t)sizeof(T), one);
    return;
  }
  const float c = weight * a.temp, ci = c * inv;
#pragma unroll
  for (int t = 0; t < STEPS; ++t)
    if (t * lanes + l < pieces) {
      float v[V];
      to_f32<T, V>(raw[t], v);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = ci * exp_of(v[k], top);
      row_store<T, V>(dp + (int64_t)(t * lanes + l) * kPiece, v);
    }
  if (l < rest) {
    const float v[1] = {ci * exp_of(last[0], top)};
    row_store<T, 1>(d0 + single * (int64_t)sizeof(T), v);
  }
  if constexpr (BLK)
    __syncthreads();
  else
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (l < el) store_entries<T>(a, row, l, el, en, c, inv, top, 0, a.vocab);
}

// ---------------------------------------------------------------------------
// Rows that do not fit the registers of a block, and few long rows: several
// blocks per row, the statistics joined by the blocks of a second launch.
// ---------------------------------------------------------------------------
constexpr int kSplitUnroll = 4;

// A block's pieces from p on, kSplitUnroll per lane; those past p1 repeat the first.
template <typename T, int V>
__device__ __forceinline__ void load_batch(const char* zp, int p, int p1,
                                           typename Raw<T, V>::vec (&raw)[kSplitUnroll]) {
#pragma unroll
  for (int u = 0; u < kSplitUnroll; ++u) {
    const int q = p + u * kBlock;
    raw[u] = raw_load<T, V>(zp + (int64_t)(q < p1 ? q : p) * 16);
  }
}

// Statistics of a lane's share of the pieces [p0, p1) and, with `end`, of the row's
// last elements.
template <typename T, int V>
__device__ __forceinline__ MaxSum lane_stats(const DistillArgs& a, const char* zp, int p0, int p1,
                                             bool end) {
  const int tid = threadIdx.x, pieces = a.vocab / V, rest = a.vocab - pieces * V;
  MaxSum st = {-INFINITY, 0.0f};
  for (int p = p0 + tid; p < p1; p += kBlock * kSplitUnroll) {
    typename Raw<T, V>::vec raw[kSplitUnroll];
    load_batch<T, V>(zp, p, p1, raw);
    // (the repeated pieces do not change the maximum)
    float v[V], m = st.m;
#pragma unroll
    for (int u = 0; u < kSplitUnroll; ++u) {
      to_f32<T, V>(raw[u], v);
#pragma unroll
      for (int k = 0; k < V; ++k) m = fmaxf(m, v[k]);
    }
    const Soft top = soft_of(m, a.c2);
    st.s *= factor(soft_of(st.m, a.c2), top);
    st.m = m;
#pragma unroll
    for (int u = 0; u < kSplitUnroll; ++u) {
      to_f32<T, V>(raw[u], v);
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < V; ++k) s += exp_of(v[k], top);
      st.s += p + u * kBlock < p1 ? s : 0.0f;
    }
  }
  if (end && tid < rest) {
    float v[1];
    row_load<T, 1>(zp + (pieces * V + tid) * (int64_t)sizeof(T), v);
    // (2^(z c2 - b) of the largest logit itself is 1 only up to b's rounding)
    st = join(st, {v[0], exp_of(v[0], soft_of(v[0], a.c2))}, a.c2);
  }
  return st;
}

// Statistics of one split of a row; the last block of a row has its lesson
// instead, as far as it needs no statistics and while z is still whole (the
// gradient may take its place).  12 rows of 64 splits 5.3 us: one pass over a
// split and the joins; 2,000 rows of 262,144 fp32 4.9 TB/s.
template <typename T, int V>
__global__ void __launch_bounds__(kBlock) k_distill_stats(DistillArgs a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ float2 s_part[kBlock / kWave];
  const int64_t row = block_index() / (a.splits + 1);
  const int c = (int)(block_index() - row * (a.splits + 1));
  if (row >= a.n) return;
  const int tid = threadIdx.x;
  if (c == a.splits) {
    if (tid >= kWave) return;
    const Entries en = entries_at(lds, 0, a.kp);
    Held<T> held;
    load_entries(a, row, tid, kWave, held);
    take_entries(a, row, tid, kWave, held);
    const bool has = share_entries<false>(a, weight_of(a, row), tid, kWave, held, en);
    share_logits(a, tid, kWave, held, en);
    // Relative to the largest of the entries' logits, whose log q is known later.
    float pivot = -INFINITY;
#pragma unroll
    for (int u = 0; u < kPerLane; ++u)
      if (held.id[u] >= 0) pivot = fmaxf(pivot, (float)held.z[u]);
    pivot = lanes_maxf(pivot, kWave);
    if (pivot == -INFINITY) pivot = 0.0f;
    const float v = lesson_of(a, tid, kWave, en, [&](float z) { return z - pivot; });
    if (tid == 0) a.lesson[row] = make_float2(v, has ? pivot : -INFINITY);
    return;
  }
  const int p0 = c * a.chunk, p1 = min(a.vocab / V, p0 + a.chunk);
  const char* zp = a.z.p + row * a.z.stride;
  MaxSum st = lane_stats<T, V>(a, zp, p0, p1, c == a.splits - 1);
  st = join_lanes(st, kWave, a.c2);
  if (lane_id() == 0) s_part[tid / kWave] = make_float2(st.m, st.s);
  __syncthreads();
  if (tid == 0) {
    st = join_waves(s_part, kBlock / kWave, a.c2);
    a.part[row * a.splits + c] = make_float2(st.m, st.s);
  }
}

// All parts of a row joined, by every wave that calls it.
__device__ __forceinline__ MaxSum row_stats(const DistillArgs& a, int64_t row) {
  MaxSum st = {-INFINITY, 0.0f};
  for (int x = lane_id(); x < a.splits; x += kWave) {
    const float2 v = a.part[row * a.splits + x];
    st = join(st, {v.x, v.y}, a.c2);
  }
  return join_lanes(st, kWave, a.c2);
}

__device__ __forceinline__ void store_loss(const DistillArgs& a, int64_t row, float2 lesson,
                                           const MaxSum& st, const Soft& t) {
  const float weight = weight_of(a, row);
  a.loss[row] = lesson.y != -INFINITY && st.s != 0.0f
                    ? weight * (a.temp * (lesson.x - t_log_q(a, lesson.y, st, t))) : 0.0f;
  if (a.lse) a.lse[row] = lse_of(st, t, a.inv_temp);
}

// The loss alone: a wave per row.  3 us for few rows, an empty launch's time.
__global__ void __launch_bounds__(kWave) k_distill_loss(DistillArgs a) {
  const int64_t row = block_index();
  if (row >= a.n) return;
  const float2 lesson = a.lesson[row];
  const MaxSum st = row_stats(a, row);
  if (threadIdx.x == 0)
    store_loss(a, row, lesson, st, soft_of(st.m, a.c2));
}

// The gradient of one split: reads it again and writes it.  64 rows of 262,144 fp32
// 25 us with the gradient alone, 5.3 TB/s; 12 of 64 splits 7.6 us, whose first half
// is the wait for ids, then logits at them, beside the split's own loads.  A far lse's
// row is one block's: 64 rows of 262,144 bf16 126 us instead of 18, 12 of 200,003
// fp32 112 instead of 8, one of 2^24 bf16 4.2 ms.  (That path takes registers, 86
// instead of 47 in 16 bits and so five waves a SIMD instead of eight, but no time:
// 64 rows of 262,144 bf16 17.5 us with it and 17.6 without, 512 107 both.)
template <typename T, int V, int MODE>
__global__ void __launch_bounds__(kBlock) k_distill_finish(DistillArgs a) {
  extern __shared__ __align__(16) char lds[];
  __shared__ int32_t s_has;
  __shared__ float2 s_part[kBlock / kWave];
  const int64_t row = block_index() / a.splits;
  const int c = (int)(block_index() - row * a.splits);
  if (row >= a.n) return;
  const int tid = threadIdx.x;
  const int pieces = a.vocab / V, rest = a.vocab - pieces * V;
  const int p0 = c * a.chunk;
  int p1 = min(pieces, p0 + a.chunk);
  bool end = c == a.splits - 1;
  const char* zp = a.z.p + row * a.z.stride;
  char* dp = a.dz.p + row * a.dz.stride;
  const Entries en = entries_at(lds, 0, a.kp);
  Held<T> held;
  if (tid < kWave) load_entries(a, row, tid, kWave, held);
  const float weight = weight_of(a, row);
  typename Raw<T, V>::vec raw[kSplitUnroll];
  int p = p0 + tid;
  if (p < p1) load_batch<T, V>(zp, p, p1, raw);
  Soft top;                // q_j = inv * exp_of(z_j, top)
  float inv = 1.0f;
  bool empty;
  if constexpr (MODE == kFused) {
    const MaxSum st = row_stats(a, row);
    empty = st.s == 0.0f;
    top = soft_of(st.m, a.c2);
    inv = 1.0f / st.s;
    if (c == 0 && tid == 0)
      store_loss(a, row, a.lesson[row], st, top);
  } else {
    const float lse = a.lse_in[row];
    if (is_far(weight, lse)) {
      // One block has the whole row, which it reads before it writes any of it.
      if (c != 0) return;
      p1 = pieces;
      end = true;
      MaxSum st = join_lanes(lane_stats<T, V>(a, zp, 0, p1, true), kWave, a.c2);
      if (lane_id() == 0) s_part[tid / kWave] = make_float2(st.m, st.s);
      __syncthreads();
      st = join_waves(s_part, kBlock / kWave, a.c2);
      empty = st.s == 0.0f;
      top = soft_of(st.m, a.c2);
      inv = 1.0f / st.s;
      if (p < p1) load_batch<T, V>(zp, p, p1, raw);
    } else {
      empty = lse == -INFINITY;
      top = soft_of(lse * a.temp, a.c2);
    }
  }
  if (tid < kWave) {
    take_entries(a, row, tid, kWave, held);
    const bool has = share_entries<true>(a, weight, tid, kWave, held, en);
    share_logits(a, tid, kWave, held, en);
    if (tid == 0) s_has = has;
  }
  __syncthreads();         // and the entries' logits are read before any is overwritten
  const bool has = s_has && !empty;
  const float scale = weight * a.temp, ci = scale * inv;
  while (p < p1) {
#pragma unroll
    for (int u = 0; u < kSplitUnroll; ++u) {
      float v[V];
      to_f32<T, V>(raw[u], v);
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] = has ? ci * exp_of(v[k], top) : 0.0f;
      if (p + u * kBlock < p1) row_store<T, V>(dp + (int64_t)(p + u * kBlock) * 16, v, a.past);
    }
    p += kBlock * kSplitUnroll;
    if (p < p1) load_batch<T, V>(zp, p, p1, raw);
  }
  if (end && tid < rest) {
    float v[1];
    row_load<T, 1>(zp + (pieces * V + tid) * (int64_t)sizeof(T), v);
    v[0] = has ? ci * exp_of(v[0], top) : 0.0f;
    row_store<T, 1>(dp + (pieces * V + tid) * (int64_t)sizeof(T), v);
  }
  if (!has) return;
  __syncthreads();
  if (tid < kWave)
    store_entries<T>(a, row, tid, kWave, en, scale, inv, top, p0 * V, end ? a.vocab : p1 * V);
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
constexpr int kMaxSplits = 64;
constexpr int kMaxSteps = 16;         // pieces per lane of a block
// A row is dealt to as few lanes as have 4 pieces each, so that a wave works on
// several rows' entries at once, or to more (a piece a lane at most) while all rows
// leave lanes of the chip idle: 100,000 rows of 172 fp32 take 26 us with 16 lanes
// each and 71 with 64, 1M of 9 50 with 4 and 137 with 16.  A wave has rows of up
// to 8 pieces a lane to itself (50,000 rows of 1,500 fp32 110 us, in blocks of 4
// waves 190), blocks the longer ones.
constexpr int kWaveSteps = 8;
constexpr int64_t kFillLanes = 256 * 1024;
// Fewer rows than this are split if they have more pieces than that: 8 rows of
// 65,536 fp32 take 10.6 us in parts and 12.3 whole, 160 of them 27.7 and 19.8, 8 of
// 20,000 10.4 and 9.4.
constexpr int64_t kFewRows = 96;
constexpr int kSplitPieces = 8192;

int split_count(int64_t n) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, 1024 / std::max<int64_t>(n, 1)));
}

struct DistillWs {
  float2* part;
  float2* lesson;
};

size_t distill_ws_layout(int64_t n, char* base, DistillWs* out) {
  Carve c{base, 0, 0};
  DistillWs w;
  // (the most that any m <= n takes, so that a workspace serves smaller calls)
  w.part = c.take<float2>((size_t)std::min<int64_t>(kMaxSplits * n, std::max<int64_t>(1024, n)));
  w.lesson = c.take<float2>((size_t)n);
  if (out) *out = w;
  return align_up(c.used, 256);
}

template <typename T, int MODE>
int launch_rows(DistillArgs& a, hipStream_t stream) {
  constexpr int V = kVec<T>;
  const int pieces = a.vocab / V;
  const bool split = pieces > 1024 * kMaxSteps || (a.n < kFewRows && pieces > kSplitPieces);
  if (split) {
    a.splits = split_count(a.n);
    a.chunk = (int)cdiv(pieces, a.splits);
    // (rows that stay in registers are faster through the caches: 16,384 rows of
    // 16,001 fp32 455 and 408 us; 512 of 262,144 bf16 in parts 140 and 171)
    a.past = (int64_t)sizeof(T) * a.n * a.vocab > kStreamBytes;
    const size_t lds = (size_t)a.kp * kEntryBytes;
    if (MODE != kBackward) {
      hipLaunchKernelGGL((k_distill_stats<T, V>), grid_of(a.n * (a.splits + 1)), dim3(kBlock), lds,
                         stream, a);
      GG_LAUNCH_CHECK("k_distill_stats");
    }
    if constexpr (MODE == kLossOnly) {
      hipLaunchKernelGGL(k_distill_loss, grid_of(a.n), dim3(kWave), 0, stream, a);
      GG_LAUNCH_CHECK("k_distill_loss");
    } else {
      hipLaunchKernelGGL((k_distill_finish<T, V, MODE>), grid_of(a.n * a.splits), dim3(kBlock), lds,
                         stream, a);
      GG_LAUNCH_CHECK("k_distill_finish");
    }
    return GG_OK;
  }
  // (a row's last elements, fewer than V, take a lane each)
  a.lanes_log = V == 8 ? 3 : 2;
  if (pieces == 0) {       // rows of less than a piece
    while (kPerLane << a.lanes_log < a.k) ++a.lanes_log;
    hipLaunchKernelGGL((k_distill_rows<T, 1, 1, false, MODE>),
                       grid_of(cdiv(a.n << a.lanes_log, kBlock)), dim3(kBlock),
                       (size_t)(kBlock >> a.lanes_log) * a.kp * kEntryBytes, stream, a);
  } else if (pieces <= kWave * kWaveSteps) {
    while (a.lanes_log < 6 &&
           (kPerLane << a.lanes_log < a.k || 4 << a.lanes_log < pieces ||
            ((1 << a.lanes_log) < pieces && a.n << a.lanes_log < kFillLanes)))
      ++a.lanes_log;
    const int steps = (int)cdiv(pieces, 1 << a.lanes_log);
    const dim3 grid = grid_of(cdiv(a.n << a.lanes_log, kBlock));
    const size_t lds = (size_t)(kBlock >> a.lanes_log) * a.kp * kEntryBytes;
    if (steps <= 1)
      hipLaunchKernelGGL((k_distill_rows<T, V, 1, false, MODE>), grid, dim3(kBlock), lds, stream, a);
    else if (steps == 2)
      hipLaunchKernelGGL((k_distill_rows<T, V, 2, false, MODE>), grid, dim3(kBlock), lds, stream, a);
    else if (steps <= 4)
      hipLaunchKernelGGL((k_distill_rows<T, V, 4, false, MODE>), grid, dim3(kBlock), lds, stream, a);
    else
      hipLaunchKernelGGL((k_distill_rows<T, V, kWaveSteps, false, MODE>), grid, dim3(kBlock), lds,
                         stream, a);
  } else {
    // With fewer rows than CUs a row has a whole CU's lanes, but for short ones (3,000
    // fp32: 8.2 us with 1,024 lanes, 7.1 with 256).
    int threads = a.n < 256 && pieces > 2048 ? 1024 : 256;
    while (threads < 1024 && threads * kMaxSteps < pieces) threads *= 2;
    const int steps = (int)cdiv(pieces, threads);
    const dim3 grid = grid_of(a.n);
    const size_t lds = (size_t)a.kp * kEntryBytes;
    if (steps <= 4)             // 3 at least
      hipLaunchKernelGGL((k_distill_rows<T, V, 4, true, MODE>), grid, dim3(threads), lds, stream, a);
    else if (steps <= 8)
      hipLaunchKernelGGL((k_distill_rows<T, V, 8, true, MODE>), grid, dim3(threads), lds, stream, a);
    else
      hipLaunchKernelGGL((k_distill_rows<T, V, 16, true, MODE>), grid, dim3(threads), lds, stream, a);
  }
  GG_LAUNCH_CHECK("k_distill_rows");
  return GG_OK;
}

int pack_args(const gg_rows_t* z, int64_t n, int64_t vocab, const void* top_ids_d, int32_t id_bits,
              int64_t ids_stride, const gg_rows_t* top, int32_t k, float temperature, float weight,
              const float* row_w_d, const gg_rows_t* dz, int32_t* status_d, DistillArgs* a) {
  GG_REQUIRE(status_d, "status is NULL");
  GG_REQUIRE(n >= 0 && n <= GG_DISTILL_MAX_ROWS, "n = %lld unsupported", (long long)n);
  GG_REQUIRE(vocab >= 1 && vocab <= GG_DISTILL_MAX_VOCAB, "vocab %lld outside 1..%d",
             (long long)vocab, GG_DISTILL_MAX_VOCAB);
  GG_REQUIRE(k >= 1 && k <= GG_DISTILL_MAX_K, "k = %d outside 1..%d", k, GG_DISTILL_MAX_K);
  GG_REQUIRE(temperature >= 1e-30f && temperature <= 1e30f, "temperature outside 1e-30 .. 1e30");
  int rc = pack_rows(z, "z", n, vocab, kBitFloats, false, &a->z);
  if (rc == GG_OK) rc = pack_rows(top, "top", n, k, kBitFloats, false, &a->top);
  if (rc == GG_OK && dz) rc = pack_rows(dz, "dz", n, vocab, 1u << z->dtype, true, &a->dz);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(id_bits == 32 || id_bits == 64, "ids of %d bits", id_bits);
  GG_REQUIRE(n == 0 || top_ids_d, "ids are NULL");
  GG_REQUIRE((uintptr_t)top_ids_d % (id_bits / 8) == 0 && ids_stride % (id_bits / 8) == 0 &&
                 ids_stride >= 0,
             "ids are not aligned");
  GG_REQUIRE((uintptr_t)row_w_d % 4 == 0, "row_w is not aligned");
  a->ids = (const char*)top_ids_d;
  a->ids_stride = ids_stride;
  a->ids64 = id_bits == 64;
  a->k = k;
  a->kp = (k + 3) / 4 * 4;
  a->top_dtype = top->dtype;
  a->n = n;
  a->vocab = (int32_t)vocab;
  a->temp = temperature;
  a->inv_temp = 1.0f / temperature;
  a->c2 = kLog2e / temperature;
  a->t_ln2 = kLn2 * temperature;
  a->weight = weight;
  a->row_w = row_w_d;
  a->status = status_d;
  return GG_OK;
}

}  // namespace
}  // namespace gg

using namespace gg;

extern "C" size_t gg_ws_distill(int64_t n, int64_t vocab) {
  if (n < 0 || n > GG_DISTILL_MAX_ROWS || vocab < 1 || vocab > GG_DISTILL_MAX_VOCAB) return 0;
  return distill_ws_layout(n, nullptr, nullptr);
}

extern "C" int gg_distill_forward(const gg_rows_t* z, int64_t n, int64_t vocab,
                                  const void* top_ids_d, int32_t id_bits, int64_t ids_stride,
                                  const gg_rows_t* top, int32_t k, float temperature, float weight,
                                  const float* row_w_d, float* loss_d, float* lse_d,
                                  const gg_rows_t* dz, int32_t* status_d, void* ws,
                                  size_t ws_bytes, hipStream_t stream) {
  DistillArgs a = {};
  const int rc = pack_args(z, n, vocab, top_ids_d, id_bits, ids_stride, top, k, temperature, weight,
                           row_w_d, dz, status_d, &a);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(n == 0 || loss_d, "loss is NULL");
  GG_REQUIRE((uintptr_t)loss_d % 4 == 0 && (uintptr_t)lse_d % 4 == 0, "loss or lse is not aligned");
  const size_t need = gg_ws_distill(n, vocab);
  GG_REQUIRE(n == 0 || (ws && (uintptr_t)ws % 8 == 0 && ws_bytes >= need),
             "workspace of %zu bytes < %zu, or not aligned", ws_bytes, need);
  if (n == 0) return GG_OK;
  DistillWs w;
  distill_ws_layout(n, (char*)ws, &w);
  a.part = w.part;
  a.lesson = w.lesson;
  a.loss = loss_d;
  a.lse = lse_d;
  GG_FOR_FLOAT(z->dtype, T, {
    return dz ? launch_rows<T, kFused>(a, stream) : launch_rows<T, kLossOnly>(a, stream);
  });
}

extern "C" int gg_distill_backward(const gg_rows_t* z, int64_t n, int64_t vocab,
                                   const void* top_ids_d, int32_t id_bits, int64_t ids_stride,
                                   const gg_rows_t* top, int32_t k, float temperature,
                                   float weight, const float* row_w_d, const float* lse_d,
                                   const gg_rows_t* dz, int32_t* status_d, hipStream_t stream) {
  GG_REQUIRE(dz, "dz: no rows given");
  DistillArgs a = {};
  const int rc = pack_args(z, n, vocab, top_ids_d, id_bits, ids_stride, top, k, temperature, weight,
                           row_w_d, dz, status_d, &a);
  if (rc != GG_OK) return rc;
  GG_REQUIRE(n == 0 || lse_d, "lse is NULL");
  GG_REQUIRE((uintptr_t)lse_d % 4 == 0, "lse is not aligned");
  if (n == 0) return GG_OK;
  a.lse_in = lse_d;
  GG_FOR_FLOAT(z->dtype, T, { return launch_rows<T, kBackward>(a, stream); });
}
