// Attention of new tokens over a paged key/value cache (causal, optional sliding window, query
// heads sharing KV heads), for gfx950.
//
//   o_r = sum_t softmax_t(scale q_r . k_t) v_t,   t <= p_r (and t > p_r - window)
//
// A tile is up to M rows (new token, query head of one KV head's group), token-major, of one
// sequence: the heads that share a KV head share its keys and values.  The scores are computed
// transposed, S^T = K Q^T with v_mfma_f32_32x32x16, so that a lane holds 16 keys of ONE row: the
// row maximum and sum are lane-local but for one exchange between the wave's halves.  Row m of
// the product is fed key pi(m), pi swapping bits 2 and 3, after which a lane's eight
// consecutive accumulators are eight consecutive keys: exactly the B operand of the second
// product O^T = V^T P^T, which therefore takes the probabilities from the registers they
// were computed in, with no pass through shared memory.
//
// The cache is laid out for these operands, 16 tokens at a time: a group's keys as [D/8][16][8] and
// its values as [2][D][8] (per page and head, P/16 groups).  Every operand load is 16 bytes per
// lane at a constant offset within a group, a group's operands are 32 D contiguous bytes, and a
// page's size only decides where its groups lie.
//
// Work is cut into units of (tile, range of keys).  The lengths are on the device only, so each
// block derives the cut from them itself: with W = sum over tiles of the keys they span, a unit
// takes C = max(min_keys, ceil(W * kv_heads / target)) keys, which bounds the number of units by
// target / kv_heads + tiles whatever the lengths are (the grid), and evens out ragged
// batches.  A tile of several units leaves partial (m, l, o) rows in the workspace, and a note of
// itself for a second launch, which joins them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "held.h"
#include "serve.h"

namespace moecache {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

template <class E>
struct Vec {
  typedef E x8 __attribute__((ext_vector_type(8)));
  typedef E x4 __attribute__((ext_vector_type(4)));
};

__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c, __bf16) {
  typedef Vec<__bf16>::x8 x8;
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c, _Float16) {
  typedef Vec<_Float16>::x8 x8;
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(x8, a), __builtin_bit_cast(x8, b), c, 0, 0, 0);
}

constexpr int kLanes = 64;
constexpr int kThreads = 256, kWaves = kThreads / kLanes;
constexpr int kIds = 1024;  // page ids of a unit held in LDS at a time
constexpr float kNegInf = -__builtin_inff();
// A row's exponentials are taken relative to its base, which follows its maximum lazily: log2 of how far
// the maximum may rise before it does, and of how far below the maximum it is then put.  fp16's numbers end at
// 2^16 and lose bits below 2^-14, so there probabilities are kept near the upper end: the largest is 2^10 to
// 2^14 (and the scores' own rounding, below 2^2 for scores up to 2^24), one has all its bits down to 2^-24 of the largest
// and is off by at most 2^-35 of it below that.  (With base and maximum alike, 16000 keys that lie 17.5 below a first
// one were off by 0.2 of their sum; with 8 and 6 sixteen times as far off as with 4 and 10.)  Measured, 4096 fp16 tokens
// behind 12288: 1022 us, with 8 and 6 1007, with 8 and 0 1003; the other cases alike.
template <class E>
constexpr float kSlack = __is_same(E, _Float16) ? 4.f : 8.f;
template <class E>
constexpr float kBelow = __is_same(E, _Float16) ? 10.f : 0.f;

// What a launch covers of the keys: all of them, those behind the tokens that every sequence begins
// with, or these tokens' (behind.h).
enum Cover { kAll, kBehind, kPrefix };

// Of the tokens that every sequence begins with, the keys that the prefix's launch takes: whole 64s.
// -1: a count that is none.
__device__ __forceinline__ int shared_of(const AttendArgs &a) {
  const int n = *a.shared;
  return n < 0 || n > (a.prefix_pages << a.kv.page_shift) ? -1 : n;
}

// One sequence's share of the batch, read defensively: whatever starts and lengths hold, rows
// stay within [0, n_tokens) and keys within the table.
struct Seq {
  int first, count, length;  // rows first .. first + count - 1; keys 0 .. length - 1
  bool bad;                  // a length its table cannot hold, or shorter than its new tokens
};
template <Cover C>
__device__ __forceinline__ Seq seq_of(const AttendArgs &args, int s) {
  const KvView &kv = args.kv;
  const int a = min(max(kv.starts[s], 0), kv.n_tokens), b = min(max(kv.starts[s + 1], a), kv.n_tokens);
  const int len = kv.lengths[s];
  bool bad = len < b - a || len > (kv.max_pages << kv.page_shift);
  if (C == kBehind && !bad && b > a) {  // what is shared comes before every new token
    const int n = shared_of(args);
    bad = n < 0 || n > len - (b - a);
  }
  return Seq{a, b - a, bad ? 0 : len, bad};
}
// The first key that the launch covers.
template <Cover C>
__device__ __forceinline__ int skip_of(const AttendArgs &a) {
  return C == kBehind ? max(0, shared_of(a)) & ~63 : 0;
}

// Tiles of a sequence, and the keys that one of them can span (its window starts at a multiple of
// 64 at or below the first row's).
template <int M>
__device__ __forceinline__ int tiles_of(const AttendArgs &a, const Seq &q) {
  return (int)((uint32_t)(q.count * a.kv.group + M - 1) / M);  // at most 2^27 rows
}
template <int M, Cover C>
__device__ __forceinline__ int span_of(const AttendArgs &a, const Seq &q) {
  if (C == kBehind) return max(0, q.length - skip_of<C>(a));  // no window there
  if (!a.window) return q.length;
  return (int)min((uint32_t)q.length, (uint32_t)a.window + (M + 64));  // of at most M tokens
}
// Units of a tile that spans `span` keys, which it shares out evenly: span / C rounded down, or with few
// rows and tiles for a quarter of the card's places and more, to the nearest whole number, which leaves
// the units' sizes closer to each other at the price of some more of them.  Measured (nearest, down): 64 sequences of
// one token over 200 to 16000 204 and 208 us, 16 with heads of 256 65.8 and 72.9, but 24 windows of 5 68.7 and 67.1; with
// fewer tiles the two are alike; in tiles of 128 rows 33 tokens over 60000 88.6 and 66.6, 1500 behind 1000 with heads
// of 256 116 and 102.
__device__ __forceinline__ int units_of(const AttendArgs &a, int span, int C) {
  return max(1, (int)((uint32_t)(span + (a.nearest ? C / 2 : 0)) / (uint32_t)C));  // both at most 2^30
}
__device__ __forceinline__ int share_of(int keys, int units) {
  return (int)(((uint32_t)(keys + units - 1) / (uint32_t)units + 63) & ~63u);
}

// The workspace: how many tiles were split, with a plan_kernel the keys of a unit, a note of each split
// tile, then the plan, then the o rows of slot (slot, kvh), then (m, l) pairs of all slots.
struct SplitTile {
  int32_t slot, units;        // its first partial result, and their number
  int32_t first, row0, rows;  // its sequence's first token row, the tile's first row in the sequence, its rows
  int32_t pad[3];
};
struct SplitTiles {
  int32_t count, keys, pad[6];
  SplitTile tile[];
};
constexpr int kPlanSeqs = kLanes;  // sequences up to which every block plans for itself
__host__ __device__ inline int64_t plan_ints(const AttendArgs &a) {  // a multiple of 16 bytes
  return a.kv.n_seqs > kPlanSeqs ? (3 * ((int64_t)a.kv.n_seqs + 1) + 3) & ~(int64_t)3 : 0;
}
__device__ __forceinline__ SplitTiles *split_tiles(const AttendArgs &a) { return (SplitTiles *)a.work; }
// units, slots and split tiles before every sequence, and in all
__device__ __forceinline__ int32_t *plan_of(const AttendArgs &a, int which) {
  return (int32_t *)((uint8_t *)a.work + sizeof(SplitTiles) + a.max_tiles * sizeof(SplitTile)) +
         which * (int64_t)(a.kv.n_seqs + 1);
}
__device__ __forceinline__ float *part_base(const AttendArgs &a) { return (float *)(plan_of(a, 0) + plan_ints(a)); }

// Keys of a unit, for tiles that span `work` keys together.
__device__ __forceinline__ int keys_of(const AttendArgs &a, int64_t work) {
  const int64_t c = (work * a.kv.kv_heads + (1 << a.target_log2) - 1) >> a.target_log2;
  return (int)min((int64_t)1 << 30, max((int64_t)a.min_keys, (c + 63) & ~(int64_t)63));
}

// What a sequence adds to the plan: units, slots (units of split tiles), split tiles.  No batch has
// 2^24 units: only starts out of order could add up to more, and then sums stay below 2^31.
struct Share {
  int units, slots, tiles;
};
template <int M, Cover V>
__device__ __forceinline__ Share share_of_seq(const AttendArgs &a, const Seq &q, int C) {
  const int per = units_of(a, span_of<M, V>(a, q), C);
  const int n = (int)min((int64_t)1 << 24, (int64_t)tiles_of<M>(a, q) * per);
  return per > 1 || V == kBehind ? Share{n, n, n / per} : Share{n, 0, 0};
}
// Sums over the lanes up to each one, by the vector unit's own exchanges (through LDS 64 sequences of 50 to
// 1500 keys took 29.0 us, now 26.8).
__device__ __forceinline__ int running(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // from 1, 2, 4, 8 lanes below, within 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // the first and third 16's to the next
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // the first 32's to the others
  return x;
}
__device__ __forceinline__ Share scan(Share s) { return Share{running(s.units), running(s.slots), running(s.tiles)}; }
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
// The sum over all lanes of numbers below 2^58.
__device__ __forceinline__ int64_t total(int64_t x) {
  const int part[3] = {(int)(x & 0xffffff), (int)(x >> 24 & 0xffffff), (int)(x >> 48)};
  int64_t sum = 0;
#pragma unroll
  for (int i = 0; i < 3; ++i) sum += (int64_t)lane_value(running(part[i]), kLanes - 1) << (24 * i);
  return sum;
}

// Where a unit stands: its sequence and its number among the sequence's units; the split tiles and
// the units of split tiles in the sequences before.
struct Place {
  int seq, index, tiles, slots;
  Seq q;
};

// Up to kPlanSeqs sequences: every wave plans for itself, a sequence to a lane, which saves a launch
// (64 sequences of 3000 keys: 70 us, with plan_kernel 76; one sequence: 14 and 18).  In rounds over more
// sequences it would cost every block: 1024 of 400 keys took 277 us, with plan_kernel 145; 4096 of
// 200 took 2325, now 371.
template <int M, Cover V>
__device__ __forceinline__ bool plan_here(const AttendArgs &a, int unit, bool last, int *C, Place *out) {
  const int lane = threadIdx.x % kLanes, lanes = min(kLanes, a.kv.n_seqs);
  const Seq q = lane < lanes ? seq_of<V>(a, lane) : Seq{0, 0, 0, false};
  const int64_t work = (int64_t)tiles_of<M>(a, q) * span_of<M, V>(a, q);
  *C = keys_of(a, total(work));  // lanes past the sequences add nothing
  const Share own = share_of_seq<M, V>(a, q, *C), sum = scan(own);
  if (last) split_tiles(a)->count = min(a.max_tiles, lane_value(sum.tiles, kLanes - 1));
  const uint64_t any = __ballot(lane < lanes && unit < sum.units);
  if (!any) return false;
  const int at = __ffsll((unsigned long long)any) - 1;
  out->seq = at;
  out->index = unit - lane_value(sum.units - own.units, at);
  out->slots = lane_value(sum.slots - own.slots, at);
  out->tiles = lane_value(sum.tiles - own.tiles, at);
  out->q = Seq{lane_value(q.first, at), lane_value(q.count, at), lane_value(q.length, at), (bool)lane_value(q.bad, at)};
  return true;
}

// More sequences: one block plans for all, and a unit's sequence is searched for, 64 at a time.
constexpr int kPlanThreads = 1024;
template <int M, Cover V>
__device__ __forceinline__ void plan_body(const AttendArgs &a) {
  constexpr int kW = kPlanThreads / kLanes;
  __shared__ int64_t works[kW];
  __shared__ Share sums[kW];
  const int lane = threadIdx.x % kLanes, wave = threadIdx.x / kLanes, n = a.kv.n_seqs;
  int64_t work = 0;
  for (int s = threadIdx.x; s < n; s += kPlanThreads) {
    const Seq q = seq_of<V>(a, s);
    work += (int64_t)tiles_of<M>(a, q) * span_of<M, V>(a, q);
  }
  work = total(work);
  if (lane == 0) works[wave] = work;
  __syncthreads();
  work = 0;
  for (int i = 0; i < kW; ++i) work += works[i];
  const int C = keys_of(a, work);
  int32_t *units = plan_of(a, 0), *slots = plan_of(a, 1), *tiles = plan_of(a, 2);
  constexpr int64_t kMost = 1 << 30;
  int64_t nu = 0, ns = 0, nt = 0;
  for (int s0 = 0; s0 < n; s0 += kPlanThreads) {
    const int s = s0 + threadIdx.x;
    const Share own = s < n ? share_of_seq<M, V>(a, seq_of<V>(a, s), C) : Share{0, 0, 0}, sum = scan(own);
    __syncthreads();
    if (lane == kLanes - 1) sums[wave] = sum;
    __syncthreads();
    int64_t u = nu + sum.units - own.units, v = ns + sum.slots - own.slots, w = nt + sum.tiles - own.tiles;
    for (int i = 0; i < kW; ++i) {
      if (i < wave) u += sums[i].units, v += sums[i].slots, w += sums[i].tiles;
      nu += sums[i].units, ns += sums[i].slots, nt += sums[i].tiles;
    }
    if (s < n) units[s] = (int)min(u, kMost), slots[s] = (int)min(v, kMost), tiles[s] = (int)min(w, kMost);
  }
  if (threadIdx.x == 0) {
    units[n] = (int)min(nu, kMost);
    split_tiles(a)->count = (int)min((int64_t)a.max_tiles, nt);
    split_tiles(a)->keys = C;
  }
}
template <int M>
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttendArgs a) {
  plan_body<M, kAll>(a);
}
template <int M, Cover V>
__device__ __forceinline__ bool plan_search(const AttendArgs &a, int unit, int *C, Place *out) {
  const int32_t *units = plan_of(a, 0);
  *C = split_tiles(a)->keys;
  if (unit >= units[a.kv.n_seqs]) return false;
  const int lane = threadIdx.x % kLanes;
  int lo = 0, hi = a.kv.n_seqs;  // the last sequence that begins at or before the unit
  while (hi - lo > 1) {
    const int step = (hi - lo + kLanes - 1) / kLanes, at = lo + lane * step;
    const uint64_t in = __ballot(at < hi && units[at] <= unit);
    const int k = in ? kLanes - 1 - __clzll((long long)in) : 0;
    lo += k * step;
    hi = min(hi, lo + step);
  }
  *out = Place{lo, unit - units[lo], plan_of(a, 2)[lo], plan_of(a, 1)[lo], seq_of<V>(a, lo)};
  return true;
}

// Keys lo .. hi - 1 that rows of a tile see, lo rounded down to a multiple of 64; the tile's units
// cut this range from lo on.
struct Range {
  int lo, hi;
};
template <int M, Cover V>
__device__ __forceinline__ Range range_of(const AttendArgs &a, const Seq &q, int tile) {
  const int rows = q.count * a.kv.group;
  const int t0 = tile * M / a.kv.group, t1 = min(tile * M + M, rows) - 1;
  const int before = q.length - q.count;
  Range r;
  r.hi = before + t1 / a.kv.group + 1;
  r.lo = V == kBehind ? skip_of<V>(a) : a.window ? max(0, before + t0 - a.window + 1) & ~63 : 0;
  return r;
}

// The rows' state in one wave: 32 rows, lane n and lane n + 32 hold row n.
template <int D>
struct Rows {
  f32x16 acc[D / 32];  // o^T: d = 32 i + 8 (r / 4) + 4 half + r % 4
  float m, l;          // base of the exponentials (log2 units, both halves alike), this lane's share of the sum
};

// Key (within its 32) of accumulator r of a score product, for this lane's half.
__device__ __forceinline__ int key_of(int r, int half) { return 16 * (r / 8) + 8 * half + r % 8; }

// Scores of keys that their row does not see become -inf: floor < t <= pos, as one comparison.
template <int N>
__device__ __forceinline__ void mask_scores(f32x16 (&s)[N], int t0, int pos, int floor) {
  // unsigned from the start: a window near 2^31 puts keys behind pos 2^31 and more past the floor
  const uint32_t first = (uint32_t)t0 + 8 * (threadIdx.x % kLanes / 32) - (uint32_t)floor - 1, seen = pos - floor;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      if (first + (32 * n + key_of(r, 0)) >= seen) s[n][r] = kNegInf;
}

// Scores to probabilities over 32 * N keys: takes the new maximum, rescales the rows where some
// row's maximum rose, and packs the B operands of the second product.
// Probabilities are rounded to the cache's type, the type the matrix cores multiply; the sum
// is taken in fp32 before that.  times(i), if given: powers of two that the probabilities of the i-th eight of this
// lane's keys are multiplied by for the product.  That rounds as without them down to p 2^e = 2^-126; what is less is
// off by up to 2^-134, so that a row is by up to 2^-134 |c| <= 2^-125 for each such key (the largest p is at least 1).
struct alignas(16) Eight {
  float v[8];
};
struct AsIs {};
template <class E, int D, int N, class T = AsIs>
__device__ __forceinline__ void softmax_step(f32x16 (&s)[N], Rows<D> &st, u32x4 (&p)[2 * N], float scale, T times = T()) {
  constexpr bool kTimes = !__is_same(T, AsIs);
  float mx = s[0][0];
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[n][r]);
  const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  mx = fmaxf(__uint_as_float(halves[0]), __uint_as_float(halves[1]));
  mx = mx * scale - kBelow<E>;  // where the base would be now
  if (__any(mx > st.m + kSlack<E>)) {
    const float top = fmaxf(st.m, mx), shrink = __builtin_amdgcn_exp2f(st.m - (top == kNegInf ? 0.f : top));
    st.l *= shrink;
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.acc[i][r] *= shrink;
    st.m = top;
  }
  const float base = st.m == kNegInf ? 0.f : st.m;
  typedef typename Vec<E>::x8 x8;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      x8 e;
      Eight f;
      if constexpr (kTimes) f = times(2 * n + c);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = __builtin_amdgcn_exp2f(fmaf(s[n][8 * c + j], scale, -base));
        st.l += v;
        if constexpr (kTimes)
          e[j] = (E)(v * f.v[j]);
        else
          e[j] = (E)v;
      }
      p[2 * n + c] = __builtin_bit_cast(u32x4, e);
    }
}

// v with the elements that are not among the first n (of its 8) cleared
__device__ __forceinline__ u32x4 keep_first(u32x4 v, int n) {
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] &= n >= 2 * i + 2 ? 0xffffffffu : n == 2 * i + 1 ? 0xffffu : 0u;
  return v;
}

// Of a step some of whose keys some rows do not see, the values of 16 keys from t0 on.  Keys at or past
// `end` hold whatever the page held: their values are cleared.  A value that is not finite must not
// reach rows that do not see its key (0 * inf is a NaN): it is cleared too, and reported, for
// add_odd to give it to the rows that do see it.
template <class E, int D>
__device__ __forceinline__ bool clean_values(u32x4 (&v)[D / 32], int t0, int end) {
  constexpr uint32_t lo = __is_same(E, __bf16) ? 0x7f80u : 0x7c00u, hi = lo << 16;
  if (t0 + 16 > end) {
    const int n = min(8, max(0, end - (t0 + 8 * (int)(threadIdx.x % kLanes / 32))));
#pragma unroll
    for (int i = 0; i < D / 32; ++i) v[i] = keep_first(v[i], n);
  }
  // an exponent of ones carries into the sign's place when one is added to it
  uint32_t odd = 0;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) odd |= (v[i][j] & 0x7fff7fffu) + (0x80008000u - (lo | hi));
  if (!__any(odd & 0x80008000u)) return false;
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[i][j] &= ((v[i][j] & lo) == lo ? 0u : 0xffffu) | ((v[i][j] & hi) == hi ? 0u : 0xffff0000u);
  return true;
}

// Element d of a head that row m of product i stands for: 32 i + m, or where an operand load brings
// two neighbouring elements (8 bits straight from memory), these are the products 2 i and 2 i + 1.
template <bool Pairs>
__device__ __forceinline__ constexpr int d_of(int i, int m) {
  return Pairs ? 64 * (i / 2) + 2 * m + i % 2 : 32 * i + m;
}
// Four consecutive elements of this lane's row, the g-th of product i's, and the first one's place.
template <int D, bool Pairs>
__device__ __forceinline__ f32x4 four_of(const Rows<D> &st, int i, int g) {
  if (!Pairs) return f32x4{st.acc[i][4 * g], st.acc[i][4 * g + 1], st.acc[i][4 * g + 2], st.acc[i][4 * g + 3]};
  const int a = i & ~1, b = i | 1, r = 4 * g + 2 * (i % 2);
  return f32x4{st.acc[a][r], st.acc[b][r], st.acc[a][r + 1], st.acc[b][r + 1]};
}
template <bool Pairs>
__device__ __forceinline__ constexpr int four_at(int i, int g, int half) {
  return Pairs ? 64 * (i / 2) + 16 * g + 8 * half + 4 * (i % 2) : 32 * i + 8 * g + 4 * half;
}

// Adds the values of keys t0 .. t1 - 1 that are not finite to the rows that see them (their weight
// there is positive: an infinity stays the infinity it was).  Rare, and slow: element by element.
template <class E, int D, class S, bool Pairs>
__device__ __forceinline__ void add_odd(Rows<D> &st, const S *values, const uint8_t *scales, int heads, const int *ids,
                                        int pg0, int shift, int64_t page_elems, int t0, int t1, int pos, int floor) {
  constexpr uint32_t exponent = __is_same(E, __bf16) ? 0x7f80u : 0x7c00u;
  const int half = threadIdx.x % kLanes / 32;
#pragma unroll 1
  for (int t = t0; t < t1; ++t) {
    const int64_t id = ids[(t >> shift) - pg0];
    const S *src = values + id * page_elems + ((t & ((1 << shift) - 1)) >> 3) * 8 * D + (t & 7);
    const bool sees = t <= pos && t > floor;
    float scale = 1.f;
    if constexpr (sizeof(S) == 1) scale = scale_of(scales[(id * heads << shift) + (t & ((1 << shift) - 1))]);
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const S c = src[d_of<Pairs>(i, 8 * (r / 4) + 4 * half + r % 4) * 8];
        uint16_t e;
        if constexpr (sizeof(S) == 1)
          e = (uint16_t)decode2(c, false, scale, scale, E());
        else
          e = c;
        st.acc[i][r] += sees && (e & exponent) == exponent ? (float)__builtin_bit_cast(E, e) : 0.f;
      }
      __builtin_amdgcn_sched_barrier(0);  // 16 values' registers at a time
    }
  }
}

// This lane's row of the tile as the B operand of S^T = K Q^T: q[c] = elements 16 c + 8 half ..., or for
// keys of 8 bits straight from memory, 16 elements to a load, 32 (c / 2) + 16 half + 8 (c % 2) ...
template <int D, bool Pairs>
__device__ __forceinline__ void load_q(const AttendArgs &a, const Seq &q, int kvh, int row, u32x4 (&out)[D / 16]) {
  const int half = threadIdx.x % kLanes / 32, rows = q.count * a.kv.group;
  if (row < rows) {
    const int tok = q.first + row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
    const uint16_t *src = (const uint16_t *)a.q + (int64_t)tok * a.q_stride + (int64_t)head * D;
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
      out[c] = *(const u32x4 *)(src + (Pairs ? c / 2 * 32 + 16 * half + c % 2 * 8 : 16 * c + 8 * half));
  } else {
#pragma unroll
    for (int c = 0; c < D / 16; ++c) out[c] = u32x4{};
  }
}

// Writes four consecutive elements of a finished row.
template <class E, int D>
__device__ __forceinline__ void store_out(const AttendArgs &a, const Seq &q, int kvh, int row, int d, f32x4 v) {
  const int tok = q.first + row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
  typename Vec<E>::x4 e;
#pragma unroll
  for (int i = 0; i < 4; ++i) e[i] = (E)v[i];
  *(typename Vec<E>::x4 *)((E *)a.out + (int64_t)tok * a.out_stride + (int64_t)head * D + d) = e;
}

template <int D, int M>
__device__ __forceinline__ float *part_o(const AttendArgs &a, int64_t slot, int kvh, int row) {
  return part_base(a) + ((slot * a.kv.kv_heads + kvh) * M + row) * D;
}
template <int D, int M>
__device__ __forceinline__ float *part_ml(const AttendArgs &a, int64_t slot, int kvh, int row) {
  return part_base(a) + (int64_t)a.max_slots * a.kv.kv_heads * M * D + ((slot * a.kv.kv_heads + kvh) * M + row) * 2;
}

// The prefix's partial results: the o rows of its slots, then their (m, l) pairs.
__device__ __forceinline__ int64_t front_row(const AttendArgs &a, int64_t slot, int kvh, int row) {
  return (slot * a.kv.kv_heads + kvh) * a.prefix_rows + row;
}
template <int D>
__device__ __forceinline__ float *front_o(const AttendArgs &a, int64_t row) {
  return a.front + row * D;
}
template <int D>
__device__ __forceinline__ float *front_ml(const AttendArgs &a, int64_t row) {
  return a.front + front_row(a, (int64_t)a.prefix_tiles * a.prefix_splits, 0, 0) * D + row * 2;
}
// Where a unit's row goes that is not the whole of it.
template <int D, int M, Cover V>
__device__ __forceinline__ float *unit_o(const AttendArgs &a, int64_t slot, int kvh, int row) {
  return V == kPrefix ? front_o<D>(a, front_row(a, slot, kvh, row)) : part_o<D, M>(a, slot, kvh, row);
}
template <int D, int M, Cover V>
__device__ __forceinline__ float *unit_ml(const AttendArgs &a, int64_t slot, int kvh, int row) {
  return V == kPrefix ? front_ml<D>(a, front_row(a, slot, kvh, row)) : part_ml<D, M>(a, slot, kvh, row);
}

// The ids of the unit's pages pg0 .. , at most kIds of them, into LDS; an id outside the pool is
// taken as page 0, and reported if its page is at or past `seen`, the first one that a row of the tile
// sees (a range that begins at a multiple of 64 holds up to three pages of 16 before it, whose entries may
// be anything).  Ends with a barrier.
__device__ __forceinline__ void load_ids(const KvView &kv, const int32_t *pages, int pg0, int pg_last, int seen, int *ids,
                                         int *bad) {
  const int n = min(kIds, pg_last - pg0 + 1);
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const int id = pages[pg0 + i];
    const bool ok = (unsigned)id < (unsigned)kv.n_pages;
    ids[i] = ok ? id : 0;
    if (!ok && pg0 + i >= seen) {
      *bad = 1;
      if (kv.status) atomicOr(kv.status, kKvBadPage);
    }
  }
  __syncthreads();
}
// The first page that a row of a tile whose first row stands at `pos` sees.
__device__ __forceinline__ int first_page(const AttendArgs &a, int pos) {
  return a.window ? max(0, pos - a.window + 1) >> a.kv.page_shift : 0;
}

// What a block works on.
struct Unit {
  int seq, kvh, tile, k0, k1;  // keys k0 .. k1 - 1, k0 a multiple of 64
  int64_t slot;                // partial-result slot, -1: the tile is this unit's alone
  Seq q;
};
// Of what all sequences begin with: the batch's rows, from its first sequence's to its last one's, as those of
// one sequence, cut into tiles and these tiles' keys into prefix_splits units alike.
struct Prefix {
  int first, rows;   // the first token's row; rows of a KV head
  int share, units;  // a unit's keys; units that have any
  int keys;
};
__device__ __forceinline__ Prefix prefix_of(const AttendArgs &a) {
  Prefix p;
  p.first = min(max(a.kv.starts[0], 0), a.kv.n_tokens);
  p.rows = (min(max(a.kv.starts[a.kv.n_seqs], p.first), a.kv.n_tokens) - p.first) * a.kv.group;
  p.keys = skip_of<kBehind>(a);
  p.share = share_of(p.keys, a.prefix_splits);
  p.units = p.keys ? (p.keys + p.share - 1) / p.share : 0;
  return p;
}
template <int M>
__device__ __forceinline__ bool prefix_unit(const AttendArgs &a, int block, Unit *u) {
  const Prefix p = prefix_of(a);
  const int unit = block / a.kv.kv_heads, split = unit % a.prefix_splits;
  u->kvh = block % a.kv.kv_heads;
  u->tile = unit / a.prefix_splits;
  u->seq = 0;
  u->q = Seq{p.first, p.rows / a.kv.group, p.keys, false};
  u->k0 = split * p.share;
  u->k1 = min(p.keys, u->k0 + p.share);
  u->slot = unit;
  return split < p.units && u->tile * M < p.rows;
}

template <int M, Cover V>
__device__ __forceinline__ bool unit_of(const AttendArgs &a, int block, Unit *u) {
  if constexpr (V == kPrefix) return prefix_unit<M>(a, block, u);
  Place pl;
  int C;
  u->kvh = block % a.kv.kv_heads;
  const int unit = block / a.kv.kv_heads;
  const bool found = a.kv.n_seqs > kPlanSeqs
                         ? plan_search<M, V>(a, unit, &C, &pl)
                         : plan_here<M, V>(a, unit, block == 0 && threadIdx.x < kLanes, &C, &pl);
  if (!found) return false;
  const int per = units_of(a, span_of<M, V>(a, pl.q), C);
  if (pl.index >= (int64_t)tiles_of<M>(a, pl.q) * per) return false;  // starts out of order
  // the tiles with the most keys first
  const int order = pl.index / per, split = pl.index % per;
  u->seq = pl.seq;
  u->q = pl.q;
  u->tile = tiles_of<M>(a, pl.q) - 1 - order;
  const Range r = range_of<M, V>(a, pl.q, u->tile);
  const int share = share_of(r.hi - r.lo, per);
  const int real = max(1, (r.hi - r.lo + share - 1) / max(1, share));  // the tile's units that have keys
  u->k0 = r.lo + split * share;
  u->k1 = min(r.hi, u->k0 + share);
  u->slot = real > 1 || V == kBehind ? pl.slots + pl.index : -1;
  if (per > 1 || V == kBehind) {
    // starts out of order can ask for more than there are
    if ((int64_t)pl.slots + (int64_t)(order + 1) * per > a.max_slots || pl.tiles + order >= a.max_tiles) return false;
    if (split == 0 && u->kvh == 0 && threadIdx.x == 0)
      split_tiles(a)->tile[pl.tiles + order] =
          SplitTile{(int)(pl.slots + pl.index), pl.q.bad ? 0 : real, pl.q.first, u->tile * M,
                    min(M, pl.q.count * a.kv.group - u->tile * M), {0, 0, 0}};
  }
  return split < real;
}

// Rows of a sequence that cannot be served become NaN.
template <class E, int D, int M>
__device__ __forceinline__ void refuse(const AttendArgs &a, const Unit &u) {
  const int rows = min(M, u.q.count * a.kv.group - u.tile * M);
  const float nan = __builtin_nanf("");
  for (int i = threadIdx.x; i < rows * (D / 4); i += kThreads)
    store_out<E, D>(a, u.q, u.kvh, u.tile * M + i / (D / 4), i % (D / 4) * 4, f32x4{nan, nan, nan, nan});
  if (threadIdx.x == 0 && a.kv.status) atomicOr(a.kv.status, kKvBadLength);
}

__device__ __forceinline__ float finish(float l) { return l == 0.f ? 0.f : 1.f / l; }

// ---------------------------------------------------------------------------------------------
// Few rows per sequence: decode and verification windows.  Bound by the bytes of the cache.  A
// block's waves take 32 rows each: of a tile of 32 all four the same ones, in turns at the unit's
// steps of 32 keys, of a tile of 64 two and two (the second pair finds the step's keys in the CU's
// cache).  Keys go straight from memory into the operand registers (LDS would only add a copy); a
// step's are requested while the step before is multiplied.  Two blocks to a CU (232 registers of
// 256 with heads of 128), 64 KB of requests in flight.  Measured, 4 KV heads of 128: 64 sequences of 200
// to 16000 keys, 1.10 GB, 203 us = 5.4 TB/s; 24 windows of 40 rows over 1000 to 9000 keys, 219 MB, 50 us where the
// last-level cache holds them, the whole call 69 on keys that it does not (and 7 of the join).  Heads of 256, whole calls: 64
// sequences of 8000 keys, 2.10 GB, 360 us = 5.8 TB/s; 24 windows of 40 rows, 494 MB, 132 us.
//
// Of a cache of 8 bits (held.h) a load of 16 bytes brings a lane two products' operands, keys' in the order that load_q
// takes the queries in, values' as two neighbouring elements (d_of); a step's bytes are half, so two steps' are under way, and
// the queries stay in LDS.  The conversions are 64 of about 260 vector instructions a step.  64 sequences of 200 to 16000
// keys, 577 MB, 113 us = 5.1 TB/s.
// ---------------------------------------------------------------------------------------------
// An operand of eight numbers of 8 bits (two words) times a power of two.
template <class E>
__device__ __forceinline__ u32x4 operand(uint32_t lo, uint32_t hi, float scale) {
  return u32x4{decode(lo, false, scale, E()), decode(lo, true, scale, E()), decode(hi, false, scale, E()),
               decode(hi, true, scale, E())};
}
// An operand of eight tokens' values times their powers of two.
__device__ __forceinline__ u32x4 times_pairs(u32x4 v, const Eight &s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f16x2 t = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_pkrtz(s.v[2 * i], s.v[2 * i + 1]));
    const uint32_t pair = v[i];  // (a cast of the vector's element would be one of its first)
    v[i] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, pair) * t);
  }
  return v;
}
// The scales of eight tokens' values, for this lane's half of 16.
__device__ __forceinline__ Eight scales_of(uint2 bytes) {
  Eight s;
#pragma unroll
  for (int j = 0; j < 8; ++j) s.v[j] = scale_of((j < 4 ? bytes.x : bytes.y) >> (8 * (j % 4)) & 255);
  return s;
}

// Keys and values of one step of 32 keys as they lie in memory, and their scales.
template <int D, bool Held>
struct Step {
  u32x4 k[Held ? D / 32 : D / 16], v[2][Held ? D / 64 : D / 32];
  uint32_t ks;
  uint2 vs[2];
};

template <int D>
struct FewLds {
  float sums[kWaves][D / 32 * 4][kLanes][4];
  float stat[kWaves][32][2];
  int ids[kIds];
  int bad;
};
template <class E, int D, int R, bool Held, Cover V>
__device__ __forceinline__ void few_body(const AttendArgs &a, FewLds<D> &lds, int block) {
  constexpr int M = 32 * R, kTurns = kWaves / R;  // waves that take turns at the steps of the same rows
  constexpr int kAhead = Held && D <= 128 ? 2 : 1;
  typedef typename std::conditional<Held, uint8_t, uint16_t>::type S;
  auto &sums = lds.sums;
  auto &stat = lds.stat;
  auto &ids = lds.ids;
  int &bad = lds.bad;
  Unit u;
  if (!unit_of<M, V>(a, block, &u)) return;
  if (u.q.bad) {
    refuse<E, D, M>(a, u);
    return;
  }
  const KvView &kv = a.kv;
  const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int half = lane / 32, n = lane % 32;
  if (threadIdx.x == 0) bad = 0;
  const int part = wave % R, turn = wave / R;
  const int rows = u.q.count * kv.group, before = u.q.length - u.q.count;
  const int trow = 32 * part + n, row = u.tile * M + trow;
  const int pos = row < rows ? before + row / kv.group : -1;
  const int window = V == kAll ? a.window : 0, floor = window ? pos - window : -1;
  const int first = before + u.tile * M / kv.group, last = before + (min(u.tile * M + M, rows) - 1) / kv.group;
  u32x4 q[D / 16];
  load_q<D, Held>(a, u.q, u.kvh, row, q);
  // heads of 256, or two steps' requests: the queries stay in LDS, where the joining of the waves has its place later
  constexpr bool kQInLds = D > 128 || (D == 128 && kAhead == 2);
  u32x4 *q_lds = (u32x4 *)&sums[0][0][0][0] + part * (D / 16) * kLanes;
  if (kQInLds && turn == 0)
#pragma unroll
    for (int c = 0; c < D / 16; ++c) q_lds[c * kLanes + lane] = q[c];

  Rows<D> st;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) st.acc[i] = f32x16{};
  st.m = kNegInf;
  st.l = 0.f;

  const int shift = kv.page_shift, P = 1 << shift;
  const int key = (lane & 19) | (lane & 4) << 1 | (lane & 8) >> 1;  // pi(lane): bits 2 and 3 swapped
  const int64_t head_elems = (int64_t)D << shift, page_elems = head_elems * kv.kv_heads;
  const S *keys = (const S *)kv.keys + u.kvh * head_elems, *values = (const S *)kv.values + u.kvh * head_elems;
  const uint8_t *ks = kv.key_scales + (u.kvh << shift), *vs = kv.value_scales + (u.kvh << shift);
  const int pg_last = (u.k1 - 1) >> shift, pg_seen = V == kPrefix ? 0 : first_page(a, first);
  const int32_t *pages = V == kPrefix ? a.prefix : kv.pages + (int64_t)u.seq * kv.max_pages;

  for (int pg0 = u.k0 >> shift; pg0 <= pg_last; pg0 += kIds) {
    __syncthreads();  // the ids of the round before have been read
    load_ids(kv, pages, pg0, pg_last, pg_seen, ids, &bad);
    const int begin = max(u.k0, pg0 << shift);
    const int end = (int)min((int64_t)u.k1, ((int64_t)pg0 + kIds) << shift);
    const int id_last = min(pg_last, pg0 + kIds - 1) - pg0;
    typedef Step<D, Held> Loads;
    auto load_k = [&](Loads &x, int t0) {
      const int t = t0 + key;
      const int id = ids[min((t >> shift) - pg0, id_last)];
      if constexpr (Held) {
        const S *src = keys + id * page_elems + (t & (P - 1) & ~15) * D + (16 * half + t % 16) * 16;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) x.k[c] = *(const u32x4 *)(src + c * 512);
        x.ks = ks[((int64_t)id * kv.kv_heads << shift) + (t & (P - 1))];
      } else {
        const S *src = keys + id * page_elems + (t & (P - 1) & ~15) * D + (16 * half + t % 16) * 8;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) x.k[c] = *(const u32x4 *)(src + 2 * c * 16 * 8);
      }
    };
    auto load_v = [&](Loads &x, int t0) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int t = t0 + 16 * c;
        const int id = ids[min((t >> shift) - pg0, id_last)];
        if constexpr (Held) {
          const S *src = values + id * page_elems + (t & (P - 1)) * D + (half * D + 2 * n) * 8;
#pragma unroll
          for (int i = 0; i < D / 64; ++i) x.v[c][i] = *(const u32x4 *)(src + 64 * i * 8);
          x.vs[c] = *(const uint2 *)(vs + ((int64_t)id * kv.kv_heads << shift) + (t & (P - 1)) + 8 * half);
        } else {
          const S *src = values + id * page_elems + (t & (P - 1)) * D + (half * D + n) * 8;
#pragma unroll
          for (int i = 0; i < D / 32; ++i) x.v[c][i] = *(const u32x4 *)(src + 32 * i * 8);
        }
      }
    };
    // requests for the wave's next kAhead steps are under way
    auto step = [&](Loads &x, int t0) {
      const int next = t0 + 32 * kTurns * kAhead;
      f32x16 s[1] = {};
      const float k_scale = Held ? scale_of(x.ks) : 1.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) {
        const u32x4 k = Held ? operand<E>(x.k[c / 2][c % 2 * 2], x.k[c / 2][c % 2 * 2 + 1], k_scale) : x.k[Held ? c / 2 : c];
        s[0] = mma(k, kQInLds ? q_lds[c * kLanes + lane] : q[c], s[0], E());
      }
      if (next < end) load_k(x, next);
      // whether some row does not see some key of the step
      const bool edge = V != kPrefix && (t0 + 31 > first || (window && t0 <= last - window));
      u32x4 p[2];
      if (edge) mask_scores<1>(s, t0, pos, floor);
      constexpr bool kFold = Held && __is_same(E, __bf16);  // else the values are multiplied
      auto times = [&](int c) { return scales_of(x.vs[c]); };
      if constexpr (kFold)
        softmax_step<E, D, 1>(s, st, p, a.scale_log2, times);
      else
        softmax_step<E, D, 1>(s, st, p, a.scale_log2);
      bool odd = false;
      if constexpr (Held) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          u32x4 v[D / 32];
#pragma unroll
          for (int i = 0; i < D / 32; ++i) {
            v[i] = operand<E>(x.v[c][i / 2][i % 2 * 2], x.v[c][i / 2][i % 2 * 2 + 1], 1.f);
            if constexpr (!kFold) v[i] = times_pairs(v[i], times(c));
          }
          if (edge) odd |= clean_values<E, D>(v, t0 + 16 * c, u.q.length);
#pragma unroll
          for (int i = 0; i < D / 32; ++i) st.acc[i] = mma(v[i], p[c], st.acc[i], E());
        }
      } else {
        if (edge) {
#pragma unroll
          for (int c = 0; c < 2; ++c) odd |= clean_values<E, D>(x.v[c], t0 + 16 * c, u.q.length);
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int i = 0; i < D / 32; ++i) st.acc[i] = mma(x.v[c][i], p[c], st.acc[i], E());
      }
      if (odd)
        add_odd<E, D, S, Held>(st, values, vs, kv.kv_heads, ids, pg0, shift, page_elems, t0, min(t0 + 32, end), pos, floor);
      if (next < end) load_v(x, next);
    };
    int t0 = begin + 32 * turn;
    if constexpr (kAhead == 1) {
      Loads x;
      if (t0 < end) load_k(x, t0), load_v(x, t0);
      for (; t0 < end; t0 += 32 * kTurns) step(x, t0);
    } else {
      Loads x[2];
      if (t0 < end) load_k(x[0], t0), load_v(x[0], t0);
      if (t0 + 32 * kTurns < end) load_k(x[1], t0 + 32 * kTurns), load_v(x[1], t0 + 32 * kTurns);
      for (; t0 < end; t0 += 64 * kTurns) {
        step(x[0], t0);
        if (t0 + 32 * kTurns < end) step(x[1], t0 + 32 * kTurns);
      }
    }
  }

  // join the waves that share rows
  st.l += __shfl_xor(st.l, 32);
  if (half == 0) stat[wave][n][0] = st.m, stat[wave][n][1] = st.l;
  __syncthreads();  // and the queries have been read
  float top = kNegInf;
#pragma unroll
  for (int w = 0; w < kTurns; ++w) top = fmaxf(top, stat[w * R + part][n][0]);
  const float base = top == kNegInf ? 0.f : top, mine = __builtin_amdgcn_exp2f(st.m - base);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) *(f32x4 *)sums[wave][4 * i + g][lane] = four_of<D, Held>(st, i, g) * mine;
  float l = 0.f;
#pragma unroll
  for (int w = 0; w < kTurns; ++w) l += stat[w * R + part][n][1] * __builtin_amdgcn_exp2f(stat[w * R + part][n][0] - base);
  __syncthreads();
  if (bad) l = __builtin_nanf("");
  if (row >= rows) return;
  if (u.slot >= 0 && turn == 0 && half == 0) {
    float *ml = unit_ml<D, M, V>(a, u.slot, u.kvh, trow);
    ml[0] = top, ml[1] = l;
  }
  const float inv = finish(l);
  for (int i = turn; i < D / 8; i += kTurns) {
    f32x4 o{};
#pragma unroll
    for (int w = 0; w < kTurns; ++w) o += *(const f32x4 *)sums[w * R + part][i][lane];
    const int d = four_at<Held>(i / 4, i % 4, half);
    if (u.slot >= 0)
      *(f32x4 *)(unit_o<D, M, V>(a, u.slot, u.kvh, trow) + d) = o;
    else
      store_out<E, D>(a, u.q, u.kvh, row, d, o * inv);
  }
}

template <class E, int D, int R>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void attend_few_kernel(AttendArgs a) {
  __shared__ __align__(16) FewLds<D> lds;
  few_body<E, D, R, false, kAll>(a, lds, blockIdx.x);
}

// ---------------------------------------------------------------------------------------------
// Many rows per sequence: prompts and their chunks.  Bound by the matrix cores and the softmax's
// vector work.  The four waves of a block take 32 rows each and share the keys: tiles of 64 keys
// and values go from memory into LDS by direct loads, the next tile while this one is multiplied.
// Two blocks to a CU: one's softmax runs beside the other's products.  A wave's 32 rows read 32 KB of
// LDS for 1024 cycles of products, the full rate of LDS; the products take 40 % of the time, the
// softmax's exponentials, sums and conversions about as much again.  The loop holds no step with
// masks (those take a path of their own, with half the speed).  Measured: 4096 tokens behind
// 12288, 32 heads of 128 on 4, 0.96 TFLOP: the call 0.915 to 0.925 ms = 1.04 PFLOP/s (a library product of 8192^3: 1.17).
// 16 heads of 256 on 4, 4096 tokens behind 4096: 0.54 ms = 0.76 PFLOP/s.
//
// Of a cache of 8 bits the next tile comes into registers and from there to LDS in 16 bits, laid out alike, a quarter
// to a wave; values' powers of two go to the probabilities in bf16 (multiplying the values, as in fp16, took 3 % more
// for the 4096 tokens).  These: the call 1.005 ms = 0.96 PFLOP/s, the kernel alone 1.01 traced.
// ---------------------------------------------------------------------------------------------
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_void;

template <int D>
struct ManyLds {
  uint8_t tiles[4 * 64 * D * 2];  // [2][K tile, V tile], each four groups
  int ids[kIds];
  int bad;
  alignas(16) float scales[2][64];  // of the V tiles' tokens, where they are not in the tile's values
};
template <class E, int D, bool Held, Cover V>
__device__ __forceinline__ void many_body(const AttendArgs &a, ManyLds<D> &shared, int block) {
  constexpr int M = 128, KT = 64;
  typedef typename std::conditional<Held, uint8_t, uint16_t>::type S;
  // bf16: values' powers of two go to the probabilities (which fp16 has no room for)
  constexpr bool kFold = Held && __is_same(E, __bf16);
  constexpr int kTileBytes = KT * D * 2;
  auto &lds = shared.tiles;
  auto &ids = shared.ids;
  int &bad = shared.bad;
  Unit u;
  if (!unit_of<M, V>(a, block, &u)) return;
  if (u.q.bad) {
    refuse<E, D, M>(a, u);
    return;
  }
  const KvView &kv = a.kv;
  const int lane = threadIdx.x % kLanes, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kLanes);
  const int half = lane / 32, n = lane % 32;
  if (threadIdx.x == 0) bad = 0;
  const int rows = u.q.count * kv.group, wrow = u.tile * M + 32 * wave, row = wrow + n;
  const int before = u.q.length - u.q.count;
  const int pos = row < rows ? before + row / kv.group : -1;
  const int window = V == kAll ? a.window : 0, floor = window ? pos - window : -1;
  // positions of this wave's first and last row (none: last below every key)
  const int first = before + wrow / kv.group;
  const int last = wrow < rows ? before + (min(wrow + 32, rows) - 1) / kv.group : -1;
  u32x4 q[D / 16];
  load_q<D, false>(a, u.q, u.kvh, row, q);

  Rows<D> st;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) st.acc[i] = f32x16{};
  st.m = kNegInf;
  st.l = 0.f;

  const int shift = kv.page_shift, P = 1 << shift;
  const int key = (lane & 19) | (lane & 4) << 1 | (lane & 8) >> 1;  // pi(lane): bits 2 and 3 swapped
  const int64_t head_elems = (int64_t)D << shift, page_elems = head_elems * kv.kv_heads;
  const S *keys = (const S *)kv.keys + u.kvh * head_elems, *values = (const S *)kv.values + u.kvh * head_elems;
  const uint8_t *ks = kv.key_scales + (u.kvh << shift), *vs = kv.value_scales + (u.kvh << shift);
  const int pg_last = (u.k1 - 1) >> shift;
  const int pg_seen = V == kPrefix ? 0 : first_page(a, before + u.tile * M / kv.group);
  const int32_t *pages = V == kPrefix ? a.prefix : kv.pages + (int64_t)u.seq * kv.max_pages;

  for (int pg0 = u.k0 >> shift; pg0 <= pg_last; pg0 += kIds) {
    __syncthreads();  // ids and tiles of the round before have been read
    load_ids(kv, pages, pg0, pg_last, pg_seen, ids, &bad);
    const int begin = max(u.k0, pg0 << shift);
    const int end = (int)min((int64_t)u.k1, ((int64_t)pg0 + kIds) << shift);
    // tile t0 into buffer b: four groups' keys and values as they lie in memory, one group to
    // a wave; a group past the end is read from the last one's place
    auto stage = [&](int t0, int b) {
      if constexpr (Held) return;
      const int t = min(t0 + 16 * wave, (end - 1) & ~15);
      const int64_t at = ids[(t >> shift) - pg0] * page_elems + (t & (P - 1)) * D + lane * 8;
      uint8_t *dst = lds + b * 2 * kTileBytes + wave * 16 * D * 2;
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
        __builtin_amdgcn_global_load_lds((global_void *)(keys + at + i * 512), (lds_void *)(dst + i * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_void *)(values + at + i * 512),
                                         (lds_void *)(dst + kTileBytes + i * 1024), 16, 0, 0);
      }
    };
    // 8 bits: into registers, from which a tile goes to LDS in 16 bits, laid out alike
    u32x4 kr[Held ? D / 64 : 1], vr[Held ? D / 64 : 1];
    uint32_t kb, vb;
    uint2 vb8[Held && !kFold ? D / 64 : 1];
    auto fetch = [&](int t0) {
      if constexpr (Held) {
        const int t = min(t0 + 16 * wave, (end - 1) & ~15);
        const int64_t id = ids[(t >> shift) - pg0], at = id * page_elems + (t & (P - 1)) * D + lane * 16;
        const int64_t sc = ((id * kv.kv_heads) << shift) + (t & (P - 1));
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          kr[i] = *(const u32x4 *)(keys + at + i * 1024);
          vr[i] = *(const u32x4 *)(values + at + i * 1024);
          if constexpr (!kFold) vb8[i] = *(const uint2 *)(vs + sc + 8 * ((i * 64 + lane) / (D / 2)));
        }
        kb = ks[sc + lane % 16];
        if constexpr (kFold) vb = vs[sc + lane % 16];
      }
    };
    auto unpack = [&](int b) {
      if constexpr (Held) {
        uint8_t *dst = lds + b * 2 * kTileBytes + wave * 16 * D * 2;
        const float s = scale_of(kb);
        if (kFold && lane < 16) shared.scales[b][wave * 16 + lane] = scale_of(vb);
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
          const int unit = i * 64 + lane;  // keys: 16 elements of a token; values: eight tokens of two elements
          uint8_t *kd = dst + (unit / 16 * 32 + unit % 16) * 16, *vd = dst + kTileBytes + unit * 32;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            *(u32x4 *)(kd + j * 256) = operand<E>(kr[i][2 * j], kr[i][2 * j + 1], s);
            u32x4 v = operand<E>(vr[i][2 * j], vr[i][2 * j + 1], 1.f);
            if constexpr (!kFold) v = times_pairs(v, scales_of(vb8[i]));
            *(u32x4 *)(vd + j * 16) = v;
          }
        }
      }
    };
    // this lane's operands within 32 keys' and 16 values' bytes
    const int koff = key / 16 * 32 * D + (16 * half + key % 16) * 16, voff = (half * D + n) * 16;
    stage(begin, 0);
    if constexpr (Held) {
      fetch(begin);
      unpack(0);
      if (begin + KT < end) fetch(begin + KT);
    }
    int b = 0;
    for (int t0 = begin; t0 < end; t0 += KT, b ^= 1) {
      asm volatile("" ::: "memory");
      // this wave's part of the tile has landed: vmcnt(0), or where it was written from registers lgkmcnt(0)
      __builtin_amdgcn_s_waitcnt(Held ? 0xc07f : 0x0f70);
      __builtin_amdgcn_s_barrier();  // everyone's has, and the other buffer is free
      asm volatile("" ::: "memory");
      if (t0 + KT < end) {
        stage(t0 + KT, b ^ 1);
        unpack(b ^ 1);
        if (Held && t0 + 2 * KT < end) fetch(t0 + 2 * KT);
      }
      // none of the wave's rows sees it
      if (V != kPrefix && (t0 > last || (window && t0 + KT - 1 <= first - window))) continue;
      const uint8_t *kt = lds + b * 2 * kTileBytes, *vt = kt + kTileBytes;
      f32x16 s[2] = {};
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          s[j] = mma(*(const u32x4 *)(kt + j * 64 * D + c * 512 + koff), q[c], s[j], E());
      const bool edge = V != kPrefix && (t0 + KT - 1 > first || (window && t0 <= last - window));
      auto softmax = [&](u32x4 (&p)[4]) {
        if constexpr (kFold)
          softmax_step<E, D, 2>(s, st, p, a.scale_log2,
                                [&](int c) { return *(const Eight *)(shared.scales[b] + 16 * c + 8 * half); });
        else
          softmax_step<E, D, 2>(s, st, p, a.scale_log2);
      };
      u32x4 p[4];
      if (!edge) {
        softmax(p);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int i = 0; i < D / 32; ++i)
            st.acc[i] = mma(*(const u32x4 *)(vt + c * 32 * D + i * 512 + voff), p[c], st.acc[i], E());
      } else {
        mask_scores<2>(s, t0, pos, floor);
        softmax(p);
        bool odd = false;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          u32x4 v[D / 32];
#pragma unroll
          for (int i = 0; i < D / 32; ++i) v[i] = *(const u32x4 *)(vt + c * 32 * D + i * 512 + voff);
          odd |= clean_values<E, D>(v, t0 + 16 * c, u.q.length);
#pragma unroll
          for (int i = 0; i < D / 32; ++i) st.acc[i] = mma(v[i], p[c], st.acc[i], E());
          __builtin_amdgcn_sched_barrier(0);
        }
        if (odd)
          add_odd<E, D, S, false>(st, values, vs, kv.kv_heads, ids, pg0, shift, page_elems, t0, min(t0 + KT, end), pos, floor);
      }
    }
  }

  // this lane's row again, from its number alone: the loop leaves no register for it
  int own = threadIdx.x % kLanes;
  asm volatile("" : "+v"(own));
  const int trow = 32 * wave + own % 32, end_row = u.tile * M + trow, own_half = own / 32;
  if (end_row >= rows) return;
  float l = st.l + __shfl_xor(st.l, 32);
  if (bad) l = __builtin_nanf("");
  if (u.slot >= 0 && own_half == 0) {
    float *ml = unit_ml<D, M, V>(a, u.slot, u.kvh, trow);
    ml[0] = st.m, ml[1] = l;
  }
  const float inv = finish(l);
#pragma unroll
  for (int i = 0; i < D / 32; ++i)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 o{st.acc[i][4 * g], st.acc[i][4 * g + 1], st.acc[i][4 * g + 2], st.acc[i][4 * g + 3]};
      const int d = 32 * i + 8 * g + 4 * own_half;
      if (u.slot >= 0)
        *(f32x4 *)(unit_o<D, M, V>(a, u.slot, u.kvh, trow) + d) = o;
      else
        store_out<E, D>(a, u.q, u.kvh, end_row, d, o * inv);
    }
}

template <class E, int D>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void attend_many_kernel(AttendArgs a) {
  __shared__ __align__(16) ManyLds<D> lds;
  many_body<E, D, false, kAll>(a, lds, blockIdx.x);
}

// ---------------------------------------------------------------------------------------------
// Joins the units of split tiles: gridDim.y blocks per tile and KV head take every gridDim.y-th of the
// tile's rows each (so that the few rows of a decode step get a block each).  The block's groups of D / 4
// lanes share out a row's units, or several rows' where there are fewer units than groups.  Bound by the
// latency of three dependent reads: 6 us for 512 units of one token, 3.5 with nothing to join.
// ---------------------------------------------------------------------------------------------
template <class E, int D, int M>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a) {
  constexpr int kPer = D / 4, kGroups = kThreads / kPer;
  __shared__ __align__(16) float sum[kGroups][D];
  __shared__ float stat[kGroups][2];
  const int item = blockIdx.x / a.kv.kv_heads, kvh = blockIdx.x % a.kv.kv_heads;
  const SplitTile t = split_tiles(a)->tile[item];
  if (item >= split_tiles(a)->count) return;
  // starts out of order can leave a note unwritten: nothing is taken from one that makes no sense
  if (t.units < 2 || t.slot < 0 || t.slot > a.max_slots - t.units || t.rows < 1 || t.rows > M || t.first < 0 ||
      t.row0 < 0 || t.row0 > (1 << 28) || t.first > a.kv.n_tokens - 1 - (t.row0 + t.rows - 1) / a.kv.group)
    return;
  const int g = threadIdx.x / kPer, d = threadIdx.x % kPer * 4;
  // groups to a row: a power of two, so that a tile of few units has several rows joined at once
  int per = 1;
  while (per < kGroups && per < t.units) per *= 2;
  const int own = g / per, at_once = kGroups / per;
  const int64_t step = (int64_t)a.kv.kv_heads * M;  // rows from unit to unit
  for (int r0 = 0; (int)(blockIdx.y + gridDim.y * r0) < t.rows; r0 += at_once) {
    const int row = blockIdx.y + gridDim.y * (r0 + own);
    float m = kNegInf, l = 0.f;
    f32x4 o{};
    if (row < t.rows) {
      const float *ml = part_ml<D, M>(a, t.slot, kvh, row), *part = part_o<D, M>(a, t.slot, kvh, row) + d;
#pragma unroll 4
      for (int i = g % per; i < t.units; i += per) {
        const float mi = ml[i * step * 2], li = ml[i * step * 2 + 1];
        const f32x4 oi = *(const f32x4 *)(part + i * step * D);
        const float top = fmaxf(m, mi), base = top == kNegInf ? 0.f : top;
        const float w = __builtin_amdgcn_exp2f(mi - base), shrink = __builtin_amdgcn_exp2f(m - base);
        l = l * shrink + w * li;
        o = o * shrink + w * oi;
        m = top;
      }
    }
    *(f32x4 *)&sum[g][d] = o;
    if (d == 0) stat[g][0] = m, stat[g][1] = l;
    __syncthreads();
    if (g % per == 0 && row < t.rows) {
      float top = kNegInf;
      for (int i = 0; i < per; ++i) top = fmaxf(top, stat[g + i][0]);
      const float base = top == kNegInf ? 0.f : top;
      o = f32x4{};
      l = 0.f;
      for (int i = 0; i < per; ++i) {
        const float w = __builtin_amdgcn_exp2f(stat[g + i][0] - base);
        o += w * *(const f32x4 *)&sum[g + i][d];
        l += w * stat[g + i][1];
      }
      store_out<E, D>(a, Seq{t.first, 0, 0, false}, kvh, t.row0 + row, d, o * finish(l));
    }
    __syncthreads();
  }
}

}  // namespace
static inline uint64_t attend_work_size(const AttendArgs &a, int rows, int dim) {
  return sizeof(SplitTiles) + a.max_tiles * sizeof(SplitTile) + plan_ints(a) * sizeof(int32_t) +
         (uint64_t)a.max_slots * a.kv.kv_heads * rows * (dim + 2) * sizeof(float);
}
namespace {

// Blocks that join: most have nothing to do.  About 4096 in all, 8 to rows / 4 of them to a tile.
static inline dim3 join_grid(const AttendArgs &a, int rows) {
  const int tiles = a.max_tiles * a.kv.kv_heads;
  int y = 8;
  while (2 * y <= rows / 4 && 2 * y * tiles <= 4096) y *= 2;
  return dim3(tiles, y);
}
template <class E, int D>
const void *join_kernel(int rows) {
  return rows == 32   ? (const void *)attend_join_kernel<E, D, 32>
         : rows == 64 ? (const void *)attend_join_kernel<E, D, 64>
                      : (const void *)attend_join_kernel<E, D, 128>;
}

template <class E, int D, int M>
hipError_t launch_kernels(const AttendArgs &a, hipStream_t s) {
  void *args[] = {const_cast<AttendArgs *>(&a)};
  const dim3 grid((unsigned)((int64_t)a.max_units * a.kv.kv_heads));
  const void *fn;
  if constexpr (M == 128)
    fn = (const void *)attend_many_kernel<E, D>;
  else
    fn = (const void *)attend_few_kernel<E, D, M / 32>;
  hipError_t e = launch_plan<D>(a, M, s);
  if (e == hipSuccess) e = hipLaunchKernel(fn, grid, dim3(kThreads), args, 0, s);
  if (e != hipSuccess) return e;
  return hipLaunchKernel(join_kernel<E, D>(M), join_grid(a, M), dim3(kThreads), args, 0, s);
}

}  // namespace

template <int D>
hipError_t launch_plan(const AttendArgs &a, int rows, hipStream_t s) {
  if (a.kv.n_seqs <= kPlanSeqs) return hipSuccess;
  void *args[] = {const_cast<AttendArgs *>(&a)};
  const void *fn = rows == 32   ? (const void *)plan_kernel<32>
                   : rows == 64 ? (const void *)plan_kernel<64>
                                : (const void *)plan_kernel<128>;
  return hipLaunchKernel(fn, dim3(1), dim3(kPlanThreads), args, 0, s);
}

template <int D>
hipError_t launch_join(const AttendArgs &a, bool half, int rows, hipStream_t s) {
  void *args[] = {const_cast<AttendArgs *>(&a)};
  return hipLaunchKernel(half ? join_kernel<_Float16, D>(rows) : join_kernel<__bf16, D>(rows), join_grid(a, rows),
                         dim3(kThreads), args, 0, s);
}

template <int D>
hipError_t launch_attend(const AttendArgs &a, bool half, int rows, hipStream_t s) {
  if (rows == 64) return half ? launch_kernels<_Float16, D, 64>(a, s) : launch_kernels<__bf16, D, 64>(a, s);
  if (rows == 32) return half ? launch_kernels<_Float16, D, 32>(a, s) : launch_kernels<__bf16, D, 32>(a, s);
  return half ? launch_kernels<_Float16, D, 128>(a, s) : launch_kernels<__bf16, D, 128>(a, s);
}

}  // namespace moecache
