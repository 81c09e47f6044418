// The choice of a token from each row of logits: temperature, top-k, top-p, min-p, then a draw
// with a given uniform number.
//
//   w_i = exp((z_i - max z) / T)
//   S1 = the k largest (equal logits: lower indices first)
//   S2 = the elements of S1 before which, in falling order, less than p * mass(S1) lies
//   S3 = the elements of S2 with w_i >= min_p
//   token = the first i, in rising index, whose running mass over S3 exceeds u * mass(S3)
//
// Whether an element is in and where the draw falls are decisions on sums of up to 2^20 weights, so
// the weights are taken in 64 bits and then held as integers of 2^-s, s = 62 - log2 of the row's
// length (at most 50): sums of integers do not depend on their order, so every split of a row over
// threads gives the same token, and two tokens' border is off by at most 2^(20 - s) of the
// largest weight.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "serve.h"

namespace moecache {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;  // of the draw, a block per row
constexpr int kSliceThreads = 256;                      // of the passes over slices of a row
constexpr int kSliceWaves = kSliceThreads / 64;
constexpr int kMaxBlocks = 64;                          // of a row's passes; its slices are their waves
constexpr int kMaxSlices = kMaxBlocks * kSliceWaves;
constexpr int kBins = 2048;
constexpr int kCandidates = 4096;
constexpr int kOwn = 512;  // of them, a block's, before it hands them over one by one

// Per row in the workspace.
struct RowWork {
  uint64_t best[kMaxBlocks];     // blocks' largest logit: rank key, then the smallest index
  uint64_t sums[kMaxSlices][3];  // slices' masses, see collect_kernel
  uint64_t mass[kBins];          // binned, in 2^-31
  uint32_t count[kBins];
  uint64_t list[kCandidates];    // codes of the elements that need ranking
  int32_t n_list;                // how many there are, in the list or not
  int32_t high, rank_bin;        // last bin of the top-p cut's; bin of the top-k cut (kBins: none)
  uint32_t before_rank;          // elements in bins before rank_bin
};

template <class Z>
__device__ __forceinline__ float logit(const void *row, int i) {
  return (float)((const Z *)row)[i] + 0.f;  // -0 + 0 = 0: the two zeros rank alike
}
// Order of floats as unsigned integers; a NaN ranks last.
__device__ __forceinline__ uint32_t rank_key(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z);
  return z != z ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float unrank(uint32_t key) {
  return __builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
// Elements in falling order, equal logits by rising index, are rising codes.
__device__ __forceinline__ uint64_t code_of(uint32_t key, int i) { return (uint64_t)~key << 32 | (uint32_t)i; }

// Calls f(logits, index of the first) for lo <= index < hi, by one wave: as many consecutive logits to a
// lane as 16 bytes hold, NaNs where there are none, four loads in flight.  Every lane takes part in
// every call.
template <class Z>
constexpr int kVec = 16 / sizeof(Z);
template <class Z, class F>
__device__ __forceinline__ void for_each(const void *row, int lo, int hi, F f) {
  constexpr int kAhead = 4, V = kVec<Z>;
  typedef Z zv __attribute__((ext_vector_type(V)));
  const Z *z = (const Z *)row;
  const float nan = __builtin_nanf("");
  const int lane = threadIdx.x % 64;
  const int skip = (int)(-(uintptr_t)(z + lo) / sizeof(Z) % V);
  const int body = min(hi, lo + skip), vecs = (hi - body) / V, tail = body + vecs * V;
  // fewer than 16 bytes on either side: lanes 0 .. V - 1 and V .. 2 V - 1
  const int at = lane < V ? lo + lane : tail + lane - V;
  const bool edge = lane < V ? at < body : lane < 2 * V && at < hi;
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = nan;
  if (edge) v[0] = (float)z[at] + 0.f;
  if (body > lo || hi > tail) f(v, at);
  for (int v0 = lane; v0 - lane < vecs; v0 += 64 * kAhead) {
    zv e[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (v0 + 64 * u < vecs) e[u] = *(const zv *)(z + body + (v0 + 64 * u) * V);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int at = v0 + 64 * u;
      if (at - lane >= vecs) break;
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = at < vecs ? (float)e[u][j] + 0.f : nan;
      f(v, body + at * V);
    }
  }
}

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor((unsigned long long)v, o);
  return v;
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
  for (int o = 32; o; o >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, o));
  return v;
}

// exp((z - top) / T) in units of 2^-shift; a row's masses are sums of these, rounded to whole units.
struct Weigh {
  float top;     // the row's largest logit
  double scale;  // 1 / T
  int shift;     // at most 50
  // With x = n ln 2 + g, |g| <= ln 2 / 2: e^x = 2^n e^g, e^g by its series to g^11 / 11! (what is left
  // is below 2^-47 of it).  0 for NaN and -inf.
  __device__ __forceinline__ double operator()(float z) const {
    const double x = ((double)z - (double)top) * scale;
    const double n = rint(x * 1.4426950408889634);
    const double g = fma(n, -1.9082149292705877e-10, fma(n, -0.6931471803691238, x));  // ln 2 in two parts
    // odd and even powers apart: two chains of half the length
    const double g2 = g * g;
    double even = 1.0 / 3628800, odd = 1.0 / 39916800;
    even = fma(even, g2, 1.0 / 40320);
    odd = fma(odd, g2, 1.0 / 362880);
    even = fma(even, g2, 1.0 / 720);
    odd = fma(odd, g2, 1.0 / 5040);
    even = fma(even, g2, 1.0 / 24);
    odd = fma(odd, g2, 1.0 / 120);
    even = fma(even, g2, 0.5);
    odd = fma(odd, g2, 1.0 / 6);
    odd = fma(odd, g2, 1.0);
    const double e = fma(odd, g, fma(even, g2, 1.0));
    const uint64_t bits = __builtin_bit_cast(uint64_t, e) + ((uint64_t)(uint32_t)((int)n + shift) << 52);
    const double w = __builtin_bit_cast(double, bits);
    // e^-64 is below a half of every unit; a NaN compares false
    return z == top ? (double)(1ull << shift) : x > -64.0 ? w : 0.0;
  }
  __device__ __forceinline__ uint64_t units(float z) const { return (uint64_t)rint((*this)(z)); }
};

// A row's settings, and its largest logit.
struct Row {
  float top, T, p, least;
  int first, k;
  bool none, greedy;  // nothing but -inf and NaN; the first largest is the answer
  __device__ Row(const SampleArgs &a, int row, uint64_t best) {
    first = (int)~(uint32_t)best;
    top = unrank((uint32_t)(best >> 32));
    T = a.temperature ? a.temperature[row] : 1.f;
    p = a.top_p ? a.top_p[row] : 1.f;
    k = a.top_k ? a.top_k[row] : 0;
    if (k <= 0 || k >= a.vocab) k = 0;
    least = a.min_p ? a.min_p[row] : 0.f;
    if (least > 1.f) least = 1.f;
    none = !(top > -__builtin_inff());
    greedy = !(T > 0.f);
  }
  __device__ __forceinline__ bool ranked() const { return k || p < 1.f; }
  __device__ __forceinline__ Weigh weigh(int shift) const {
    return Weigh{top, 1.0 / (double)T, shift};
  }
};

// Bins of (top - z) / T, rising with falling logits; weights beyond the last are below half of 2^-s.
struct Binning {
  float top, scale, limit, per;
  __device__ Binning(const Row &r, int shift) : top(r.top), scale(2.f / r.T) {
    limit = (float)(shift + 1) * 0.69314718f + 0.01f;
    per = kBins / limit;
  }
  // (of halves: two logits may be further apart than the largest float)
  __device__ __forceinline__ float depth(float z) const { return z == top ? 0.f : (0.5f * top - 0.5f * z) * scale; }
  __device__ __forceinline__ int bin(float x) const { return x < limit ? min(kBins - 1, (int)(x * per)) : kBins; }
  // the same as a number to compare with starts and ends of bins: bin <= b is place < end(b)
  __device__ __forceinline__ float place(float x) const { return x < limit ? fminf(x * per, kBins - 0.5f) : __builtin_inff(); }
  static __device__ __forceinline__ float end(int b) { return b >= kBins - 1 ? __builtin_inff() : (float)(b + 1); }
};

// The largest of the blocks' bests; every wave of the block for itself.
__device__ __forceinline__ uint64_t row_best(const RowWork &w, int blocks) {
  const int lane = threadIdx.x % 64;
  return wave_max(lane < blocks ? w.best[lane] : 0);
}

// Pass 1, a wave per slice of a row: its largest logit; the row's bins are cleared on the way.
template <class Z>
__global__ __launch_bounds__(kSliceThreads) void largest_kernel(SampleArgs a, int len) {
  RowWork &w = ((RowWork *)a.work)[blockIdx.y];
  const void *z = (const Z *)a.logits + (int64_t)blockIdx.y * a.stride;
  const int slice = blockIdx.x * kSliceWaves + threadIdx.x / 64, lo = min(a.vocab, slice * len);
  for (int i = blockIdx.x * kSliceThreads + threadIdx.x; i < kBins; i += gridDim.x * kSliceThreads)
    w.mass[i] = 0, w.count[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) w.n_list = 0;
  uint64_t best = 0;
  for_each<Z>(z, lo, min(a.vocab, lo + len), [&](const float (&v)[kVec<Z>], int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kVec<Z>; ++j) best = max(best, (uint64_t)rank_key(v[j]) << 32 | (uint32_t)~(i + j));
  });
  __shared__ uint64_t scratch[kSliceWaves];
  best = wave_max(best);
  if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = best;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kSliceWaves; ++i) best = max(best, scratch[i]);
    w.best[blockIdx.x] = best;
  }
}

// Pass 2, for rows with a filter by rank: elements (for top-k) and mass (for top-p) by bin, four
// blocks' slices to a block (each block adds its bins to the row's one by one).  The
// masses here are of 32-bit exponentials, rounded to 2^-31: they only choose which bins need
// ranking, with their errors allowed for (least_of, most_of).
template <class Z>
__global__ __launch_bounds__(kThreads) void bins_kernel(SampleArgs a, int blocks, int len, int shift) {
  RowWork &w = ((RowWork *)a.work)[blockIdx.y];
  const Row r(a, blockIdx.y, row_best(w, blocks));
  if (r.none || r.greedy || !r.ranked()) return;
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  for (int i = threadIdx.x; i < kBins; i += kThreads) mass[i] = 0, count[i] = 0;
  __syncthreads();
  const void *z = (const Z *)a.logits + (int64_t)blockIdx.y * a.stride;
  const int lo = min(a.vocab, (int)(blockIdx.x * kWaves + threadIdx.x / 64) * len);
  const Binning bin(r, shift);
  const bool by_mass = r.p < 1.f, by_count = r.k != 0;
  for_each<Z>(z, lo, min(a.vocab, lo + len), [&](const float (&v)[kVec<Z>], int) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kVec<Z>; ++j) {
      const float x = bin.depth(v[j]);
      const int b = bin.bin(x);
      if (b >= kBins) continue;
      if (by_mass) {
        const uint32_t m = (uint32_t)rintf(__builtin_amdgcn_exp2f(x * -1.44269504f) * 0x1p31f);
        atomicAdd((unsigned long long *)&mass[b], (unsigned long long)m);
      }
      if (by_count) atomicAdd(&count[b], 1u);
    }
  });
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    if (mass[i]) atomicAdd((unsigned long long *)&w.mass[i], (unsigned long long)mass[i]);
    if (count[i]) atomicAdd(&w.count[i], count[i]);
  }
}

// Bounds on the exact mass, in 2^-31, of elements whose binned masses sum to m: half a unit for each of at most
// V elements, and the exponentials' own error (their arguments, up to 44, are off by a few
// parts in 2^24: the results by less than 2^-15).
__device__ __forceinline__ double least_of(uint64_t m, int V) { return (double)m * (1.0 - 0x1p-15) - 0.5 * V; }
__device__ __forceinline__ double most_of(uint64_t m, int V) { return (double)m * (1.0 + 0x1p-15) + 0.5 * V; }

// Pass 3: which bins may hold a cut (every block of a row finds them for itself), the elements of
// those bins into the row's list, and each slice's exact masses of
//   0: elements in bins before the list's
//   1: those of them that min_p keeps
//   2: elements in bins between the top-p cut's and the top-k cut's
template <class Z>
__global__ __launch_bounds__(kSliceThreads) void collect_kernel(SampleArgs a, int len, int shift) {
  RowWork &w = ((RowWork *)a.work)[blockIdx.y];
  constexpr int kPer = kBins / kSliceThreads;
  uint64_t mass[kPer];  // asked for together with the row's settings
  uint32_t count[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    mass[i] = w.mass[threadIdx.x * kPer + i];
    count[i] = w.count[threadIdx.x * kPer + i];
  }
  const Row r(a, blockIdx.y, row_best(w, gridDim.x));
  if (r.none || r.greedy) return;
  __shared__ uint64_t mine[kOwn], scratch[kSliceWaves];
  __shared__ uint32_t counts[kSliceWaves];
  __shared__ int cuts[3], n_mine, place;
  __shared__ double reach[2];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, V = a.vocab;
  // bins low .. high and rank_bin go into the list; bins past `last` hold nothing that is kept
  int low = kBins, high = kBins, rank_bin = kBins;
  if (threadIdx.x == 0) n_mine = 0;
  if (r.ranked()) {
    uint64_t up = 0;
    uint32_t up_n = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) up += mass[i], up_n += count[i];
    uint64_t before = up;
    uint32_t before_n = up_n;
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t m = __shfl_up((unsigned long long)up, o);
      const uint32_t n = __shfl_up(up_n, o);
      if (lane >= o) up += m, up_n += n;
    }
    if (lane == 63) scratch[wave] = up, counts[wave] = up_n;
    if (threadIdx.x == 0) cuts[0] = 0, cuts[1] = kBins - 1, cuts[2] = kBins;
    __syncthreads();
    before = up - before;
    before_n = up_n - before_n;
    uint64_t all = 0;
    uint32_t all_n = 0;
    for (int i = 0; i < kSliceWaves; ++i) {
      if (i < wave) before += scratch[i], before_n += counts[i];
      all += scratch[i];
      all_n += counts[i];
    }
    const bool cut_k = r.k && (uint32_t)r.k < all_n;  // else top-k cuts nothing but weights of 0
    if (threadIdx.x == 0 && !cut_k) reach[0] = least_of(all, V), reach[1] = most_of(all, V);
    if (cut_k) {
      uint64_t at = before;
      uint32_t n = before_n;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (n < (uint32_t)r.k && n + count[i] >= (uint32_t)r.k) {  // in one thread's one bin
          cuts[2] = threadIdx.x * kPer + i;
          reach[0] = least_of(at, V), reach[1] = most_of(at + mass[i], V);
          if (blockIdx.x == 0) w.before_rank = n;
        }
        at += mass[i];
        n += count[i];
      }
    }
    __syncthreads();
    low = high = rank_bin = cuts[2];
    if (r.p < 1.f) {
      // what top-p reaches for lies between these
      const double least = (double)r.p * reach[0], most = (double)r.p * reach[1] + 1.0;
      uint64_t at = before;
      int begun = 0, ended = kBins - 1;
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int b = threadIdx.x * kPer + i;
        // the last bin that begins before it for certain, the first that ends past it for certain
        if (most_of(at, V) < least) begun = b;
        at += mass[i];
        if (least_of(at, V) >= most) ended = min(ended, b);
      }
      for (int o = 32; o; o >>= 1) begun = max(begun, __shfl_xor(begun, o)), ended = min(ended, __shfl_xor(ended, o));
      if (lane == 0) atomicMax(&cuts[0], begun), atomicMin(&cuts[1], ended);
      __syncthreads();
      high = min(cuts[1], rank_bin);
      low = min(cuts[0], high);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) w.high = high, w.rank_bin = rank_bin;
  }
  __syncthreads();

  const void *z = (const Z *)a.logits + (int64_t)blockIdx.y * a.stride;
  const int slice = blockIdx.x * kSliceWaves + wave, lo = min(V, slice * len);
  const Binning bin(r, shift);
  const Weigh weigh = r.weigh(shift);
  const double least = (double)r.least * (double)(1ull << shift);
  const float low_start = (float)low, high_end = bin.end(high), rank_start = (float)rank_bin,
              rank_end = bin.end(rank_bin), last_end = rank_bin < kBins ? rank_end : __builtin_inff();
  const bool parted = high < rank_bin && low < kBins;  // elements past the list's first part count apart
  // whole units, exact in a double up to 2^53: so many sums at a time
  uint64_t before_low = 0, kept_low = 0, between = 0;
  double before_d = 0, kept_d = 0, between_d = 0;
  int room = 1 << (53 - shift);
  auto flush = [&]() __attribute__((always_inline)) {
    before_low += (uint64_t)before_d, kept_low += (uint64_t)kept_d, between += (uint64_t)between_d;
    before_d = kept_d = between_d = 0;
    room = 1 << (53 - shift);
  };
  for_each<Z>(z, lo, min(V, lo + len), [&](const float (&v)[kVec<Z>], int i) __attribute__((always_inline)) {
    // with a top-k cut few of a row's elements matter: most calls end here
    float f[kVec<Z>], least_f = __builtin_inff();
#pragma unroll
    for (int j = 0; j < kVec<Z>; ++j) least_f = fminf(least_f, f[j] = bin.place(bin.depth(v[j])));
    if (!__any(least_f < last_end)) return;
#pragma unroll
    for (int j = 0; j < kVec<Z>; ++j) {
      const bool listed = (f[j] >= low_start && f[j] < high_end) || (f[j] >= rank_start && f[j] < rank_end);
      if (listed) {
        const uint64_t code = code_of(rank_key(v[j]), i + j);
        const int at = atomicAdd(&n_mine, 1);
        if (at < kOwn) {
          mine[at] = code;
        } else {
          const int far = atomicAdd(&w.n_list, 1);
          if (far < kCandidates) w.list[far] = code;
        }
      }
      const double x = weigh(v[j]), n = rint(x);
      const bool in = f[j] < last_end && !listed, early = !parted || f[j] < low_start;
      before_d += in && early ? n : 0;
      kept_d += in && early && !(x < least) ? n : 0;
      between_d += in && !early ? n : 0;
    }
    if ((room -= kVec<Z>) < kVec<Z>) flush();
  });
  flush();
  before_low = wave_sum(before_low), kept_low = wave_sum(kept_low), between = wave_sum(between);
  if (lane < 3) w.sums[slice][lane] = lane == 0 ? before_low : lane == 1 ? kept_low : between;
  __syncthreads();
  if (threadIdx.x == 0 && n_mine) place = atomicAdd(&w.n_list, min(n_mine, kOwn));
  __syncthreads();
  for (int i = threadIdx.x; i < min(n_mine, kOwn); i += kSliceThreads)
    if (place + i < kCandidates) w.list[place + i] = mine[i];
}

// The cut as a code, found by going over the whole row: for rows with more elements in the bins
// that hold a cut than the list takes (few distinct logits).  A total in falling order (of ones,
// or of weights), over elements up to the code `in`, first reaches `want` at the code returned; want is at least 1
// and at most the total.
template <class Z>
__device__ uint64_t select_row(const void *z, int V, const Weigh &weigh, uint64_t want, bool weighted, uint64_t in,
                               uint64_t *hist, uint64_t *scratch, uint64_t *found) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  uint32_t key = 0;
  uint64_t above = 0;  // total over keys above the prefix's range
  for (int bits = 24; bits >= 0; bits -= 8) {
    for (int i = threadIdx.x; i < 256; i += kThreads) hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < V; i += kThreads) {
      const float x = logit<Z>(z, i);
      const uint32_t k = rank_key(x);
      if (code_of(k, i) > in || (bits < 24 && k >> (bits + 8) != key >> (bits + 8))) continue;
      const uint64_t n = weighted ? weigh.units(x) : 1;
      if (n) atomicAdd((unsigned long long *)&hist[k >> bits & 255], (unsigned long long)n);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint64_t sum = above;
      int d = 255;
      while (d > 0 && sum + hist[d] < want) sum += hist[d--];
      found[0] = d;
      found[1] = sum;
    }
    __syncthreads();
    key |= (uint32_t)found[0] << bits;
    above = found[1];
    __syncthreads();
  }
  // equal logits: the first `ties` of them by index
  const uint64_t one = weighted ? weigh.units(unrank(key)) : 1;
  const uint64_t ties = one ? (want - above + one - 1) / one : 1;
  uint64_t seen = 0;
  for (int base = 0; base < V; base += kThreads) {
    const int i = base + threadIdx.x;
    const bool tie = i < V && rank_key(logit<Z>(z, i)) == key && code_of(key, i) <= in;
    const uint64_t mask = __ballot(tie);
    if (lane == 0) scratch[wave] = __popcll(mask);
    __syncthreads();
    uint64_t before = seen;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) before += scratch[w];
      seen += scratch[w];
    }
    before += __popcll(mask & ((1ull << lane) - 1));
    if (tie && before + 1 == ties) found[0] = i;
    __syncthreads();
    if (seen >= ties) break;
  }
  const uint64_t cut = code_of(key, seen >= ties ? (int)found[0] : V);
  __syncthreads();
  return cut;
}

// What top-p reaches for, of a mass: at least 1, so that the first element stays.
__device__ __forceinline__ uint64_t reach_of(float p, uint64_t mass) {
  const double part = ceil((double)p * (double)mass);
  return part < 1.0 ? 1 : min(mass, (uint64_t)part);
}

// Pass 4, a block per row: ranks the listed elements, which gives the cut, then finds the slice in
// which the draw falls, and the element in it.
template <class Z>
__global__ __launch_bounds__(kThreads) void draw_kernel(SampleArgs a, int blocks, int len, int shift) {
  __shared__ uint64_t codes[kCandidates], parts[kCandidates];
  __shared__ uint64_t hist[256], scratch[kWaves], found[2], in_slice[kMaxSlices];
  __shared__ int n_early;
  const int row = blockIdx.x, V = a.vocab, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int slices = blocks * kSliceWaves;
  const RowWork &w = ((const RowWork *)a.work)[row];
  const void *z = (const Z *)a.logits + (int64_t)row * a.stride;
  const Row r(a, row, row_best(w, blocks));
  if (r.none || r.greedy) {
    if (threadIdx.x == 0) {
      a.token[row] = r.none ? -1 : r.first;
      if (a.prob) a.prob[row] = r.none ? 0.f : 1.f;
    }
    return;
  }
  const Weigh weigh = r.weigh(shift);
  const double least = (double)r.least * (double)(1ull << shift);
  auto kept = [&](float v, int i, uint64_t cut) -> uint64_t {
    if (code_of(rank_key(v), i) > cut) return 0;
    const double x = weigh(v);
    return x < least ? 0 : (uint64_t)rint(x);
  };
  uint64_t cut = ~0ull;  // code of the last element that the filters by rank keep
  const int n = r.ranked() ? w.n_list : 0;
  if (n <= kCandidates) {
    if ((int)threadIdx.x < kMaxSlices) {
      const bool real = (int)threadIdx.x < slices;
      in_slice[threadIdx.x] = real ? w.sums[threadIdx.x][1] : 0;
      const uint64_t ahead = wave_sum(real ? w.sums[threadIdx.x][0] : (uint64_t)0);
      const uint64_t between = wave_sum(real ? w.sums[threadIdx.x][2] : (uint64_t)0);
      if (lane == 0) scratch[wave] = ahead, scratch[kMaxSlices / 64 + wave] = between;
      if (threadIdx.x == 0) found[0] = found[1] = 0, n_early = 0;
    }
    for (int i = threadIdx.x; i < n; i += kThreads) {
      codes[i] = w.list[i];
      parts[i] = weigh.units(unrank(~(uint32_t)(codes[i] >> 32)));
    }
    __syncthreads();
    if (n) {
      uint64_t ahead = 0, between = 0;
#pragma unroll
      for (int i = 0; i < kMaxSlices / 64; ++i) ahead += scratch[i], between += scratch[kMaxSlices / 64 + i];
      const int high = w.high, rank_bin = w.rank_bin;
      const Binning bin(r, shift);
      constexpr int kEach = kCandidates / kThreads;
      uint64_t code[kEach], before[kEach];  // own elements, the listed mass before them
      int rank[kEach], at[kEach];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = e * kThreads + threadIdx.x;
        code[e] = i < n ? codes[i] : ~0ull;
        const float v = unrank(~(uint32_t)(code[e] >> 32));
        at[e] = i < n ? bin.bin(bin.depth(v)) : kBins;
        before[e] = 0;
        rank[e] = 0;
        if (i < n && at[e] < rank_bin) atomicAdd(&n_early, 1);
      }
      for (int j = 0; j < n; ++j) {
        const uint64_t other = codes[j], m = parts[j];
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (e * kThreads < n && other < code[e]) before[e] += m, ++rank[e];
      }
      __syncthreads();
      // the top-k cut, and the listed mass up to it (all, without one)
      const bool cut_k = r.k && rank_bin < kBins;
      const int want = cut_k ? n_early + r.k - (int)w.before_rank - 1 : n - 1;
#pragma unroll
      for (int e = 0; e < kEach; ++e)
        if (e * kThreads + (int)threadIdx.x < n && rank[e] == want)
          found[0] = code[e], found[1] = before[e] + parts[e * kThreads + threadIdx.x];
      __syncthreads();
      cut = found[0];
      if (r.p < 1.f) {
        const uint64_t reach = reach_of(r.p, ahead + between + found[1]);
        __syncthreads();
        if (threadIdx.x == 0) found[0] = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e)
          if (e * kThreads + (int)threadIdx.x < n && code[e] <= cut &&
              ahead + (at[e] > high ? between : 0) + before[e] < reach)
            atomicMax((unsigned long long *)&found[0], (unsigned long long)code[e]);
        __syncthreads();
        cut = found[0];
      }
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = e * kThreads + threadIdx.x;
        if (i >= n) break;
        const uint64_t m = kept(unrank(~(uint32_t)(code[e] >> 32)), (int)(uint32_t)code[e], cut);
        if (m) atomicAdd((unsigned long long *)&in_slice[(uint32_t)code[e] / len], (unsigned long long)m);
      }
    }
  } else {
    if (r.k) cut = select_row<Z>(z, V, weigh, (uint64_t)r.k, false, cut, hist, scratch, found);
    if (r.p < 1.f) {
      uint64_t mass = 0;
      for (int i = threadIdx.x; i < V; i += kThreads) {
        const float x = logit<Z>(z, i);
        if (code_of(rank_key(x), i) <= cut) mass += weigh.units(x);
      }
      mass = wave_sum(mass);
      if (lane == 0) scratch[wave] = mass;
      __syncthreads();
      mass = 0;
      for (int i = 0; i < kWaves; ++i) mass += scratch[i];
      __syncthreads();
      cut = select_row<Z>(z, V, weigh, reach_of(r.p, mass), true, cut, hist, scratch, found);
    }
    for (int s = wave; s < kMaxSlices; s += kWaves) {
      const int lo = min(V, s * len), hi = s < slices ? min(V, lo + len) : lo;
      uint64_t mass = 0;
      for (int i = lo + lane; i < hi; i += 64) mass += kept(logit<Z>(z, i), i, cut);
      mass = wave_sum(mass);
      if (lane == 0) in_slice[s] = mass;
    }
  }
  __syncthreads();

  // the draw, the slice it falls into, the wave's run of the slice, the element
  constexpr int kPer = kMaxSlices / 64;
  uint64_t up = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) up += in_slice[lane * kPer + i];
  const uint64_t own = up;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t v = __shfl_up((unsigned long long)up, o);
    if (lane >= o) up += v;
  }
  const uint64_t mass = __shfl((unsigned long long)up, 63);
  const float u = a.u[row];
  const double want = (double)u * (double)mass;
  const uint64_t target = !(want > 0.0) ? 0 : want >= (double)mass ? mass - 1 : min(mass - 1, (uint64_t)want);
  const int at = max(0, __ffsll((unsigned long long)__ballot(target < up)) - 1);
  uint64_t before = __shfl((unsigned long long)(up - own), at);
  int slice = at * kPer;
  for (int i = 1; i < kPer && target >= before + in_slice[slice]; ++i) before += in_slice[slice++];
  const int begin = min(V, slice * len), end = min(V, begin + len);
  const int run = (end - begin + kWaves - 1) / kWaves, lo = min(end, begin + wave * run), hi = min(end, lo + run);
  uint64_t mine = 0;
  for (int i = lo + lane; i < hi; i += 64) mine += kept(logit<Z>(z, i), i, cut);
  mine = wave_sum(mine);
  __syncthreads();
  if (lane == 0) scratch[wave] = mine;
  __syncthreads();
  for (int i = 0; i < wave; ++i) before += scratch[i];
  if (target < before || target >= before + mine) return;
  for (int base = lo; base < hi; base += 64) {
    const int i = base + lane;
    const uint64_t m = i < hi ? kept(logit<Z>(z, i), i, cut) : 0;
    uint64_t sum = m;
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t v = __shfl_up((unsigned long long)sum, o);
      if (lane >= o) sum += v;
    }
    if (m && target >= before + sum - m && target < before + sum) {
      a.token[row] = i;
      if (a.prob) a.prob[row] = (float)((double)m / (double)mass);
    }
    before += __shfl((unsigned long long)sum, 63);
    if (target < before) return;
  }
}

// Blocks for a row's passes: about 1024 over all rows, each wave with at least 256 elements.
void split_row(int rows, int vocab, int *blocks, int *len) {
  int n = (1024 + rows - 1) / rows;
  const int most = (vocab + 256 * kSliceWaves - 1) / (256 * kSliceWaves);
  n = n > kMaxBlocks ? kMaxBlocks : n;
  *blocks = n > most ? most : n;
  *len = (vocab + *blocks * kSliceWaves - 1) / (*blocks * kSliceWaves);
}

template <class Z>
hipError_t launch(const SampleArgs &a, hipStream_t s) {
  int shift = 50, blocks, len;
  while ((int64_t)1 << (62 - shift) < a.vocab) --shift;
  split_row(a.rows, a.vocab, &blocks, &len);
  const dim3 grid(blocks, a.rows);
  void *first[] = {const_cast<SampleArgs *>(&a), &len}, *then[] = {const_cast<SampleArgs *>(&a), &len, &shift};
  void *last[] = {const_cast<SampleArgs *>(&a), &blocks, &len, &shift};
  hipError_t e = hipLaunchKernel((const void *)largest_kernel<Z>, grid, dim3(kSliceThreads), first, 0, s);
  if (e == hipSuccess && (a.top_k || a.top_p))
    e = hipLaunchKernel((const void *)bins_kernel<Z>, dim3((blocks * kSliceWaves + kWaves - 1) / kWaves, a.rows),
                        dim3(kThreads), last, 0, s);
  if (e == hipSuccess) e = hipLaunchKernel((const void *)collect_kernel<Z>, grid, dim3(kSliceThreads), then, 0, s);
  if (e == hipSuccess) e = hipLaunchKernel((const void *)draw_kernel<Z>, dim3(a.rows), dim3(kThreads), last, 0, s);
  return e;
}

}  // namespace

size_t sample_work_bytes(int rows) { return (size_t)rows * sizeof(RowWork); }

hipError_t launch_sample(const SampleArgs &a, int type, hipStream_t s) {
  return type == 0 ? launch<float>(a, s) : type == 1 ? launch<__bf16>(a, s) : launch<_Float16>(a, s);
}

}  // namespace moecache
