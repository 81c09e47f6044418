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
// A row is never sorted.  Its elements are counted and weighed into 2048 bins of depth below the largest
// logit, coarsely (32-bit exponentials); that tells which bin or two hold the top-k and the top-p cut.
// Then one exact pass sums the weights before those bins by slice of the row and lists the bins' own
// elements, some tens; these are sorted, which gives the cut; and the draw finds its slice, and in
// it the element.  Bound by four passes in a chain, none of them near the rate of memory, short rows by
// the launches.  Measured: 64 rows of 152001 fp32 logits, every row with settings of its own, 8.3 + 13.0 +
// 18.1 + 9.5 us (one read of the logits: 8.3); one row 3.9 + 5.2 + 7.7 + 7.8; 320 rows of 32003 bf16 9.6 + 12.8 +
// 23.9 + 11.8.  Of the exact pass's 18.1 (23.9) us 4 (4) are the launch and the row's settings, 3 (5) the bins and the
// cuts in them, which every block of a row finds for itself, 11 (14.5) the logits: their places among the bins, and
// 64-bit exponentials of 21 instructions for those not behind a top-k cut or below min_p (of all logits, with no
// cuts to look for, 10 in either case; the instructions alone, at the card's rate, 5 for the 64 rows).
#include <hip/hip_runtime.h>

#include <cstdint>

#include "serve.h"

namespace moecache {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;  // of the draw, a block per row
constexpr int kSliceThreads = 256;                      // of the passes over slices of a row
constexpr int kSliceWaves = kSliceThreads / 64;
constexpr int kMaxBlocks = 64;                          // of a row's passes; its slices are their waves
constexpr int kMaxSlices = kMaxBlocks * kSliceWaves;
constexpr int kBins = 2048;
constexpr int kCandidates = 4096;
constexpr int kOwn = 512;  // of them, a block's, before it hands them over one by one

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

// exp((z - top) / T) in units of 2^-shift, for a finite top; a row's masses are sums of these, rounded to
// whole units.
struct Weigh {
  double top;      // the row's largest logit
  double scale;    // log2(e) / T
  double deepest;  // of z - top: 2^-900
  double magic;    // 1.5 * 2^52 + shift: a sum with it is rounded to whole numbers, and holds them below
  double c[11];    // of 2^f
  __device__ Weigh(float top_, float T_, int shift) : Weigh((double)top_, fmin((double)T_, 1e300), shift) {}
  __device__ Weigh(double top_, double T, int shift)  // a finite T: z - top may not be
      : top(top_), scale(1.4426950408889634 / T), deepest(T * (-900.0 * 0.69314718055994531)),
        magic(0x1.8p52 + shift),
        // the polynomial of degree 10 with the least largest relative error on |f| <= 1/2 (2^-52), by Remez' exchange
        c{1.0, 0.6931471805599498, 0.24022650695908773, 0.05550410866445366, 0.009618129108031203,
          0.0013333558229309474, 0.00015403529966033974, 1.5252657716476882e-05, 1.321566021119544e-06,
          1.0208609179389605e-07, 7.037746430390509e-09} {
#pragma unroll
    for (int k = 0; k < 11; ++k) asm("" : "+s"(c[k]));  // in scalar registers, which an fma takes as they are
  }
  // With y = (z - top) / T log2(e) = n + f, n whole, |f| <= 1/2: 2^y = 2^n 2^f.  0 for NaN and -inf, but for
  // a rounding (the maximum of a NaN and a number is the number).
  __device__ __forceinline__ double operator()(float z) const {
    const double d = fmax((double)z - top, deepest), t = fma(d, scale, magic);
    const double f = fma(d, scale, magic - t), f2 = f * f;
    // odd and even powers apart: two chains of half the length
    double even = c[10], odd = c[9];
#pragma unroll
    for (int k = 8; k >= 0; k -= 2) {
      even = fma(even, f2, c[k]);
      if (k) odd = fma(odd, f2, c[k - 1]);
    }
    const double e = fma(odd, f, even);
    // n + shift, the low bits of t, to the exponent
    const uint64_t bits = __builtin_bit_cast(uint64_t, e) + (__builtin_bit_cast(uint64_t, t) << 52);
    return __builtin_bit_cast(double, bits);
  }
  __device__ __forceinline__ uint64_t units(float z) const { return (uint64_t)rint((*this)(z)); }
};

// A row's settings, and its largest logit.
struct Row {
  float top, T, p, least, u;
  int first, k;
  bool none, greedy;  // nothing but -inf and NaN; the first largest is the answer
  bool wild;          // +inf among the logits: all weight is theirs
  __device__ Row(const SampleArgs &a, int row, uint64_t best) {
    first = (int)~(uint32_t)best;
    top = unrank((uint32_t)(best >> 32));
    T = a.temperature ? a.temperature[row] : 1.f;
    p = a.top_p ? a.top_p[row] : 1.f;
    k = a.top_k ? a.top_k[row] : 0;
    if (k <= 0 || k >= a.vocab) k = 0;
    least = a.min_p ? a.min_p[row] : 0.f;
    u = a.u[row];
    if (least > 1.f) least = 1.f;
    none = !(top > -__builtin_inff());
    greedy = !(T > 0.f);
    wild = top == __builtin_inff();
  }
  __device__ __forceinline__ bool ranked() const { return k || p < 1.f; }
  __device__ __forceinline__ Weigh weigh(int shift) const {
    return Weigh(top, T, shift);
  }
};

// Bins of (top - z) / T, rising with falling logits; weights past the last are below half of 2^-shift.
struct Binning {
  float half, scale, depth;  // of a place: its (top - z) / T
  __device__ Binning(const Row &r, int shift) : half(0.5f * r.top) {
    const float limit = (float)(shift + 1) * 0.69314718f + 0.01f;
    scale = fminf(2.f / r.T * (kBins / limit), 3.4e38f);  // finite: 0 times it is 0
    depth = limit / kBins;
  }
  // Where a logit lies among the bins: in bin (int)place if that is below kBins (a NaN is not).  Of
  // halves: two logits may be further apart than the largest float.
  __device__ __forceinline__ float place(float z) const {
#pragma clang fp contract(off)  // the top's own half less its half is 0
    return (half - 0.5f * z) * scale;
  }
};

// The largest logit of elements lo .. hi - 1, one wave's: its rank key, then its first index.
template <class Z>
__device__ __forceinline__ uint64_t largest_of(const void *z, int lo, int hi) {
  uint64_t best = 0;
  for_each<Z>(z, lo, hi, [&](const float (&v)[kVec<Z>], int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kVec<Z>; ++j) best = max(best, (uint64_t)rank_key(v[j]) << 32 | (uint32_t)~(i + j));
  });
  return wave_max(best);
}

// Elements (for top-k) and mass (for top-p) by bin of elements lo .. hi - 1, one wave's.  The masses here
// are of 32-bit exponentials, rounded to 2^-31: they only choose which bins need ranking, with their
// errors allowed for (least_of, most_of).
template <class Z>
__device__ __forceinline__ void bin_elements(const void *z, int lo, int hi, const Row &r, int shift, uint64_t *mass,
                                             uint32_t *count) {
  const Binning bin(r, shift);
  const bool by_mass = r.p < 1.f, by_count = r.k != 0;
  const float exponent = bin.depth * -1.44269504f;
  for_each<Z>(z, lo, hi, [&](const float (&v)[kVec<Z>], int) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kVec<Z>; ++j) {
      const float f = bin.place(v[j]);
      if (!(f < kBins)) continue;
      if (by_mass) {
        const uint32_t m = (uint32_t)rintf(__builtin_amdgcn_exp2f(f * exponent) * 0x1p31f);
        atomicAdd((unsigned long long *)&mass[(int)f], (unsigned long long)m);
      }
      if (by_count) atomicAdd(&count[(int)f], 1u);
    }
  });
}

// What the exact mass, in 2^-31, of elements whose binned masses sum to m lies between, as good as surely:
// the exponentials' arguments are off by a few parts in 2^24 of up to 44 (most of the mass is at a few), the
// roundings of 2^20 elements add up to some 500 units at random.  Where it does not, the exact sums show
// that the cut is not in the list, and the row is gone over.
__device__ __forceinline__ double least_of(uint64_t m) { return (double)m * (1.0 - 0x1p-18) - 4096; }
__device__ __forceinline__ double most_of(uint64_t m) { return (double)m * (1.0 + 0x1p-18) + 4096; }

// Which bins may hold a cut: bins low .. high and rank_bin need their elements ranked; bins past
// `last` hold nothing that is kept or counts.
struct Cuts {
  int low, high, rank_bin;  // all kBins: no cut; rank_bin kBins: no top-k cut
  uint32_t before_rank;     // elements in bins before rank_bin
};
// By a block of N threads, from the bins threadIdx.x * kBins / N on in each; uniform over the block.
template <int N>
__device__ __forceinline__ Cuts find_cuts(const uint64_t (&mass)[kBins / N], const uint32_t (&count)[kBins / N],
                                          const Row &r) {
  constexpr int kPer = kBins / N;
  __shared__ uint64_t masses[N / 64];
  __shared__ uint32_t counts[N / 64], before_rank;
  __shared__ int cuts[3];
  __shared__ double reach[2];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
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
  if (lane == 63) masses[wave] = up, counts[wave] = up_n;
  if (threadIdx.x == 0) cuts[0] = 0, cuts[1] = kBins - 1, cuts[2] = kBins, before_rank = 0;
  __syncthreads();
  before = up - before;
  before_n = up_n - before_n;
  uint64_t all = 0;
  uint32_t all_n = 0;
  for (int i = 0; i < N / 64; ++i) {
    if (i < wave) before += masses[i], before_n += counts[i];
    all += masses[i];
    all_n += counts[i];
  }
  const bool cut_k = r.k && (uint32_t)r.k < all_n;  // else top-k cuts nothing but weights of 0
  if (threadIdx.x == 0 && !cut_k) reach[0] = least_of(all), reach[1] = most_of(all);
  if (cut_k) {
    uint64_t at = before;
    uint32_t n = before_n;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if (n < (uint32_t)r.k && n + count[i] >= (uint32_t)r.k) {  // in one thread's one bin
        cuts[2] = threadIdx.x * kPer + i;
        reach[0] = least_of(at), reach[1] = most_of(at + mass[i]);
        before_rank = n;
      }
      at += mass[i];
      n += count[i];
    }
  }
  __syncthreads();
  Cuts c{cuts[2], cuts[2], cuts[2], before_rank};
  if (r.p < 1.f) {
    // what top-p reaches for lies between these
    const double least = (double)r.p * reach[0], most = (double)r.p * reach[1] + 1.0;
    uint64_t at = before;
    int begun = 0, ended = kBins - 1;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = threadIdx.x * kPer + i;
      // the last bin that begins before that, the first that ends past it
      if (most_of(at) < least) begun = b;
      at += mass[i];
      if (least_of(at) >= most) ended = min(ended, b);
    }
    for (int o = 32; o; o >>= 1) begun = max(begun, __shfl_xor(begun, o)), ended = min(ended, __shfl_xor(ended, o));
    if (lane == 0) atomicMax(&cuts[0], begun), atomicMin(&cuts[1], ended);
    __syncthreads();
    c.high = min(cuts[1], c.rank_bin);
    c.low = min(cuts[0], c.high);
  }
  return c;
}

// Exact masses of elements lo .. hi - 1, one wave's: of all that may be kept (up to the last bin
// with a cut; all, without a filter by rank), of those in bins before the list's, of those of them that min_p
// keeps.  push(code) gets the elements of the bins to be ranked.
struct Masses {
  uint64_t all, ahead, kept;
};
template <class Z, class Push>
__device__ __forceinline__ Masses weigh_elements(const void *z, int lo, int hi, const Row &r, const Cuts &c, int shift,
                                                 Push push) {
  const Binning bin(r, shift);
  const Weigh weigh = r.weigh(shift);
  const double least = (double)r.least * (double)(1ull << shift);
  const float low_start = (float)c.low, high_end = (float)(c.high + 1), rank_start = (float)c.rank_bin,
              rank_end = (float)(c.rank_bin + 1);
  const bool ranked = c.low < kBins, cut_k = c.rank_bin < kBins;
  // past this place nothing asks for a weight; where nothing is cut by rank, only the kept mass does
  float last_end = (float)min(c.rank_bin + 1, kBins);
  if (!ranked && r.least > 0.f) last_end = fminf(last_end, -logf(r.least) / bin.depth * 1.0001f + 1.f);
  const bool one_sum = !ranked && !(least > 0.0);
  // whole units, exact in a double up to 2^53: so many sums at a time
  Masses m{0, 0, 0};
  double all = 0, ahead = 0, kept = 0;
  int room = 1 << (53 - shift);
  auto flush = [&]() __attribute__((always_inline)) {
    m.all += (uint64_t)all, m.ahead += (uint64_t)ahead, m.kept += (uint64_t)kept;
    all = ahead = kept = 0;
    room = 1 << (53 - shift);
  };
  auto four = [&](const float *v, int i) __attribute__((always_inline)) {
    const float first = bin.place(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])));
    // with a top-k cut few of a row's elements matter: most calls end here
    if (!__any(first < last_end)) return;
    // without a branch between them, so that one element's arithmetic fills another's waits
    double x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = weigh(v[j]);
    if (one_sum || (!cut_k && !__any(first < high_end))) {
      // all behind the cut, as most are under top-p alone: one sum (past the last bin all round to 0)
#pragma unroll
      for (int j = 0; j < 4; ++j) all += rint(x[j]);
    } else {
      bool any = false;
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        f[j] = bin.place(v[j]);
        const double n = f[j] < last_end ? rint(x[j]) : 0.0, early = f[j] < low_start ? n : 0.0;
        all += n;
        ahead += early;
        kept += x[j] < least ? 0.0 : early;
        any |= (f[j] >= low_start && f[j] < high_end) || (f[j] >= rank_start && f[j] < rank_end);
      }
      if (any) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (f[j] < kBins && ((f[j] >= low_start && f[j] < high_end) || (f[j] >= rank_start && f[j] < rank_end)))
            push(code_of(rank_key(v[j]), i + j));
      }
    }
  };
  for_each<Z>(z, lo, hi, [&](const float (&v)[kVec<Z>], int i) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < kVec<Z>; j += 4) four(v + j, i + j);
    if ((room -= kVec<Z>) < kVec<Z>) flush();
  });
  flush();
  if (one_sum) m.ahead = m.kept = m.all;
  return Masses{wave_sum(m.all), wave_sum(m.ahead), wave_sum(m.kept)};
}

// A row's part of the workspace.
struct RowWork {
  uint64_t best[kMaxBlocks];   // blocks' largest logit: rank key, then the smallest index
  Masses sums[kMaxSlices];
  uint64_t mass[kBins];        // binned, in 2^-31
  uint32_t count[kBins];
  uint64_t list[kCandidates];  // codes of the elements that need ranking
  Cuts cuts;
  int32_t n_list, pad;         // elements that need ranking, in the list or not
};

// The largest of the blocks' bests; every wave of the block for itself.
__device__ __forceinline__ uint64_t row_best(const RowWork &w, int blocks) {
  const int lane = threadIdx.x % 64;
  return wave_max(lane < blocks ? w.best[lane] : 0);
}

// The cut as a code, found by going over the whole row: for rows with more elements in the bins
// that hold a cut than the list takes (few distinct logits: a call over a row of 152001 equal ones takes 0.83 ms, over
// 64 such rows 1.03; over bf16 logits of 12 to 28, a sixteenth to an eighth apart, 0.09 and 0.13).  A total in falling order (of ones,
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

// The running mass that the drawn element is the first to exceed.
__device__ __forceinline__ uint64_t target_of(float u, uint64_t mass) {
  const double want = (double)u * (double)mass;
  return !(want > 0.0) ? 0 : want >= (double)mass ? mass - 1 : min(mass - 1, (uint64_t)want);
}

// What top-p reaches for, of a mass: at least 1, so that the first element stays.
__device__ __forceinline__ uint64_t reach_of(float p, uint64_t mass) {
  const double part = ceil((double)p * (double)mass);
  return part < 1.0 ? 1 : min(mass, (uint64_t)part);
}

// What the last step of a row works on, in LDS.
struct Last {
  uint64_t codes[kCandidates];  // the listed elements
  union {
    uint64_t before[kCandidates];  // sorted: the listed mass before each
    struct {                       // until then: a row's bins
      uint64_t mass[kBins];
      uint32_t count[kBins];
    };
  };
  uint64_t hist[256], scratch[kWaves], found[2], in_slice[kMaxSlices];
  int n, n_early, at;
};

// Sorts n codes, a power of two, by the whole block (a bitonic network: 78 steps for 4096).
__device__ __forceinline__ void sort_codes(uint64_t *codes, int n) {
  for (int k = 2; k <= n; k *= 2)
    for (int j = k / 2; j; j /= 2) {
      for (int i = threadIdx.x; i < n / 2; i += kThreads) {
        const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
        const uint64_t x = codes[lo], y = codes[hi];
        if ((x > y) == ((lo & k) == 0)) codes[lo] = y, codes[hi] = x;
      }
      __syncthreads();
    }
}

// The last step, a block per row: ranks the listed elements, which gives the cut, then finds the slice
// (of `len` elements, its kept mass but for the listed ones in in_slice) in which the draw falls, and
// the element in it.  n elements are to be listed; where they are more than the list takes, or the cut turns
// out not to be among them, the row is gone over instead.  all, ahead: exact masses of what may be kept, and of what is before the list.
template <class Z, int kHalves>
__device__ __forceinline__ void rank_and_draw(const SampleArgs &a, int row, const void *z, const Row &r, const Cuts &c,
                                              int n, uint64_t all, uint64_t ahead, int slices, int len, int shift,
                                              Last &s) {
  const int V = a.vocab, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const Weigh weigh = r.weigh(shift);
  const double least = (double)r.least * (double)(1ull << shift);
  auto kept = [&](float v, int i, uint64_t cut) -> uint64_t {
    if (code_of(rank_key(v), i) > cut) return 0;
    const double x = weigh(v);
    return x < least ? 0 : (uint64_t)rint(x);
  };
  uint64_t cut = ~0ull;  // code of the last element that the filters by rank keep
  bool known = c.low == kBins;  // nothing is cut by rank
  if (!known && n > 0 && n <= kCandidates) {
    // the listed elements in falling order, and the listed mass before each
    int size = 1;
    while (size < n) size *= 2;
    for (int i = n + threadIdx.x; i < size; i += kThreads) s.codes[i] = ~0ull;
    if (threadIdx.x == 0) s.n_early = 0, s.at = -1;
    __syncthreads();
    sort_codes(s.codes, size);
    const Binning bin(r, shift);
    constexpr int kEach = kCandidates / kThreads;
    const int each = (size + kThreads - 1) / kThreads, from = threadIdx.x * each;
    uint64_t mass[kEach], up = 0;
    int early = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      mass[e] = 0;
      if (e >= each || from + e >= n) continue;
      const float v = unrank(~(uint32_t)(s.codes[from + e] >> 32));
      mass[e] = weigh.units(v);
      up += mass[e];
      early += (int)bin.place(v) < c.rank_bin;
    }
    if (early) atomicAdd(&s.n_early, early);
    uint64_t at = up;
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t v = __shfl_up((unsigned long long)up, o);
      if (lane >= o) up += v;
    }
    if (lane == 63) s.scratch[wave] = up;
    __syncthreads();
    at = up - at;
    uint64_t listed = 0;
    for (int i = 0; i < kWaves; ++i) {
      if (i < wave) at += s.scratch[i];
      listed += s.scratch[i];
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e)
      if (e < each && from + e < n) {
        s.before[from + e] = at;
        at += mass[e];
      }
    __syncthreads();
    // the top-k cut (the last listed element, without one), then the top-p cut
    const auto through = [&](int i) { return i + 1 < n ? s.before[i + 1] : listed; };
    int last = r.k && c.rank_bin < kBins ? s.n_early + r.k - (int)c.before_rank - 1 : n - 1;
    last = min(max(last, 0), n - 1);
    known = true;
    if (r.p < 1.f) {
      const uint64_t reach = reach_of(r.p, all - (listed - through(last)));
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = from + e;
        if (e < each && i <= last && ahead + s.before[i] < reach &&
            (int)bin.place(unrank(~(uint32_t)(s.codes[i] >> 32))) <= c.high)
          atomicMax(&s.at, i);
      }
      __syncthreads();
      known = s.at >= 0 && ahead + through(max(0, s.at)) >= reach;
      last = max(0, s.at);
    }
    if (known) {
      cut = s.codes[last];
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = from + e;
        if (e >= each || i > last) continue;
        const uint64_t code = s.codes[i], m = kept(unrank(~(uint32_t)(code >> 32)), (int)(uint32_t)code, cut);
        if (m) atomicAdd((unsigned long long *)&s.in_slice[(uint32_t)code / len], (unsigned long long)m);
      }
    }
  }
  if (!known) {
    if (r.k) cut = select_row<Z>(z, V, weigh, (uint64_t)r.k, false, cut, s.hist, s.scratch, s.found);
    if (r.p < 1.f) {
      uint64_t mass = 0;
      for (int i = threadIdx.x; i < V; i += kThreads) {
        const float x = logit<Z>(z, i);
        if (code_of(rank_key(x), i) <= cut) mass += weigh.units(x);
      }
      mass = wave_sum(mass);
      if (lane == 0) s.scratch[wave] = mass;
      __syncthreads();
      mass = 0;
      for (int i = 0; i < kWaves; ++i) mass += s.scratch[i];
      __syncthreads();
      cut = select_row<Z>(z, V, weigh, reach_of(r.p, mass), true, cut, s.hist, s.scratch, s.found);
    }
    for (int i = wave; i < kMaxSlices; i += kWaves) {
      const int lo = min(V, i * len), hi = i < slices ? min(V, lo + len) : lo;
      uint64_t mass = 0;
      for (int j = lo + lane; j < hi; j += 64) mass += kept(logit<Z>(z, j), j, cut);
      mass = wave_sum(mass);
      if (lane == 0) s.in_slice[i] = mass;
    }
  }
  __syncthreads();

  // the draw, the slice it falls into, the wave's run of the slice, the element
  constexpr int kPer = kMaxSlices / 64;
  uint64_t up = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) up += s.in_slice[lane * kPer + i];
  const uint64_t own = up;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t v = __shfl_up((unsigned long long)up, o);
    if (lane >= o) up += v;
  }
  const uint64_t mass = __shfl((unsigned long long)up, 63);
  const uint64_t target = target_of(r.u, mass);
  const int at = max(0, __ffsll((unsigned long long)__ballot(target < up)) - 1);
  uint64_t before = __shfl((unsigned long long)(up - own), at);
  int slice = at * kPer;
  for (int i = 1; i < kPer && target >= before + s.in_slice[slice]; ++i) before += s.in_slice[slice++];
  const int begin = min(V, slice * len), end = min(V, begin + len);
  const int run = (end - begin + kWaves - 1) / kWaves, lo = min(end, begin + wave * run), hi = min(end, lo + run);
  // steps of kHalves times four neighbours to a lane, asked for together; most runs end within one
  constexpr int kEach = 4, kHalf = 64 * kEach, kStep = kHalves * kHalf;
  uint64_t m[kHalves][kEach] = {}, mine = 0;
  auto take = [&](int base) __attribute__((always_inline)) {
    float v[kHalves][kEach];
    uint64_t sum = 0;
#pragma unroll
    for (int e = 0; e < kHalves * kEach; ++e)
      v[e / kEach][e % kEach] = logit<Z>(z, min(base + e / kEach * kHalf + lane * kEach + e % kEach, hi - 1));
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) m[h][e] = 0;
      if (base + h * kHalf < hi) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
          const int i = base + h * kHalf + lane * kEach + e;
          sum += m[h][e] = i < hi ? kept(v[h][e], i, cut) : 0;
        }
      }
    }
    return sum;
  };
  for (int base = lo; base < hi; base += kStep) mine += take(base);
  mine = wave_sum(mine);
  if (lane == 0) s.scratch[wave] = mine;
  __syncthreads();
  for (int i = 0; i < wave; ++i) before += s.scratch[i];
  if (target < before || target >= before + mine) return;
  const bool again = hi - lo > kStep;  // else m is the run's
  for (int base = lo; base < hi; base += kStep) {
    if (again) take(base);
#pragma unroll
    for (int h = 0; h < kHalves; ++h) {
      uint64_t sum = 0;
#pragma unroll
      for (int e = 0; e < kEach; ++e) sum += m[h][e];
      const uint64_t own = sum;
      for (int o = 1; o < 64; o <<= 1) {
        const uint64_t v = __shfl_up((unsigned long long)sum, o);
        if (lane >= o) sum += v;
      }
      uint64_t at = before + sum - own;
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        if (target >= at && target < at + m[h][e]) {
          a.token[row] = base + h * kHalf + lane * kEach + e;
          if (a.prob) a.prob[row] = (float)((double)m[h][e] / (double)mass);
        }
        at += m[h][e];
      }
      before += __shfl((unsigned long long)sum, 63);
      if (target < before) return;
    }
  }
}

// Rows that need no weights: nothing to choose from; the first largest is chosen; infinite logits
// share all of the mass evenly: the filters keep the first so many of them.  By the whole block.
template <class Z>
__device__ __forceinline__ bool settled(const SampleArgs &a, int row, const void *z, const Row &r, uint64_t *scratch) {
  if (!r.none && !r.greedy && !r.wild) return false;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, V = a.vocab;
  int token = r.none ? -1 : r.first;
  float prob = r.none ? 0.f : 1.f;
  if (r.wild && !r.greedy) {
    uint64_t n = 0;
    for (int i = threadIdx.x; i < V; i += kThreads) n += logit<Z>(z, i) == r.top;
    n = wave_sum(n);
    __syncthreads();
    if (lane == 0) scratch[wave] = n;
    __syncthreads();
    n = 0;
    for (int i = 0; i < kWaves; ++i) n += scratch[i];
    if (r.k) n = min(n, (uint64_t)r.k);
    if (r.p < 1.f) n = reach_of(r.p, n);
    const uint64_t target = target_of(r.u, n);
    uint64_t seen = 0;
    for (int base = 0; base < V; base += kThreads) {
      const int i = base + threadIdx.x;
      const bool hit = i < V && logit<Z>(z, i) == r.top;
      const uint64_t mask = __ballot(hit);
      __syncthreads();
      if (lane == 0) scratch[wave] = __popcll(mask);
      __syncthreads();
      uint64_t before = seen + __popcll(mask & ((1ull << lane) - 1));
      for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += scratch[w];
        seen += scratch[w];
      }
      if (hit && before == target) {
        a.token[row] = i;
        if (a.prob) a.prob[row] = (float)(1.0 / (double)n);
      }
      if (seen > target) break;
    }
    return true;
  }
  if (threadIdx.x == 0) {
    a.token[row] = token;
    if (a.prob) a.prob[row] = prob;
  }
  return true;
}

// ---------------------------------------------------------------------------------------------
// Rows of up to kWhole elements: a block per row takes all steps in one launch (each goes over the
// row again, from L2), a quarter of its wave's share at a time.  320 rows of 8000: 31.5 us, by launches
// over slices 40.6; 320 of 16000 40.5 and 45.9, one of 16000 22.1 and 21.4.
// ---------------------------------------------------------------------------------------------
constexpr int kWhole = 16384, kRowSlices = 4 * kWaves;

template <class Z>
__global__ __launch_bounds__(kThreads, 4) void row_kernel(SampleArgs a, int shift) {
  __shared__ Last s;
  const int row = blockIdx.x, V = a.vocab, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const void *z = (const Z *)a.logits + (int64_t)row * a.stride;
  const int len = (V + kRowSlices - 1) / kRowSlices;
  const int lo = min(V, 4 * wave * len), hi = min(V, lo + 4 * len);
  uint64_t best = largest_of<Z>(z, lo, hi);
  if (lane == 0) s.scratch[wave] = best;
  for (int i = threadIdx.x; i < kBins; i += kThreads) s.mass[i] = 0, s.count[i] = 0;
  if (threadIdx.x < kMaxSlices) s.in_slice[threadIdx.x] = 0;
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  for (int i = 0; i < kWaves; ++i) best = max(best, s.scratch[i]);
  const Row r(a, row, best);
  if (settled<Z>(a, row, z, r, s.scratch)) return;
  Cuts c{kBins, kBins, kBins, 0};
  if (r.ranked()) {
    bin_elements<Z>(z, lo, hi, r, shift, s.mass, s.count);
    __syncthreads();
    uint64_t mass[kBins / kThreads];
    uint32_t count[kBins / kThreads];
#pragma unroll
    for (int i = 0; i < kBins / kThreads; ++i) {
      mass[i] = s.mass[threadIdx.x * (kBins / kThreads) + i];
      count[i] = s.count[threadIdx.x * (kBins / kThreads) + i];
    }
    c = find_cuts<kThreads>(mass, count, r);
  }
  __syncthreads();  // `scratch` and the bins have been read
  uint64_t all = 0, ahead = 0;
#pragma unroll 1
  for (int i = 0; i < 4; ++i) {
    const int begin = min(hi, lo + i * len);
    const Masses m = weigh_elements<Z>(z, begin, min(hi, begin + len), r, c, shift,
                                       [&](uint64_t code) __attribute__((always_inline)) {
                                         const int at = atomicAdd(&s.n, 1);
                                         if (at < kCandidates) s.codes[at] = code;
                                       });
    all += m.all, ahead += m.ahead;
    if (lane == 0) s.in_slice[4 * wave + i] = m.kept;
  }
  if (lane == 0) s.scratch[wave] = all, s.hist[wave] = ahead;
  __syncthreads();
  all = ahead = 0;
  for (int i = 0; i < kWaves; ++i) all += s.scratch[i], ahead += s.hist[i];
  const int n = s.n;
  __syncthreads();
  rank_and_draw<Z, 1>(a, row, z, r, c, n, all, ahead, kRowSlices, len, shift, s);
}

// ---------------------------------------------------------------------------------------------
// Longer rows: slices of a row over several blocks, a launch per step.
// ---------------------------------------------------------------------------------------------
// Step 1, a wave per slice: the largest logit; the row's bins are cleared on the way.
template <class Z>
__global__ __launch_bounds__(kSliceThreads) void largest_kernel(SampleArgs a, int len) {
  RowWork &w = ((RowWork *)a.work)[blockIdx.y];
  const void *z = (const Z *)a.logits + (int64_t)blockIdx.y * a.stride;
  const int lo = min(a.vocab, (int)(blockIdx.x * kSliceWaves + threadIdx.x / 64) * len);
  for (int i = blockIdx.x * kSliceThreads + threadIdx.x; i < kBins; i += gridDim.x * kSliceThreads)
    w.mass[i] = 0, w.count[i] = 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) w.n_list = 0;
  __shared__ uint64_t scratch[kSliceWaves];
  uint64_t best = largest_of<Z>(z, lo, min(a.vocab, lo + len));
  if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = best;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < kSliceWaves; ++i) best = max(best, scratch[i]);
    w.best[blockIdx.x] = best;
  }
}

// Step 2, for rows with a filter by rank: the bins, kWaves slices to a block (each block adds its bins
// to the row's one by one).
template <class Z>
__global__ __launch_bounds__(kThreads) void bins_kernel(SampleArgs a, int blocks, int len, int shift) {
  RowWork &w = ((RowWork *)a.work)[blockIdx.y];
  const Row r(a, blockIdx.y, row_best(w, blocks));
  if (r.none || r.greedy || r.wild || !r.ranked()) return;
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  for (int i = threadIdx.x; i < kBins; i += kThreads) mass[i] = 0, count[i] = 0;
  __syncthreads();
  const void *z = (const Z *)a.logits + (int64_t)blockIdx.y * a.stride;
  const int lo = min(a.vocab, (int)(blockIdx.x * kWaves + threadIdx.x / 64) * len);
  bin_elements<Z>(z, lo, min(a.vocab, lo + len), r, shift, mass, count);
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) {
    if (mass[i]) atomicAdd((unsigned long long *)&w.mass[i], (unsigned long long)mass[i]);
    if (count[i]) atomicAdd(&w.count[i], count[i]);
  }
}

// Step 3: the cuts' bins (every block of a row finds them for itself), their elements into the row's
// list, each slice's exact masses.  Five waves a SIMD: 1280 blocks, as 320 rows have, run at once.
template <class Z>
__global__ __launch_bounds__(kSliceThreads, 5) void collect_kernel(SampleArgs a, int len, int shift) {
  RowWork &w = ((RowWork *)a.work)[blockIdx.y];
  const void *z = (const Z *)a.logits + (int64_t)blockIdx.y * a.stride;
  constexpr int kPer = kBins / kSliceThreads;
  uint64_t mass[kPer];  // asked for together with the row's settings
  uint32_t count[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    mass[i] = w.mass[threadIdx.x * kPer + i];
    count[i] = w.count[threadIdx.x * kPer + i];
  }
  const Row r(a, blockIdx.y, row_best(w, gridDim.x));
  if (r.none || r.greedy || r.wild) return;
  __shared__ uint64_t mine[kOwn];
  __shared__ int n_mine, place;
  if (threadIdx.x == 0) n_mine = 0;
  Cuts c{kBins, kBins, kBins, 0};
  if (r.ranked()) c = find_cuts<kSliceThreads>(mass, count, r);
  if (blockIdx.x == 0 && threadIdx.x == 0) w.cuts = c;
  __syncthreads();
  const int slice = blockIdx.x * kSliceWaves + threadIdx.x / 64, lo = min(a.vocab, slice * len);
  const Masses m = weigh_elements<Z>(z, lo, min(a.vocab, lo + len), r, c, shift,
                                     [&](uint64_t code) __attribute__((always_inline)) {
                                       const int at = atomicAdd(&n_mine, 1);
                                       if (at < kOwn) {
                                         mine[at] = code;
                                       } else {
                                         const int far = atomicAdd(&w.n_list, 1);
                                         if (far < kCandidates) w.list[far] = code;
                                       }
                                     });
  if (threadIdx.x % 64 == 0) w.sums[slice] = m;
  __syncthreads();
  if (threadIdx.x == 0 && n_mine) place = atomicAdd(&w.n_list, min(n_mine, kOwn));
  __syncthreads();
  for (int i = threadIdx.x; i < min(n_mine, kOwn); i += kSliceThreads)
    if (place + i < kCandidates) w.list[place + i] = mine[i];
}

// Step 4, a block per row.
template <class Z>
__global__ __launch_bounds__(kThreads) void draw_kernel(SampleArgs a, int blocks, int len, int shift) {
  __shared__ Last s;
  const int row = blockIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64, slices = blocks * kSliceWaves;
  const RowWork &w = ((const RowWork *)a.work)[row];
  const void *z = (const Z *)a.logits + (int64_t)row * a.stride;
  const uint64_t head = w.list[threadIdx.x];  // asked for before its length is known
  // and so are the rest; none of it is used where the row is settled
  const Masses m = (int)threadIdx.x < slices ? w.sums[threadIdx.x] : Masses{0, 0, 0};
  const Cuts c = w.cuts;
  const int n_list = w.n_list;
  const Row r(a, row, row_best(w, blocks));
  if (settled<Z>(a, row, z, r, s.scratch)) return;
  static_assert(kMaxSlices <= kThreads && kMaxSlices / 64 <= kWaves, "a thread per slice");
  if (threadIdx.x < kMaxSlices) {
    s.in_slice[threadIdx.x] = m.kept;
    const uint64_t all = wave_sum(m.all), ahead = wave_sum(m.ahead);
    if (lane == 0) s.scratch[wave] = all, s.hist[wave] = ahead;
  }
  const int n = r.ranked() ? n_list : 0;
  if ((int)threadIdx.x < n) s.codes[threadIdx.x] = head;
  for (int i = threadIdx.x + kThreads; i < min(n, kCandidates); i += kThreads) s.codes[i] = w.list[i];
  __syncthreads();
  uint64_t all = 0, ahead = 0;
#pragma unroll
  for (int i = 0; i < kMaxSlices / 64; ++i) all += s.scratch[i], ahead += s.hist[i];
  __syncthreads();
  rank_and_draw<Z, 2>(a, row, z, r, c, n, all, ahead, slices, len, shift, s);
}

// Blocks for a row's passes: 1024 or some more over all rows, each wave with at least 256 elements.
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
  if (a.vocab <= kWhole) {
    void *args[] = {const_cast<SampleArgs *>(&a), &shift};
    return hipLaunchKernel((const void *)row_kernel<Z>, dim3(a.rows), dim3(kThreads), args, 0, s);
  }
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

size_t sample_work_bytes(int rows, int vocab) { return vocab <= kWhole ? 0 : (size_t)rows * sizeof(RowWork); }

hipError_t launch_sample(const SampleArgs &a, int type, hipStream_t s) {
  return type == 0 ? launch<float>(a, s) : type == 1 ? launch<__bf16>(a, s) : launch<_Float16>(a, s);
}

}  // namespace moecache
