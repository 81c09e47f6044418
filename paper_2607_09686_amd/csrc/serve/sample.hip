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
// length: sums of integers do not depend on their order, so every split of a row over threads gives
// the same token, and two tokens' border is off by at most 2^(20 - s) of the largest weight.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "serve.h"

namespace moecache {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

template <class Z>
__device__ __forceinline__ float logit(const void *row, int i) {
  return (float)((const Z *)row)[i] + 0.f;  // -0 + 0 = 0: the two zeros rank alike
}
// Order of floats as unsigned integers; a NaN ranks last.
__device__ __forceinline__ uint32_t rank_key(float z) {
  const uint32_t b = __builtin_bit_cast(uint32_t, z);
  return z != z ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Weigh {
  float top;  // the row's largest logit
  double scale, unit;  // 1 / T, 2^s
  // exp((z - top) / T), 0 for NaN and -inf
  __device__ __forceinline__ double weight(float z) const {
    if (z == top) return 1.0;
    const double x = ((double)z - (double)top) * scale;
    return x > -64.0 ? exp(x) : 0.0;  // 2^-s > e^-64: nothing is lost, and NaN goes to 0
  }
  __device__ __forceinline__ uint64_t parts(double w) const { return (uint64_t)rint(w * unit); }
};

// Elements kept by rank: key above `key`, or equal to it at an index up to `last`.
struct Cut {
  uint32_t key;
  int last;
  __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= last); }
};

template <class T>
__device__ __forceinline__ T block_sum(T v, T *scratch) {
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  if (threadIdx.x % 64 == 0) scratch[threadIdx.x / 64] = v;
  __syncthreads();
  T sum = 0;
  for (int w = 0; w < kWaves; ++w) sum += scratch[w];
  __syncthreads();
  return sum;
}

// One row per block: the row is read once per step of the selection.
template <class Z>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(SampleArgs a, int shift) {
  __shared__ uint64_t hist[256];
  __shared__ uint64_t scratch[kWaves];
  __shared__ uint64_t found[2];
  const int row = blockIdx.x, V = a.vocab, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const void *z = (const Z *)a.logits + (int64_t)row * a.stride;

  // the largest logit and its first index
  uint64_t best = 0;
  for (int i = threadIdx.x; i < V; i += kThreads)
    best = max(best, (uint64_t)rank_key(logit<Z>(z, i)) << 32 | (uint32_t)~i);
  for (int o = 32; o; o >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, o));
  if (lane == 0) scratch[wave] = best;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) best = max(best, scratch[w]);
  __syncthreads();
  const int first = (int)~(uint32_t)best;
  const float top = logit<Z>(z, first), T = a.temperature ? a.temperature[row] : 1.f;
  const bool none = !(top > -__builtin_inff());  // nothing but -inf and NaN
  if (none || !(T > 0.f)) {
    if (threadIdx.x == 0) {
      a.token[row] = none ? -1 : first;
      if (a.prob) a.prob[row] = none ? 0.f : 1.f;
    }
    return;
  }
  const Weigh wt{top, 1.0 / (double)T, (double)(1ull << shift)};

  // the cut after the element at which a running total in falling order (of ones, or of
  // weights) first reaches `want`; want is at least 1 and at most the total over `in`
  auto select = [&](uint64_t want, bool weighted, Cut in) -> Cut {
    uint32_t key = 0;
    uint64_t above = 0;  // total over keys above the prefix's range
    for (int bits = 24; bits >= 0; bits -= 8) {
      for (int i = threadIdx.x; i < 256; i += kThreads) hist[i] = 0;
      __syncthreads();
      for (int i = threadIdx.x; i < V; i += kThreads) {
        const float x = logit<Z>(z, i);
        const uint32_t k = rank_key(x);
        if (!in.keeps(k, i) || (bits < 24 && k >> (bits + 8) != key >> (bits + 8))) continue;
        const uint64_t n = weighted ? wt.parts(wt.weight(x)) : 1;
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
    const uint64_t one = weighted ? wt.parts(wt.weight(__builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key))) : 1;
    const uint64_t ties = one ? (want - above + one - 1) / one : 1;
    uint64_t seen = 0;
    for (int base = 0; base < V; base += kThreads) {
      const int i = base + threadIdx.x;
      const bool tie = i < V && rank_key(logit<Z>(z, i)) == key && in.keeps(key, i);
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
    const Cut cut{key, seen >= ties ? (int)found[0] : V};
    __syncthreads();
    return cut;
  };

  Cut cut{0u, V};
  const int k = a.top_k ? a.top_k[row] : 0;
  if (k > 0 && k < V) cut = select((uint64_t)k, false, cut);
  const float p = a.top_p ? a.top_p[row] : 1.f;
  if (p < 1.f) {
    uint64_t mass = 0;
    for (int i = threadIdx.x; i < V; i += kThreads) {
      const float x = logit<Z>(z, i);
      if (cut.keeps(rank_key(x), i)) mass += wt.parts(wt.weight(x));
    }
    mass = block_sum(mass, scratch);
    const double part = ceil((double)p * (double)mass);
    const uint64_t want = part < 1.0 ? 1 : min(mass, (uint64_t)part);
    cut = select(want, true, cut);
  }
  const float least = a.min_p ? a.min_p[row] : 0.f;
  const double floor = least > 1.f ? 1.0 : (double)least;

  auto kept = [&](int i) -> uint64_t {
    const float x = logit<Z>(z, i);
    if (!cut.keeps(rank_key(x), i)) return 0;
    const double w = wt.weight(x);
    return w < floor ? 0 : wt.parts(w);
  };
  // every wave sums a run of the row; the draw falls into one of them
  const int seg = (V + kWaves - 1) / kWaves, lo = min(V, wave * seg), hi = min(V, lo + seg);
  uint64_t mine = 0;
  for (int i = lo + lane; i < hi; i += 64) mine += kept(i);
  for (int o = 32; o; o >>= 1) mine += __shfl_xor((unsigned long long)mine, o);
  if (lane == 0) scratch[wave] = mine;
  __syncthreads();
  uint64_t before = 0, mass = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    mass += scratch[w];
  }
  const float u = a.u[row];
  const double want = (double)u * (double)mass;
  const uint64_t target = !(want > 0.0) ? 0 : want >= (double)mass ? mass - 1 : min(mass - 1, (uint64_t)want);
  if (target < before || target >= before + mine) return;
  for (int base = lo; base < hi; base += 64) {
    const int i = base + lane;
    const uint64_t w = i < hi ? kept(i) : 0;
    uint64_t up = w;
    for (int o = 1; o < 64; o <<= 1) {
      const uint64_t v = __shfl_up((unsigned long long)up, o);
      if (lane >= o) up += v;
    }
    if (w && target >= before + up - w && target < before + up) {
      a.token[row] = i;
      if (a.prob) a.prob[row] = (float)((double)w / (double)mass);
    }
    before += __shfl((unsigned long long)up, 63);
    if (target < before) return;
  }
}

template <class Z>
hipError_t launch(const SampleArgs &a, hipStream_t s) {
  int shift = 62;
  while ((int64_t)1 << (62 - shift) < a.vocab) --shift;
  void *args[] = {const_cast<SampleArgs *>(&a), &shift};
  return hipLaunchKernel((const void *)sample_row_kernel<Z>, dim3(a.rows), dim3(kThreads), args, 0, s);
}

}  // namespace

hipError_t launch_sample(const SampleArgs &a, int type, hipStream_t s) {
  return type == 0 ? launch<float>(a, s) : type == 1 ? launch<__bf16>(a, s) : launch<_Float16>(a, s);
}

}  // namespace moecache
