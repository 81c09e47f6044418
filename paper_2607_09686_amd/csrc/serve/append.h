// What the kernels share that walk a batch's new tokens in runs of eight positions: appending to a
// paged cache and reading it back.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "serve.h"

namespace moecache {
namespace {

constexpr int kThreads = 256, kRun = 8, kShares = 4;
constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements as fp32; I the input's type.
template <class I>
struct In {
  typedef I x8 __attribute__((ext_vector_type(8)));
  static __device__ __forceinline__ void load(const void *p, int64_t at, float (&v)[8]) {
    const x8 e = *(const x8 *)((const I *)p + at);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)e[i];
  }
};
template <>
struct In<float> {
  static __device__ __forceinline__ void load(const void *p, int64_t at, float (&v)[8]) {
    const f32x4 a = *(const f32x4 *)((const float *)p + at), b = *(const f32x4 *)((const float *)p + at + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
};
template <class E>
__device__ __forceinline__ u32x4 pack(const float (&v)[8]) {
  typedef E x8 __attribute__((ext_vector_type(8)));
  x8 e;
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = (E)v[i];
  return __builtin_bit_cast(u32x4, e);
}

// Runs are numbered so that a sequence's first one has a number its block can find without a
// sum over the sequences before it: floor(start / 8) + 2 s.  n tokens touch at most n / 8 + 2 runs,
// so the numbers do not collide; some stand for nothing.
__device__ __forceinline__ int first_run(const KvView &kv, int s) {
  return min(max(kv.starts[s], 0), kv.n_tokens) / kRun + 2 * s;
}

// The new tokens that a block takes: positions p .. p + n - 1 of one sequence, all in one page.
struct Run {
  int row, position, n;  // row: of the first one among the new tokens
  int page;
  bool bad, write;  // a sequence that cannot be served; whether the page is one
};
// `teller`: the thread that reports what is wrong with the run
__device__ __forceinline__ bool run_of(const KvView &kv, int run, bool teller, Run *r) {
  const int lane = threadIdx.x % 64;
  // the last sequence whose first run is at or before this one, 64 probes at a time
  int lo = 0, hi = kv.n_seqs;
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64, at = lo + lane * step;
    const uint64_t in = __ballot(at < hi && first_run(kv, at) <= run);
    const int k = in ? 63 - __clzll((long long)in) : 0;
    lo += k * step;
    hi = min(hi, lo + step);
  }
  const int seq = lo;
  const int first = min(max(kv.starts[seq], 0), kv.n_tokens);
  const int count = min(max(kv.starts[seq + 1], first), kv.n_tokens) - first, length = kv.lengths[seq];
  if (count == 0) return false;
  const bool bad = length < count || length > (kv.max_pages << kv.page_shift);
  const int before = bad ? 0 : length - count;  // one that cannot be served is walked as if it began at 0
  // this block's tokens j0 .. j1 - 1 of the sequence
  const int local = run - first_run(kv, seq);
  if (local < 0) return false;
  const int64_t p0 = ((int64_t)(before / kRun) + local) * kRun;
  const int j0 = (int)(max(p0, (int64_t)before) - before);
  const int j1 = (int)min(p0 + kRun - before, (int64_t)count);
  if (j0 >= j1) return false;
  *r = Run{first + j0, before + j0, j1 - j0, 0, bad, !bad};
  if (bad) {
    if (teller && kv.status) atomicOr(kv.status, kKvBadLength);
  } else {
    r->page = kv.pages[(int64_t)seq * kv.max_pages + (int)(p0 >> kv.page_shift)];
    if ((unsigned)r->page >= (unsigned)kv.n_pages) {
      r->write = false;
      r->page = 0;
      if (teller && kv.status) atomicOr(kv.status, kKvBadPage);
    }
  }
  return true;
}

// The sines and cosines of the block's tokens; ends with a barrier.
typedef float Turns[kRun][129];  // a row per token, on banks of their own
__device__ __forceinline__ void turns_of(const AppendArgs &a, const Run &r, Turns &cs, Turns &sn) {
  const int half = a.rope_dim / 2;
  for (int i = threadIdx.x; i < r.n * half; i += kThreads) {
    const int t = i / half, f = i % half;
    const double turns = (double)(r.position + t) * a.freq[f] * kTurn;
    const float part = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.f * part, &s, &c);
    cs[t][f] = r.bad ? __builtin_nanf("") : c;
    sn[t][f] = r.bad ? __builtin_nanf("") : s;
  }
  __syncthreads();
}

// The first and second eight elements of a head that part `part` of it (16 elements) holds, and their turn.
struct Part {
  bool turned, halves;
  int ea, eb;
};
__device__ __forceinline__ Part part_of(const AppendArgs &a, int part) {
  const int R = a.rope_dim;
  const bool turned = part * 16 < R, halves = turned && !a.adjacent;
  return Part{turned, halves, halves ? part * 8 : part * 16, halves ? R / 2 + part * 8 : part * 16 + 8};
}
// Turns them in place by a part's eight sines and cosines.
__device__ __forceinline__ void turn(const Part &p, const float *c, const float *s, bool bad, float (&x)[8], float (&y)[8]) {
  if (p.halves) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = x[j], b = y[j];
      x[j] = a * c[j] - b * s[j];
      y[j] = b * c[j] + a * s[j];
    }
  } else if (p.turned) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float a = x[2 * j], b = x[2 * j + 1], d = y[2 * j], e = y[2 * j + 1];
      x[2 * j] = a * c[j] - b * s[j];
      x[2 * j + 1] = b * c[j] + a * s[j];
      y[2 * j] = d * c[4 + j] - e * s[4 + j];
      y[2 * j + 1] = e * c[4 + j] + d * s[4 + j];
    }
  } else if (bad) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = y[j] = __builtin_nanf("");
  }
}

// Values in 16 bits: one element of a head per thread and round over the run's tokens; [P/16][2][D][8]
template <class E, class I>
__device__ __forceinline__ void append_values(const AppendArgs &a, const Run &r, int in_page) {
  const KvView &kv = a.kv;
  const int D = a.dim;
  const int64_t head_elems = (int64_t)D << kv.page_shift;
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < kv.kv_heads * D; i += gridDim.y * kThreads) {
    const int head = i / D, d = i % D;
    const I *src = (const I *)a.v + (int64_t)r.row * a.v_stride + i;
    E *dst = (E *)kv.values + ((int64_t)r.page * kv.kv_heads + head) * head_elems + (in_page & ~7) * D + d * 8;
    if (r.n == kRun) {
      float x[8];
#pragma unroll
      for (int t = 0; t < kRun; ++t) x[t] = (float)src[t * a.v_stride];
      *(u32x4 *)dst = pack<E>(x);
    } else {
      for (int t = 0; t < r.n; ++t) dst[(in_page & 7) + t] = (E)(float)src[t * a.v_stride];
    }
  }
}

}  // namespace
}  // namespace moecache
