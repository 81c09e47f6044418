// Appends the new tokens' keys and values to a paged cache (layout: attend.h), turning keys and
// queries by their position on the way.
//
//   (x_a, x_b) -> (x_a cos t - x_b sin t, x_b cos t + x_a sin t),  t = position * freq_i
//
// for the rope_dim / 2 pairs of a head: (i, i + rope_dim / 2), or (2i, 2i + 1).  The angle is taken
// in 64 bits and reduced to a part of a turn before the sine and cosine are taken in 32 (at
// position 100 000 an angle in 32 bits is off by 0.004); every element is rounded once, to the cache's type.
//
// Bound by the bytes it moves, in one decode step by its launch.  A block takes the new tokens of
// one sequence within one aligned run of eight positions: they share a page, their values are
// whole 16-byte units of the cache, and the block's angles are shared by all heads.  Four blocks
// to a run share out its heads, so that a decode step's few runs still fill the card.  Measured: 64
// tokens of 32 + 2 x 4 heads of 128, 4.2 us (an empty launch takes about 2); 4096 tokens of them from fp32,
// 126 MB, 25 us = 5.0 TB/s.
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

template <class E, class I>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  const KvView &kv = a.kv;
  __shared__ float cs[kRun][129], sn[kRun][129];  // a row per token, on banks of their own
  const int lane = threadIdx.x % 64, run = blockIdx.x;
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
  if (count == 0) return;
  const bool bad = length < count || length > (kv.max_pages << kv.page_shift);
  const int before = bad ? 0 : length - count;  // one that cannot be served is walked as if it began at 0
  // this block's tokens j0 .. j1 - 1 of the sequence
  const int local = run - first_run(kv, seq);
  if (local < 0) return;
  const int64_t p0 = ((int64_t)(before / kRun) + local) * kRun;
  const int j0 = (int)(max(p0, (int64_t)before) - before);
  const int j1 = (int)min(p0 + kRun - before, (int64_t)count);
  if (j0 >= j1) return;
  const int n = j1 - j0, D = a.dim, R = a.rope_dim;
  int page = 0;
  bool write = !bad;
  if (bad) {
    if (threadIdx.x == 0 && blockIdx.y == 0 && kv.status) atomicOr(kv.status, kKvBadLength);
  } else {
    page = kv.pages[(int64_t)seq * kv.max_pages + (int)(p0 >> kv.page_shift)];
    if ((unsigned)page >= (unsigned)kv.n_pages) {
      write = false;
      page = 0;
      if (threadIdx.x == 0 && blockIdx.y == 0 && kv.status) atomicOr(kv.status, kKvBadPage);
    }
  }
  for (int i = threadIdx.x; i < n * (R / 2); i += kThreads) {
    const int t = i / (R / 2), f = i % (R / 2);
    const double turns = (double)(before + j0 + t) * a.freq[f] * kTurn;
    const float part = (float)(turns - rint(turns));
    float s, c;
    sincospif(2.f * part, &s, &c);
    cs[t][f] = bad ? __builtin_nanf("") : c;
    sn[t][f] = bad ? __builtin_nanf("") : s;
  }
  __syncthreads();

  const int P = 1 << kv.page_shift, in_page = (before + j0) & (P - 1);
  const int64_t head_elems = (int64_t)D << kv.page_shift;
  // queries and keys: 16 elements (eight pairs) of a head per thread and round, tokens fastest, so
  // that neighbours read and write runs of both the rows and the cache's groups
  const int per_head = D / 16, q_heads = a.q ? kv.heads : 0;
  const int units = (q_heads + kv.kv_heads) * per_head * n;
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < units; i += gridDim.y * kThreads) {
    const int t = n == kRun ? i % kRun : i % n, u = n == kRun ? i / kRun : i / n;
    const int part = u % per_head, h = u / per_head;
    const bool is_q = h < q_heads;
    const int head = is_q ? h : h - q_heads;
    const int64_t row = first + j0 + t;
    const bool turned = part * 16 < R;
    const bool halves = turned && !a.adjacent;
    const int ea = halves ? part * 8 : part * 16, eb = halves ? R / 2 + part * 8 : part * 16 + 8;
    const void *src = is_q ? a.q : a.k;
    const int64_t at = row * (is_q ? a.q_stride : a.k_stride) + (int64_t)head * D;
    float x[8], y[8], ox[8], oy[8];
    In<I>::load(src, at + ea, x);
    In<I>::load(src, at + eb, y);
    if (halves) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float c = cs[t][part * 8 + j], s = sn[t][part * 8 + j];
        ox[j] = x[j] * c - y[j] * s;
        oy[j] = y[j] * c + x[j] * s;
      }
    } else if (turned) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float c = cs[t][part * 8 + j], s = sn[t][part * 8 + j];
        const float c2 = cs[t][part * 8 + 4 + j], s2 = sn[t][part * 8 + 4 + j];
        ox[2 * j] = x[2 * j] * c - x[2 * j + 1] * s;
        ox[2 * j + 1] = x[2 * j + 1] * c + x[2 * j] * s;
        oy[2 * j] = y[2 * j] * c2 - y[2 * j + 1] * s2;
        oy[2 * j + 1] = y[2 * j + 1] * c2 + y[2 * j] * s2;
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        ox[j] = bad ? __builtin_nanf("") : x[j];
        oy[j] = bad ? __builtin_nanf("") : y[j];
      }
    }
    if (is_q) {
      uint16_t *dst = (uint16_t *)a.q_out + row * a.q_out_stride + (int64_t)head * D;
      *(u32x4 *)(dst + ea) = pack<E>(ox);
      *(u32x4 *)(dst + eb) = pack<E>(oy);
    } else if (write) {
      const int tp = in_page + t;  // keys: [P/16][D/8][16][8]
      uint16_t *dst = kv.keys + ((int64_t)page * kv.kv_heads + head) * head_elems + (tp & ~15) * D + (tp & 15) * 8;
      *(u32x4 *)(dst + ea / 8 * 128) = pack<E>(ox);
      *(u32x4 *)(dst + eb / 8 * 128) = pack<E>(oy);
    }
  }
  if (!write) return;
  // values: one element of a head per thread and round over the run's tokens; [P/16][2][D][8]
  for (int i = blockIdx.y * kThreads + threadIdx.x; i < kv.kv_heads * D; i += gridDim.y * kThreads) {
    const int head = i / D, d = i % D;
    const I *src = (const I *)a.v + (int64_t)(first + j0) * a.v_stride + i;
    E *dst = (E *)kv.values + ((int64_t)page * kv.kv_heads + head) * head_elems + (in_page & ~7) * D + d * 8;
    if (n == kRun) {
      float x[8];
#pragma unroll
      for (int t = 0; t < kRun; ++t) x[t] = (float)src[t * a.v_stride];
      *(u32x4 *)dst = pack<E>(x);
    } else {
      for (int t = 0; t < n; ++t) dst[(in_page & 7) + t] = (E)(float)src[t * a.v_stride];
    }
  }
}

template <class E, class I>
hipError_t launch(const AppendArgs &a, hipStream_t s) {
  void *args[] = {const_cast<AppendArgs *>(&a)};
  const int runs = a.kv.n_tokens / kRun + 2 * a.kv.n_seqs;
  return hipLaunchKernel((const void *)append_kernel<E, I>, dim3(runs, kShares), dim3(kThreads), args, 0, s);
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, bool half, bool in_f32, hipStream_t s) {
  if (half) return in_f32 ? launch<_Float16, float>(a, s) : launch<_Float16, _Float16>(a, s);
  return in_f32 ? launch<__bf16, float>(a, s) : launch<__bf16, __bf16>(a, s);
}

}  // namespace moecache
