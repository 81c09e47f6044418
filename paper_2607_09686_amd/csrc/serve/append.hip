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
// 126 MB, 29.5 us = 4.3 TB/s (25 where the last-level cache holds the inputs).
#include "append.h"

namespace moecache {
namespace {

template <class E, class I>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  const KvView &kv = a.kv;
  __shared__ Turns cs, sn;
  Run r;
  if (!run_of(kv, blockIdx.x, threadIdx.x == 0 && blockIdx.y == 0, &r)) return;
  turns_of(a, r, cs, sn);

  const int n = r.n, D = a.dim;
  const int P = 1 << kv.page_shift, in_page = r.position & (P - 1);
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
    const int64_t row = r.row + t;
    const Part p = part_of(a, part);
    const void *src = is_q ? a.q : a.k;
    const int64_t at = row * (is_q ? a.q_stride : a.k_stride) + (int64_t)head * D;
    float x[8], y[8];
    In<I>::load(src, at + p.ea, x);
    In<I>::load(src, at + p.eb, y);
    turn(p, cs[t] + part * 8, sn[t] + part * 8, r.bad, x, y);
    if (is_q) {
      uint16_t *dst = (uint16_t *)a.q_out + row * a.q_out_stride + (int64_t)head * D;
      *(u32x4 *)(dst + p.ea) = pack<E>(x);
      *(u32x4 *)(dst + p.eb) = pack<E>(y);
    } else if (r.write) {
      const int tp = in_page + t;  // keys: [P/16][D/8][16][8]
      uint16_t *dst = kv.keys + ((int64_t)r.page * kv.kv_heads + head) * head_elems + (tp & ~15) * D + (tp & 15) * 8;
      *(u32x4 *)(dst + p.ea / 8 * 128) = pack<E>(x);
      *(u32x4 *)(dst + p.eb / 8 * 128) = pack<E>(y);
    }
  }
  if (r.write) append_values<E, I>(a, r, in_page);
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
