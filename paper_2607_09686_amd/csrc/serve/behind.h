// Attention over a cache of 8 bits, and of a batch whose sequences begin with the same tokens.
//
// What all sequences begin with is read once: with S its tokens (whole 64s of them),
//
//   o = (l1 o1 2^(m1 - m) + l2 o2 2^(m2 - m)) / (l1 2^(m1 - m) + l2 2^(m2 - m)),   m = max(m1, m2)
//
// joins a row's sums over the keys before S and from S on.  The first come from a launch that takes the whole
// batch's rows as those of one sequence (no row there has a mask, so they need not know their own), the second
// from the ordinary one with its ranges cut at S, every tile of which leaves partial results.
#pragma once

#include "attend.h"

namespace moecache {
// these are in the ordinary attention's files
extern template hipError_t launch_plan<64>(const AttendArgs &, int, hipStream_t);
extern template hipError_t launch_plan<128>(const AttendArgs &, int, hipStream_t);
extern template hipError_t launch_plan<256>(const AttendArgs &, int, hipStream_t);
extern template hipError_t launch_join<64>(const AttendArgs &, bool, int, hipStream_t);
extern template hipError_t launch_join<128>(const AttendArgs &, bool, int, hipStream_t);
extern template hipError_t launch_join<256>(const AttendArgs &, bool, int, hipStream_t);
namespace {

template <class E, int D, int R>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void held_few_kernel(AttendArgs a) {
  __shared__ __align__(16) FewLds<D> lds;
  few_body<E, D, R, true, kAll>(a, lds, blockIdx.x);
}
template <class E, int D>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void held_many_kernel(AttendArgs a) {
  __shared__ __align__(16) ManyLds<D> lds;
  many_body<E, D, true, kAll>(a, lds, blockIdx.x);
}

// Units over what is shared, in tiles of FM rows, and then units behind it, in tiles of M, in one launch: the first
// are bound by the matrix cores where the batch is large, the others by the cache's bytes.
template <class E, int D, int FM, int M, bool Held>
__global__ __launch_bounds__(kThreads, D > 128 ? 1 : 2) void behind_kernel(AttendArgs a) {
  __shared__ __align__(16) union {
    FewLds<D> few;
    ManyLds<D> many;
  } lds;
  const int front = a.prefix_tiles * a.prefix_splits * a.kv.kv_heads, block = blockIdx.x;
  if (block < front) {
    if constexpr (FM == 128)
      many_body<E, D, Held, kPrefix>(a, lds.many, block);
    else
      few_body<E, D, FM / 32, Held, kPrefix>(a, lds.few, block);
  } else {
    if constexpr (M == 128)
      many_body<E, D, Held, kBehind>(a, lds.many, block - front);
    else
      few_body<E, D, M / 32, Held, kBehind>(a, lds.few, block - front);
  }
}
template <int M>
__global__ __launch_bounds__(kPlanThreads) void plan_behind_kernel(AttendArgs a) {
  plan_body<M, kBehind>(a);
}
// Joins what the launch left of each row: the prefix's units and then the tile's own.  As the ordinary joining; a
// group of D / 4 lanes reads kAtOnce of a row's partial results at once.  Bound by where they lie (the writers' caches are
// other ones): 64 sequences behind 8192 tokens, calls of 45.6 us; 46.5 with four at once, 50 to 52 with 512 threads.
constexpr int kJoinThreads = 256, kAtOnce = 2;
// Blocks that join, up to rows / 4 and at least 4 of them to a tile: about 2048 in all, what the card holds at once (the
// 64 sequences' 320 tiles with 8 each 43.2 us, with 4 42.0; the 36 of 8 sequences 29.5 and 32.8); fewer than 4 where
// all of them (up to 2^23 tiles) would be more threads than a grid holds.
static inline dim3 join_behind_grid(const AttendArgs &a, int rows) {
  const int64_t tiles = (int64_t)a.max_tiles * a.kv.kv_heads;
  int y = 4;
  while (2 * y <= rows / 4 && 2 * y * tiles <= 2048) y *= 2;
  while (y > 1 && y * tiles * kJoinThreads >= (int64_t)1 << 32) y /= 2;
  return dim3((unsigned)tiles, y);
}
template <class E, int D, int M>
__global__ __launch_bounds__(kJoinThreads) void join_behind_kernel(AttendArgs a) {
  constexpr int kPer = D / 4, kGroups = kJoinThreads / kPer;
  __shared__ __align__(16) float sum[kGroups][D];
  __shared__ float stat[kGroups][2];
  const int item = blockIdx.x / a.kv.kv_heads, kvh = blockIdx.x % a.kv.kv_heads;
  const SplitTile t = split_tiles(a)->tile[item];
  const Prefix pre = prefix_of(a);
  if (item >= split_tiles(a)->count) return;
  // a sequence that cannot be served has no units; starts out of order can leave a note unwritten: nothing is taken from
  // one that makes no sense
  if (t.units < 1 || t.slot < 0 || t.slot > a.max_slots - t.units || t.rows < 1 || t.rows > M || t.first < 0 ||
      t.row0 < 0 || t.row0 > (1 << 28) || t.first > a.kv.n_tokens - 1 - (t.row0 + t.rows - 1) / a.kv.group)
    return;
  const int64_t row0 = (int64_t)(t.first - pre.first) * a.kv.group + t.row0;  // among the prefix's rows
  const int front = row0 >= 0 && row0 + t.rows <= pre.rows ? pre.units : 0, units = front + t.units;
  const int g = threadIdx.x / kPer, d = threadIdx.x % kPer * 4;
  int per = 1;  // groups to a row
  while (per < kGroups && per * kAtOnce < units) per *= 2;
  const int own = g / per, at_once = kGroups / per;
  const int64_t step = (int64_t)a.kv.kv_heads * M, front_step = (int64_t)a.kv.kv_heads * a.prefix_rows;
  for (int r0 = 0; (int)(blockIdx.y + gridDim.y * r0) < t.rows; r0 += at_once) {
    const int row = blockIdx.y + gridDim.y * (r0 + own);
    float m = kNegInf, l = 0.f;
    f32x4 o{};
    if (row < t.rows) {
      const float *ml = part_ml<D, M>(a, t.slot, kvh, row), *part = part_o<D, M>(a, t.slot, kvh, row) + d;
      const int at = (int)row0 + row;
      const int64_t from = front ? front_row(a, at / a.prefix_rows * a.prefix_splits, kvh, at % a.prefix_rows) : 0;
      for (int i0 = g % per; i0 < units; i0 += per * kAtOnce) {
        float mi[kAtOnce], li[kAtOnce];
        f32x4 oi[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const int i = i0 + per * j;
          mi[j] = kNegInf, li[j] = 0.f, oi[j] = f32x4{};
          if (i < units) {
            const bool own_unit = i >= front;
            const float *x = own_unit ? ml + (i - front) * step * 2 : front_ml<D>(a, from + i * front_step);
            mi[j] = x[0], li[j] = x[1];
            oi[j] = *(const f32x4 *)(own_unit ? part + (i - front) * step * D : front_o<D>(a, from + i * front_step) + d);
          }
        }
        float top = m;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) top = fmaxf(top, mi[j]);
        const float base = top == kNegInf ? 0.f : top, shrink = __builtin_amdgcn_exp2f(m - base);
        l *= shrink, o *= shrink, m = top;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
          const float w = __builtin_amdgcn_exp2f(mi[j] - base);
          l += w * li[j];
          o += w * oi[j];
        }
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

template <class E, int D, bool Held>
hipError_t launch_behind(const AttendArgs &a, int rows, hipStream_t s) {
  void *args[] = {const_cast<AttendArgs *>(&a)};
  hipError_t e = hipSuccess;
  if (a.kv.n_seqs > kPlanSeqs)
    e = hipLaunchKernel(rows == 32   ? (const void *)plan_behind_kernel<32>
                        : rows == 64 ? (const void *)plan_behind_kernel<64>
                                     : (const void *)plan_behind_kernel<128>,
                        dim3(1), dim3(kPlanThreads), args, 0, s);
  // all rows together are at least as many as the mean sequence's
  const void *fn = rows == 128              ? (const void *)behind_kernel<E, D, 128, 128, Held>
                   : a.prefix_rows == 128   ? rows == 64 ? (const void *)behind_kernel<E, D, 128, 64, Held>
                                                         : (const void *)behind_kernel<E, D, 128, 32, Held>
                   : a.prefix_rows == 64    ? rows == 64 ? (const void *)behind_kernel<E, D, 64, 64, Held>
                                                         : (const void *)behind_kernel<E, D, 64, 32, Held>
                                            : (const void *)behind_kernel<E, D, 32, 32, Held>;
  const int64_t units = (int64_t)a.prefix_tiles * a.prefix_splits + a.max_units;
  if (e == hipSuccess) e = hipLaunchKernel(fn, dim3((unsigned)(units * a.kv.kv_heads)), dim3(kThreads), args, 0, s);
  if (e != hipSuccess) return e;
  return hipLaunchKernel(rows == 32   ? (const void *)join_behind_kernel<E, D, 32>
                         : rows == 64 ? (const void *)join_behind_kernel<E, D, 64>
                                      : (const void *)join_behind_kernel<E, D, 128>,
                         join_behind_grid(a, rows), dim3(kJoinThreads), args, 0, s);
}

template <class E, int D>
hipError_t launch_held(const AttendArgs &a, int rows, hipStream_t s) {
  void *args[] = {const_cast<AttendArgs *>(&a)};
  hipError_t e = launch_plan<D>(a, rows, s);
  if (e == hipSuccess)
    e = hipLaunchKernel(rows == 32   ? (const void *)held_few_kernel<E, D, 1>
                        : rows == 64 ? (const void *)held_few_kernel<E, D, 2>
                                     : (const void *)held_many_kernel<E, D>,
                        dim3((unsigned)((int64_t)a.max_units * a.kv.kv_heads)), dim3(kThreads), args, 0, s);
  return e == hipSuccess ? launch_join<D>(a, __is_same(E, _Float16), rows, s) : e;
}

template <class E, int D>
hipError_t launch_ext(const AttendArgs &a, int rows, hipStream_t s) {
  if (!a.shared) return launch_held<E, D>(a, rows, s);
  return a.kv.key_scales ? launch_behind<E, D, true>(a, rows, s) : launch_behind<E, D, false>(a, rows, s);
}

}  // namespace

template <int D>
hipError_t launch_attend_ext(const AttendArgs &a, bool half, int rows, hipStream_t s) {
  return half ? launch_ext<_Float16, D>(a, rows, s) : launch_ext<__bf16, D>(a, rows, s);
}

}  // namespace moecache
