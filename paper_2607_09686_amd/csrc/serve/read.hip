// The keys and values of the batch's tokens, taken out of a paged cache of 16 or 8 bits as rows (the
// inverse of appending, without its turn).
//
// Bound by the bytes it moves.  A wave takes the tokens of one sequence within one aligned run of
// eight positions, as a block does in appending, or a share of them where runs are few.  Of keys a lane takes eight
// elements of a token, of values two of eight tokens, which it writes as a piece of each token's row: a wave's pieces
// lie next to each other.  Measured: 65531 tokens of 4 heads of 128 from 8 bits, 202 MB, 33 us = 6.1 TB/s (a third of them
// read); with 16 elements of a key to a lane, whose two stores leave every other 16 bytes out, 38.6.
#include "append.h"
#include "held.h"

namespace moecache {
namespace {

// Rows go past the second-level caches, where they would only take the place of what is read: 65531 tokens of 4 heads of
// 128 33 us, else 44 (32000 from 16 bits 22.4 and 25.4).
template <class T>
__device__ __forceinline__ void put(void *p, T v) {
  __builtin_nontemporal_store(v, (T *)p);
}

template <class E, bool Held>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadArgs a) {
  constexpr int kUnit = Held ? 16 : 8;  // elements in 16 bytes
  const KvView &kv = a.kv;
  Run r;
  if (!run_of(kv, blockIdx.x * (kThreads / 64) + threadIdx.x / 64, threadIdx.x % 64 == 0 && blockIdx.y == 0, &r)) return;
  const int n = r.n, D = a.dim, P = 1 << kv.page_shift, in_page = r.position & (P - 1);
  const int64_t pool = (int64_t)r.page * kv.kv_heads, head_elems = (int64_t)D << kv.page_shift;
  const float none = __builtin_nanf("");
  const u32x4 nan = pack<E>({none, none, none, none, none, none, none, none});
  const int units = D / 8, keys = kv.kv_heads * units * kRun, all = keys + kv.kv_heads * D / 2;
  for (int i = blockIdx.y * 64 + threadIdx.x % 64; i < all; i += gridDim.y * 64) {
    if (i < keys) {  // eight elements of a token
      const int t = i / 2 % kRun, u = i / (2 * kRun) % (units / 2) * 2 + i % 2, head = i / kRun / units, tp = in_page + t;
      if (t >= n) continue;
      uint16_t *dst = (uint16_t *)a.k + (int64_t)(r.row + t) * a.k_stride + head * D + u * 8;
      const int64_t at = (pool + head) * head_elems + (tp & ~15) * D + (tp & 15) * kUnit;
      if (!r.write) {
        put(dst, nan);
      } else if constexpr (Held) {
        const uint2 c = *(const uint2 *)((const uint8_t *)kv.keys + at + u / 2 * 256 + u % 2 * 8);
        const float s = scale_of(kv.key_scales[((pool + head) << kv.page_shift) + tp]);
        put(dst, u32x4{decode(c.x, false, s, E()), decode(c.x, true, s, E()), decode(c.y, false, s, E()),
                       decode(c.y, true, s, E())});
      } else {
        put(dst, *(const u32x4 *)(kv.keys + at + u * 128));
      }
      continue;
    }
    // values: two neighbouring elements of all eight tokens to a lane
    const int tp = in_page & ~7, head = (i - keys) / (D / 2), d = (i - keys) % (D / 2) * 2;
    uint32_t out[kRun];
    if (!r.write) {
#pragma unroll
      for (int t = 0; t < kRun; ++t) out[t] = nan[0];
    } else if constexpr (Held) {
      const u32x4 c = *(const u32x4 *)((const uint8_t *)kv.values + (pool + head) * head_elems + tp * D + d * 8);
      const uint2 e = *(const uint2 *)(kv.value_scales + ((pool + head) << kv.page_shift) + tp);
#pragma unroll
      for (int t = 0; t < kRun; t += 2) {
        const uint32_t two = (t < 4 ? e.x : e.y) >> (8 * (t % 4));
        const float s0 = scale_of(two & 255), s1 = scale_of(two >> 8 & 255);
        const uint32_t x = decode2(c[t / 4], t % 4 != 0, s0, s1, E()), y = decode2(c[2 + t / 4], t % 4 != 0, s0, s1, E());
        out[t] = __builtin_amdgcn_perm(y, x, 0x05040100);
        out[t + 1] = __builtin_amdgcn_perm(y, x, 0x07060302);
      }
    } else {
      const u32x4 *src = (const u32x4 *)(kv.values + (pool + head) * head_elems + tp * D + d * 8);
      const u32x4 x = src[0], y = src[1];
#pragma unroll
      for (int t = 0; t < kRun; t += 2) {
        out[t] = __builtin_amdgcn_perm(y[t / 2], x[t / 2], 0x05040100);
        out[t + 1] = __builtin_amdgcn_perm(y[t / 2], x[t / 2], 0x07060302);
      }
    }
#pragma unroll
    for (int t = 0; t < kRun; ++t) {
      const int row = t - (in_page & 7);
      if (row >= 0 && row < n) put((uint16_t *)a.v + (int64_t)(r.row + row) * a.v_stride + head * D + d, out[t]);
    }
  }
}

template <class E>
hipError_t launch(const ReadArgs &a, hipStream_t s) {
  void *args[] = {const_cast<ReadArgs *>(&a)};
  const int runs = a.kv.n_tokens / kRun + 2 * a.kv.n_seqs;
  const void *fn = a.kv.key_scales ? (const void *)read_kernel<E, true> : (const void *)read_kernel<E, false>;
  int shares = 1;
  while (shares < 8 && 2 * shares * runs <= 16384) shares *= 2;  // waves enough to fill the card twice
  return hipLaunchKernel(fn, dim3((runs + kThreads / 64 - 1) / (kThreads / 64), shares), dim3(kThreads), args, 0, s);
}

}  // namespace

hipError_t launch_read(const ReadArgs &a, bool half, hipStream_t s) {
  return half ? launch<_Float16>(a, s) : launch<__bf16>(a, s);
}

}  // namespace moecache
