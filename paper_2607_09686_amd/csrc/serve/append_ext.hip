// Appending with a norm of each head before its turn, and to a cache of 8 bits (held.h).
//
//   x <- x / sqrt(mean(x^2) + eps) * w   (queries, keys, or both), then the turn (append.hip)
//
// with the sum of squares in fp32; every element is rounded once, to the queries' type or to the
// cache's 8 bits.  A wave takes whole heads of up to eight tokens, 16 elements to a lane, so that a
// head's sum and its largest magnitude are exchanged between lanes of one wave.  Values in 8 bits are
// turned from tokens' rows to the cache's [D][8] through LDS where the run is whole.
//
// Bound by its launch in a decode step (64 tokens of 32 + 2 x 4 heads of 128: 5.1 us, in 8 bits 6.3; the
// call's host side is 10.7), else by a wave's chain of loads, exchanges and stores over its heads, of which the next
// one's elements are requested ahead: 4096 tokens of them from fp32 in 8 bits, 122 MB, 28.3 us = 4.3 TB/s (31.1
// without the request ahead, 31.7 with sines, cosines and weights kept in registers, which leaves two waves a SIMD);
// 16384 from bf16, 319 MB, 70.5 us = 4.5 TB/s.
#include <algorithm>

#include "append.h"
#include "held.h"

namespace moecache {
namespace {

// Lane i's value beside lane i ^ 16's, and ^ 32's, in some order.
__device__ __forceinline__ f32x2 rows_16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ f32x2 rows_32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f32x2{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
// op over a head's lanes, which are toks apart; with a whole run's eight tokens by the vector unit's own exchanges.
template <class Op>
__device__ __forceinline__ float over_head(float v, int toks, int parts, Op op) {
  if (toks == kRun) {
    const int next = __builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x128, 0xf, 0xf, false);  // lane i ^ 8
    v = op(v, __uint_as_float((uint32_t)next));
    f32x2 r = rows_16(v);
    v = op(r[0], r[1]);
    if (parts == 4) return v;
    r = rows_32(v);
    return op(r[0], r[1]);
  }
  for (int o = toks; o < toks * parts; o *= 2) v = op(v, __shfl_xor(v, o));
  return v;
}

// 16 weights of a norm.
template <class E>
__device__ __forceinline__ void weights(const AppendArgs &a, const void *w, const Part &p, float (&x)[8], float (&y)[8]) {
  if (a.norm_f32) {
    In<float>::load(w, p.ea, x);
    In<float>::load(w, p.eb, y);
  } else {
    In<E>::load(w, p.ea, x);
    In<E>::load(w, p.eb, y);
  }
}

template <class E, class I, bool Held>
__global__ __launch_bounds__(kThreads) void append_ext_kernel(AppendArgs a) {
  const KvView &kv = a.kv;
  __shared__ Turns cs, sn;
  __shared__ __align__(16) uint8_t tile[kThreads / 64][64 * 16];
  Run r;
  if (!run_of(kv, blockIdx.x, threadIdx.x == 0 && blockIdx.y == 0, &r)) return;

  const int n = r.n, D = a.dim, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int P = 1 << kv.page_shift, in_page = r.position & (P - 1);
  const int64_t head_elems = (int64_t)D << kv.page_shift, first_elem = (int64_t)r.page * kv.kv_heads * head_elems;
  // lanes: tokens fastest, then a head's parts, then heads; heads of 256 take a run in two sets of tokens
  const int parts = D / 16;
  int toks = 1;
  while (toks < n && toks < kRun && toks * parts < 64) toks *= 2;
  const int per_wave = 64 / (toks * parts);
  const int tok = lane % toks, part = lane / toks % parts, sub = lane / (toks * parts);
  const int q_heads = a.q ? kv.heads : 0, k_end = q_heads + kv.kv_heads, heads = k_end + (Held ? kv.kv_heads : 0);
  const Part turned = part_of(a, part);
  const int h_first = (blockIdx.y * (kThreads / 64) + wave) * per_wave + sub;
  const int h_step = gridDim.y * (kThreads / 64) * per_wave;

  for (int t = tok; t - tok < n; t += toks) {
    const bool active = t < n;
    const int64_t row = r.row + (active ? t : 0);
    const I *q_row = (const I *)a.q + row * a.q_stride, *k_row = (const I *)a.k + row * a.k_stride;
    const I *v_row = (const I *)a.v + row * a.v_stride;
    E *const q_out = (E *)a.q_out + row * a.q_out_stride;
    const int tp = in_page + t;
    // the next head's elements are requested before this one's are used
    float nx[8], ny[8];
    auto request = [&](int h) {
      const int hr = min(h, heads - 1);  // lanes without a head of theirs read another's
      const I *src = hr < q_heads ? q_row + (int64_t)hr * D
                     : hr < k_end ? k_row + (int64_t)(hr - q_heads) * D
                                  : v_row + (int64_t)(hr - k_end) * D;
      const bool as_is = Held && hr >= k_end;  // values: 16 elements together
      In<I>::load(src, as_is ? part * 16 : turned.ea, nx);
      In<I>::load(src, as_is ? part * 16 + 8 : turned.eb, ny);
    };
    request(h_first);
    if (t == tok) turns_of(a, r, cs, sn);
    const float *const c = cs[min(t, kRun - 1)] + part * 8, *const s = sn[min(t, kRun - 1)] + part * 8;

    for (int h = h_first; h - sub < heads; h += h_step) {
      float ox[8], oy[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) ox[j] = nx[j], oy[j] = ny[j];
      request(h + h_step);
      const bool there = active && h < heads, is_q = h < q_heads, is_v = Held && h >= k_end;
      const void *w = is_q ? a.q_norm : is_v ? nullptr : a.k_norm;
      if (__any(there && w)) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += ox[j] * ox[j] + oy[j] * oy[j];
        sum = over_head(sum, toks, parts, [](float x, float y) { return x + y; });
        if (w) {
          const float f = 1.f / sqrtf(sum / (float)D + a.eps);
          float wx[8], wy[8];
          weights<E>(a, w, turned, wx, wy);
#pragma unroll
          for (int j = 0; j < 8; ++j) ox[j] = ox[j] * f * wx[j], oy[j] = oy[j] * f * wy[j];
        }
      }
      if (!is_v) turn(turned, c, s, r.bad, ox, oy);
      if (is_q && there) {
        E *dst = q_out + (int64_t)h * D;
        *(u32x4 *)(dst + turned.ea) = pack<E>(ox);
        *(u32x4 *)(dst + turned.eb) = pack<E>(oy);
      }
      if (!r.write || !__any(!is_q && there)) continue;
      const int head = h - (is_v ? k_end : q_heads);
      const int64_t pool = first_elem + (int64_t)head * head_elems;
      if constexpr (!Held) {
        if (!is_q && there) {  // keys: [P/16][D/8][16][8]
          uint16_t *dst = kv.keys + pool + (tp & ~15) * D + (tp & 15) * 8;
          *(u32x4 *)(dst + turned.ea / 8 * 128) = pack<E>(ox);
          *(u32x4 *)(dst + turned.eb / 8 * 128) = pack<E>(oy);
        }
      } else {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fmaxf(magnitude(ox[j]), magnitude(oy[j])));
        most = over_head(most, toks, parts, [](float x, float y) { return fmaxf(x, y); });
        const int e = scale_byte<E>(most);
        const float inverse = __uint_as_float((uint32_t)(254 - e) << 23);
        const uint32_t c8[4] = {encode(ox[0], ox[1], ox[2], ox[3], inverse), encode(ox[4], ox[5], ox[6], ox[7], inverse),
                                encode(oy[0], oy[1], oy[2], oy[3], inverse), encode(oy[4], oy[5], oy[6], oy[7], inverse)};
        if (!is_q && there && part == 0)
          (is_v ? kv.value_scales : kv.key_scales)[(((int64_t)r.page * kv.kv_heads + head) << kv.page_shift) + tp] = e;
        if (!is_q && !is_v && there) {  // keys: [P/16][D/16][16][16]
          uint8_t *dst = (uint8_t *)kv.keys + pool + (tp & ~15) * D + (tp & 15) * 16;
          *(uint2 *)(dst + turned.ea / 16 * 256 + turned.ea % 16) = uint2{c8[0], c8[1]};
          *(uint2 *)(dst + turned.eb / 16 * 256 + turned.eb % 16) = uint2{c8[2], c8[3]};
        }
        if (!__any(is_v && there)) continue;
        // values: [P/16][2][D][8].  A whole run's lie in units of 8 or (heads of 256) 4 tokens
        uint8_t *dst = (uint8_t *)kv.values + pool + (tp & ~7) * D;
        if (n == kRun) {
          uint8_t *mine = tile[wave] + (sub * D + part * 16) * toks + tok;
          if (toks == kRun) {
#pragma unroll
            for (int j = 0; j < 16; ++j) mine[j * kRun] = (uint8_t)(c8[j / 4] >> (8 * (j % 4)));
          } else {
#pragma unroll
            for (int j = 0; j < 16; ++j) mine[j * 4] = (uint8_t)(c8[j / 4] >> (8 * (j % 4)));
          }
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          const u32x4 u = *(const u32x4 *)(tile[wave] + lane * 16);
          __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
          // this lane's unit lies in the same head as its elements
          const int d = lane * 16 / toks % D;
          if (is_v && there) {
            if (toks == kRun) {
              *(u32x4 *)(dst + d * 8) = u;
            } else {
#pragma unroll
              for (int i = 0; i < 4; ++i) *(uint32_t *)(dst + (d + i) * 8 + (tp & 4)) = u[i];
            }
          }
        } else if (is_v && there) {
#pragma unroll
          for (int j = 0; j < 16; ++j) dst[(part * 16 + j) * 8 + (tp & 7)] = (uint8_t)(c8[j / 4] >> (8 * (j % 4)));
        }
      }
    }
  }
  if (!Held && r.write) append_values<E, I>(a, r, in_page);
}

// Blocks aimed at, to share out a run's heads where there are few runs: what the card holds (4096 tokens: 28.3 us, with
// half as many 31.7, with twice as many 32.3).
constexpr int kBlocks = 1024;

template <class E, class I>
hipError_t launch(const AppendArgs &a, hipStream_t s) {
  void *args[] = {const_cast<AppendArgs *>(&a)};
  const int runs = a.kv.n_tokens / kRun + 2 * a.kv.n_seqs;
  const bool held = a.kv.key_scales;
  const void *fn = held ? (const void *)append_ext_kernel<E, I, true> : (const void *)append_ext_kernel<E, I, false>;
  // what a wave takes of a run at once: 128 elements of its eight tokens, one KV head of 64 being half of that
  const int items = (((a.q ? a.kv.heads : 0) + a.kv.kv_heads * (held ? 2 : 1)) * a.dim + 127) / 128;
  const int shares = std::min((items + 3) / 4, std::max(1, (kBlocks + runs - 1) / runs));
  return hipLaunchKernel(fn, dim3(runs, shares), dim3(kThreads), args, 0, s);
}

}  // namespace

hipError_t launch_append_ext(const AppendArgs &a, bool half, bool in_f32, hipStream_t s) {
  if (half) return in_f32 ? launch<_Float16, float>(a, s) : launch<_Float16, _Float16>(a, s);
  return in_f32 ? launch<__bf16, float>(a, s) : launch<__bf16, __bf16>(a, s);
}

}  // namespace moecache
