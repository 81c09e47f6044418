// Appending with a norm of each head before its turn, and to a cache of 8 bits (held.h).
//
//   x <- x / sqrt(mean(x^2) + eps) * w   (queries, keys, or both), then the turn (append.hip)
//
// with the sum of squares in fp32; every element is rounded once, to the queries' type or to the
// cache's 8 bits.  A wave takes whole heads of up to eight tokens, 16 elements to a lane, so that a
// head's sum and its largest magnitude are exchanged between lanes of one wave.  Values in 8 bits are
// turned from tokens' rows to the cache's [D][8] through LDS where the run is whole.
#include "append.h"
#include "held.h"

namespace moecache {
namespace {

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
  if (!run_of(kv, &r)) return;
  turns_of(a, r, cs, sn);

  const int n = r.n, D = a.dim, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int P = 1 << kv.page_shift, in_page = r.position & (P - 1);
  const int64_t head_elems = (int64_t)D << kv.page_shift;
  // lanes: tokens fastest, then a head's parts, then heads (or a second set of tokens of the same one)
  const int parts = D / 16;
  int toks = 1;
  while (toks < n && toks < kRun && toks * parts < 64) toks *= 2;
  const int per_wave = 64 / (toks * parts), sets = (n + toks - 1) / toks;
  const int tok = lane % toks, part = lane / toks % parts, sub = lane / (toks * parts);
  const int q_heads = a.q ? kv.heads : 0, heads = q_heads + kv.kv_heads * (Held ? 2 : 1);
  const Part turned = part_of(a, part), plain{false, false, part * 16, part * 16 + 8};
  const int items = (heads * sets + per_wave - 1) / per_wave, waves = kThreads / 64;
  for (int item = blockIdx.y * waves + wave; item < items; item += gridDim.y * waves) {
    const int at = item * per_wave + sub, h = at / sets, t = at % sets * toks + tok;
    const bool active = h < heads && t < n;
    const bool is_q = h < q_heads, is_v = Held && h >= q_heads + kv.kv_heads;
    const int head = is_q ? h : is_v ? h - q_heads - kv.kv_heads : h - q_heads;
    const int64_t row = r.row + t;
    const Part p = is_v ? plain : turned;
    float ox[8] = {}, oy[8] = {};
    if (active) {
      const void *src = is_q ? a.q : is_v ? a.v : a.k;
      const int64_t from = row * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + (int64_t)head * D;
      In<I>::load(src, from + p.ea, ox);
      In<I>::load(src, from + p.eb, oy);
    }
    const void *w = is_q ? a.q_norm : is_v ? nullptr : a.k_norm;
    if (__any(active && w)) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += ox[j] * ox[j] + oy[j] * oy[j];
      for (int o = toks; o < toks * parts; o *= 2) sum += __shfl_xor(sum, o);
      if (active && w) {
        const float f = 1.f / sqrtf(sum / (float)D + a.eps);
        float wx[8], wy[8];
        weights<E>(a, w, p, wx, wy);
#pragma unroll
        for (int j = 0; j < 8; ++j) ox[j] = ox[j] * f * wx[j], oy[j] = oy[j] * f * wy[j];
      }
    }
    if (!is_v) {
      float x[8], y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = ox[j], y[j] = oy[j];
      const int ts = min(t, kRun - 1);
      turn(p, cs[ts], sn[ts], part, r.bad, x, y, ox, oy);
    }
    if (is_q && active) {
      uint16_t *dst = (uint16_t *)a.q_out + row * a.q_out_stride + (int64_t)head * D;
      *(u32x4 *)(dst + p.ea) = pack<E>(ox);
      *(u32x4 *)(dst + p.eb) = pack<E>(oy);
    }
    const int tp = in_page + t;
    if constexpr (!Held) {
      if (!is_q && active && r.write) {  // keys: [P/16][D/8][16][8]
        uint16_t *dst = kv.keys + ((int64_t)r.page * kv.kv_heads + head) * head_elems + (tp & ~15) * D + (tp & 15) * 8;
        *(u32x4 *)(dst + p.ea / 8 * 128) = pack<E>(ox);
        *(u32x4 *)(dst + p.eb / 8 * 128) = pack<E>(oy);
      }
    } else if (r.write && __any(!is_q && active)) {
      float most = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = fmaxf(most, fmaxf(magnitude(ox[j]), magnitude(oy[j])));
      for (int o = toks; o < toks * parts; o *= 2) most = fmaxf(most, __shfl_xor(most, o));
      const int e = scale_byte<E>(most);
      const float inverse = __uint_as_float((uint32_t)(254 - e) << 23);
      const uint32_t c[4] = {encode(ox[0], ox[1], ox[2], ox[3], inverse), encode(ox[4], ox[5], ox[6], ox[7], inverse),
                             encode(oy[0], oy[1], oy[2], oy[3], inverse), encode(oy[4], oy[5], oy[6], oy[7], inverse)};
      const int64_t pool = ((int64_t)r.page * kv.kv_heads + head) * head_elems;
      if (!is_q && active && part == 0)
        (is_v ? kv.value_scales : kv.key_scales)[(((int64_t)r.page * kv.kv_heads + head) << kv.page_shift) + tp] = e;
      if (!is_q && !is_v && active) {  // keys: [P/16][D/16][16][16]
        uint8_t *dst = (uint8_t *)kv.keys + pool + (tp & ~15) * D + (tp & 15) * 16;
        *(uint2 *)(dst + p.ea / 16 * 256 + p.ea % 16) = uint2{c[0], c[1]};
        *(uint2 *)(dst + p.eb / 16 * 256 + p.eb % 16) = uint2{c[2], c[3]};
      }
      // values: [P/16][2][D][8].  A whole run's lie in units of 8 or (heads of 256) 4 tokens
      uint8_t *dst = (uint8_t *)kv.values + pool + (tp & ~7) * D;
      if (n == kRun) {
        uint8_t *mine = tile[wave];
#pragma unroll
        for (int j = 0; j < 16; ++j) mine[(sub * D + part * 16 + j) * toks + tok] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const u32x4 u = *(const u32x4 *)(mine + lane * 16);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        // this lane's unit lies in the same head and part of it as its elements
        const int d = lane * 16 / toks % D;
        if (is_v && active) {
          if (toks == kRun) {
            *(u32x4 *)(dst + d * 8) = u;
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) *(uint32_t *)(dst + (d + i) * 8 + (tp & 4)) = u[i];
          }
        }
      } else if (is_v && active) {
#pragma unroll
        for (int j = 0; j < 16; ++j) dst[(part * 16 + j) * 8 + (tp & 7)] = (uint8_t)(c[j / 4] >> (8 * (j % 4)));
      }
    }
  }
  if (!Held && r.write) append_values<E, I>(a, r, in_page);
}

template <class E, class I>
hipError_t launch(const AppendArgs &a, hipStream_t s) {
  void *args[] = {const_cast<AppendArgs *>(&a)};
  const int runs = a.kv.n_tokens / kRun + 2 * a.kv.n_seqs;
  const void *fn = a.kv.key_scales ? (const void *)append_ext_kernel<E, I, true> : (const void *)append_ext_kernel<E, I, false>;
  return hipLaunchKernel(fn, dim3(runs, kShares), dim3(kThreads), args, 0, s);
}

}  // namespace

hipError_t launch_append_ext(const AppendArgs &a, bool half, bool in_f32, hipStream_t s) {
  if (half) return in_f32 ? launch<_Float16, float>(a, s) : launch<_Float16, _Float16>(a, s);
  return in_f32 ? launch<__bf16, float>(a, s) : launch<__bf16, __bf16>(a, s);
}

}  // namespace moecache
