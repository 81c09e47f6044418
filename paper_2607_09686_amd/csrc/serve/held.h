// A cache of 8 bits: a head's vector x of one token is held as e4m3 numbers c_d and one power of two,
//
//   x_d ~ c_d 2^e,   e = ceil(log2(max |x_d| / 448)) within [lo, hi],   c_d = e4m3(x_d / 2^e)
//
// rounded to nearest even, |c_d| <= 448 (the type's largest); what is not finite is held as NaN and does not
// count for e.  The scale is a power of two because an e4m3 number keeps its relative precision under it (2^-4, as
// any scale would), the division is exact, and so is the product c 2^e in the queries' type: a number of 4
// significant bits.  The limits keep it a normal number there (in fp16, whose numbers end sooner, any number):
// bf16 2^-109 to 448 2^119, fp16 2^-24 to 448 2^7 = 57344.  So attention over such a cache is attention over what
// a read of it gives, with no rounding of its own but where bf16 probabilities take values' powers of two and
// leave its normal numbers (p 2^e < 2^-126: a row is off by at most 2^-125 for each such token).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace moecache {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <class E>
constexpr int kLeastScale = __is_same(E, _Float16) ? 127 - 15 : 127 - 100;
template <class E>
constexpr int kMostScale = __is_same(E, _Float16) ? 127 + 7 : 127 + 119;

// e + 127 for the largest magnitude, which is finite: m 2^x / 448 = (m / 1.75) 2^(x - 8), 1 <= m < 2
template <class E>
__device__ __forceinline__ int scale_byte(float largest) {
  const int e = (int)((__float_as_uint(largest) + 0x1fffffu) >> 23) - 8;
  return min(max(e, kLeastScale<E>), kMostScale<E>);
}
// 2^e of e + 127.  255 is no scale; read as 254, it leaves rows alone that give it no weight.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(min(byte, 254u) << 23); }

// What counts for e of an element.
__device__ __forceinline__ float magnitude(float x) {
  const float a = fabsf(x);
  return a < __builtin_inff() ? a : 0.f;
}
// Four elements' numbers; inverse = 2^-e.
__device__ __forceinline__ uint32_t encode(float a, float b, float c, float d, float inverse) {
  const float v[4] = {a, b, c, d};
  float w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = fabsf(v[i]) < __builtin_inff() ? fminf(fmaxf(v[i] * inverse, -448.f), 448.f) : __builtin_nanf("");
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], r, true);
}
// Two numbers (the lower or upper half of four) times a power of two, exactly, in 16 bits.
__device__ __forceinline__ uint32_t decode(uint32_t v, bool upper, float scale, __bf16) {
  const bf16x2 r = upper ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, true)
                         : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, scale, false);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t decode(uint32_t v, bool upper, float scale, _Float16) {
  const f16x2 r = upper ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, scale, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, scale, false);
  return __builtin_bit_cast(uint32_t, r);
}
// Two numbers, each times a scale of its own.
__device__ __forceinline__ uint32_t decode2(uint32_t v, bool upper, float s0, float s1, __bf16) {
  const f32x2 f = upper ? __builtin_amdgcn_cvt_pk_f32_fp8(v, true) : __builtin_amdgcn_cvt_pk_f32_fp8(v, false);
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)(f[0] * s0), (__bf16)(f[1] * s1)});
}
__device__ __forceinline__ uint32_t decode2(uint32_t v, bool upper, float s0, float s1, _Float16) {
  const f32x2 f = upper ? __builtin_amdgcn_cvt_pk_f32_fp8(v, true) : __builtin_amdgcn_cvt_pk_f32_fp8(v, false);
  return __builtin_bit_cast(uint32_t, f16x2{(_Float16)(f[0] * s0), (_Float16)(f[1] * s1)});
}

}  // namespace
}  // namespace moecache
