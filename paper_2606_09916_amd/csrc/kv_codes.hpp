// 8-bit codes as bf16 matrix operands. Both codes are exact in bf16: an int8 has 7
// significant bits, an E4M3 value 4.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "attend.hpp"

namespace ikv {

typedef __bf16 bf16x8_k __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_k __attribute__((ext_vector_type(2)));
typedef float f32x4_k __attribute__((ext_vector_type(4)));

// Two values exact in bf16, packed (the upper halves of their float32 bits).
__device__ __forceinline__ uint32_t pack_exact(float lo, float hi) {
  return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ float int8_at(uint32_t w, int byte) { return float(int8_t(w >> (8 * byte))); }
template <bool HI> __device__ __forceinline__ uint32_t e4m3_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI));
}

// 4 adjacent E4M3 codes of a word times a power of two -> 4 bf16, exactly.
__device__ __forceinline__ uint2 e4m3_scaled4(uint32_t w, float scale) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true)));
}

// Whether a scale is anything but a normal power of two: those are 0 .. 253 once the exponent is
// rotated down, less one; a mantissa, a sign, zero and what is not finite lie above.
__device__ __forceinline__ bool no_power(float scale) {
  const uint32_t t = __float_as_uint(scale) - 0x00800000u;
  return (t >> 23 | t << 9) > 253u;
}

// The same times any scale, each product rounded to bf16; NaN where the scale is not finite.
__device__ __forceinline__ uint2 e4m3_times4(uint32_t w, float scale) {
  if (!(fabsf(scale) < INFINITY)) return make_uint2(0x7fc07fc0u, 0x7fc07fc0u);
  bf16x2_k y[2];
  y[0][0] = __bf16(__builtin_amdgcn_cvt_f32_fp8(w, 0) * scale);
  y[0][1] = __bf16(__builtin_amdgcn_cvt_f32_fp8(w, 1) * scale);
  y[1][0] = __bf16(__builtin_amdgcn_cvt_f32_fp8(w, 2) * scale);
  y[1][1] = __bf16(__builtin_amdgcn_cvt_f32_fp8(w, 3) * scale);
  return make_uint2(__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1]));
}

// 4 adjacent codes of a word -> 4 bf16.
template <int FMT> __device__ __forceinline__ uint2 codes4(uint32_t w) {
  if constexpr (FMT == KV_E4M3) return make_uint2(e4m3_pair<false>(w), e4m3_pair<true>(w));
  else return make_uint2(pack_exact(int8_at(w, 0), int8_at(w, 1)), pack_exact(int8_at(w, 2), int8_at(w, 3)));
}

// One word of two rows (4 adjacent channels each) -> for each of the 4 channels, the bf16
// pair (row a, row b).
template <int FMT> __device__ __forceinline__ void codes_across(uint32_t a, uint32_t b, uint32_t (&o)[4]) {
  if constexpr (FMT == KV_E4M3) {
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x05010400u), hi = __builtin_amdgcn_perm(b, a, 0x07030602u);
    o[0] = e4m3_pair<false>(lo);
    o[1] = e4m3_pair<true>(lo);
    o[2] = e4m3_pair<false>(hi);
    o[3] = e4m3_pair<true>(hi);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = pack_exact(int8_at(a, i), int8_at(b, i));
  }
}

// bf16 values that are not finite, by pairs. Zero weights of rows that do not see an entry would
// turn them into NaN, so where some row does not, the product takes the pair without them, and
// they are added afterwards to the sums of the rows that do.
__device__ __forceinline__ bool odd_low(uint32_t w) { return (w & 0x7f80u) == 0x7f80u; }
__device__ __forceinline__ bool odd_high(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ uint32_t bf16_finite(uint32_t w) {
  return (odd_low(w) ? 0u : w & 0xffffu) | (odd_high(w) ? 0u : w & 0xffff0000u);
}
// The same for 4 E4M3 codes of a word, whose only value that is not finite is NaN, 0x7f and 0xff:
// 0x80 in each such byte. (0x7f + 1 stays within its byte.)
__device__ __forceinline__ uint32_t e4m3_nans(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t e4m3_finite(uint32_t w, uint32_t nans) { return w & ~(nans | (nans - (nans >> 7))); }

}  // namespace ikv
