// fp64 <-> bf16 on the device, with a single rounding to nearest even.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fademem {

// fp64 -> fp32 with round-to-odd: the hardware conversion rounds to
// nearest; if that moved away from zero, step back one ulp (truncation),
// then set the last bit when the conversion was inexact.  Rounding the
// result to bf16 to nearest even then equals a single correct rounding of
// x to bf16, because fp32 carries 16 more significand bits than bf16.
__device__ __forceinline__ float f64_to_f32_odd(double x) {
  const float f = float(x);
  const double xd = double(f);
  uint32_t b = __float_as_uint(f);
  b -= (fabs(xd) > fabs(x)) ? 1u : 0u;
  b |= (xd != x) ? 1u : 0u;
  return __uint_as_float(b);
}

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// Two fp64 values -> packed bf16x2 (low half = lo), each rounded to nearest even.
__device__ __forceinline__ uint32_t pack_bf16_rne(double lo, double hi) {
  bf16x2_t v;
  v[0] = (__bf16)f64_to_f32_odd(lo);
  v[1] = (__bf16)f64_to_f32_odd(hi);
  return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ double bf16_lo(uint32_t w) { return double(__uint_as_float(w << 16)); }
__device__ __forceinline__ double bf16_hi(uint32_t w) { return double(__uint_as_float(w & 0xffff0000u)); }

}  // namespace fademem
