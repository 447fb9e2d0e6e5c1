// The symmetric 8-bit quantizer of W1.58A8 on the device: code = rne(x / scale)
// within +-127, scale = max|x| / 127, in IEEE fp32.
#pragma once

#include "catq_internal.h"

namespace catq {

// Magnitudes are compared as integers: the order is that of |x|, an infinity is
// above every finite value and a NaN above that, so a maximum over the bits
// carries a non-finite value to the scale (fmaxf would drop a NaN).
__device__ __forceinline__ unsigned int mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ float quant8_scale(unsigned int mag) {
  return mag >= 0x7f800000u ? __builtin_nanf("") : __uint_as_float(mag) / 127.0f;
}

// N values to rne(x / s), as floats.  The product with the reciprocal differs from the
// quotient by less than 127 * 2^-22 = 3.03e-5, so the two round alike unless the product is that
// near to a half: only where one of them is (and where 1/s overflows: the test fails for
// a NaN) are the quotients formed.  |x| <= 127 s up to one rounding of a normal s, so only
// the quotient by a subnormal s can need the clamp.  0 for s = 0 and for a NaN scale.
template <int N>
__device__ __forceinline__ void quant8_n(float (&x)[N], float scale) {
  const bool some = scale > 0.f;
  const float s = some ? scale : 1.0f, inv = some ? 1.0f / scale : 0.0f;
  float r[N];
  bool near = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const float t = x[j] * inv;
    r[j] = rintf(t);
    near |= !(fabsf(t - r[j]) <= 0.49996f);
  }
  if (near) {
#pragma unroll
    for (int j = 0; j < N; ++j) r[j] = some ? fminf(fmaxf(rintf(x[j] / s), -127.f), 127.f) : 0.f;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = r[j];
}

// Four codes (floats within +-127) as bytes, the first lowest.
__device__ __forceinline__ unsigned int pack_codes(float a, float b, float c, float d) {
  return ((unsigned)(int)a & 0xffu) | (((unsigned)(int)b & 0xffu) << 8) |
         (((unsigned)(int)c & 0xffu) << 16) | ((unsigned)(int)d << 24);
}

}  // namespace catq
