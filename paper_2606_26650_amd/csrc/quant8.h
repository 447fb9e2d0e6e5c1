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

// rne(x / s) as a float.  The product with the reciprocal differs from the quotient
// by less than 127 * 2^-22 = 3e-5, so the two round alike unless the product is that
// near to a half: only then (and where 1/s overflows: the test fails for a NaN) is
// the quotient formed.  |x| <= 127 s up to one rounding of a normal s, so only the
// quotient by a subnormal s (1/s overflows) can need the clamp.  0 for s = 0 and for
// a NaN scale.
struct Quant8 {
  float s, inv;
  __device__ __forceinline__ explicit Quant8(float scale)
      : s(scale > 0.f ? scale : 1.0f), inv(scale > 0.f ? 1.0f / scale : 0.0f) {}
  __device__ __forceinline__ float operator()(float x) const {
    const float t = x * inv;
    float r = rintf(t);
    if (!(fabsf(t - r) <= 0.4999f)) r = inv > 0.f ? fminf(fmaxf(rintf(x / s), -127.f), 127.f) : 0.f;
    return r;
  }
};

// Four codes (floats within +-127) as bytes, the first lowest.
__device__ __forceinline__ unsigned int pack_codes(float a, float b, float c, float d) {
  return ((unsigned)(int)a & 0xffu) | (((unsigned)(int)b & 0xffu) << 8) |
         (((unsigned)(int)c & 0xffu) << 16) | ((unsigned)(int)d << 24);
}

}  // namespace catq
