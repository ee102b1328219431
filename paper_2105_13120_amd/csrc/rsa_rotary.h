// Rotation by position, shared by the ring's rows (rsa_rotate.hip) and the cache's new tokens (rsa_cache.hip).
#pragma once
#include "rsa_common.h"

namespace rsa {

// How the first R elements of a head are paired, and the angles per position.
struct Rotary {
  int R, adjacent;        // R = 0: nothing is turned
  const float *inv_freq;  // R / 2
  float sign;             // -1: the transposed rotation
};

// cos and sin of pos * freq, the angle taken as the exact product: of the turns pos * freq / (2 pi) only the fraction
// counts, which 24 bits lose from position 10^4 on.  So the product and 1 / (2 pi) are two 53-bit words each:
// the fraction errs by less than 2^-50 of a turn at any position before it is rounded to fp32, once, as a number of at
// most one half; with the sine's own rounding the results err by less than 2^-22.
__device__ __forceinline__ float2 angle_of(int64_t pos, float freq) {
#pragma clang fp contract(off)  // (t is to be the rounded product, whose error te is)
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;  // 1 / (2 pi)
  const double n = (double)pos, f = (double)freq, p = n * f, pe = __builtin_fma(n, f, -p);
  const double t = p * hi, te = __builtin_fma(p, hi, -t) + __builtin_fma(p, lo, pe * hi);
  const float x = 2.f * (float)((t - __builtin_rint(t)) + te);
  return make_float2(cospif(x), sinpif(x));
}

}  // namespace rsa
