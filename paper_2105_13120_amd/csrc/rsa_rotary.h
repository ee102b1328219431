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

// The angle pos * freq in half turns, within one, taken as the exact product: of the turns pos * freq / (2 pi) only the fraction
// counts, which 24 bits lose from position 10^4 on.  So the product and 1 / (2 pi) are two 53-bit words each:
// the fraction errs by less than 2^-50 of a turn at any position.
__device__ __forceinline__ double half_turns_of(int64_t pos, float freq) {
#pragma clang fp contract(off)  // (t is to be the rounded product, whose error te is)
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;  // 1 / (2 pi)
  const double n = (double)pos, f = (double)freq, p = n * f, pe = __builtin_fma(n, f, -p);
  const double t = p * hi, te = __builtin_fma(p, hi, -t) + __builtin_fma(p, lo, pe * hi);
  return 2.0 * ((t - __builtin_rint(t)) + te);
}

// Its cosine and sine.  What the half turns' rounding to fp32 leaves, d, below 2^-25 of a half turn, turns the
// rounded one's cosine and sine by pi d, of which the first order is enough: without it a sine next to 0 at half a turn lost
// all its digits.  The results err by the functions' own rounding and one more.
__device__ __forceinline__ float2 angle_of(int64_t pos, float freq) {
#pragma clang fp contract(off)
  const double half_turns = half_turns_of(pos, freq);
  const float x = (float)half_turns, d = (float)(half_turns - (double)x) * 3.14159265f, c = cospif(x), s = sinpif(x);
  return make_float2(__builtin_fmaf(-s, d, c), __builtin_fmaf(c, d, s));
}

}  // namespace rsa
