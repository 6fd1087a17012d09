// Cosine and sine of a token's position times a frequency, and pairs of channels turned by them.  Not part of the C ABI.
#pragma once
#include "common.h"

namespace ptq {

struct CosSin { double c, s; };

// scale cos, scale sin of position * freq.  The product is kept exactly, as the sum of two float64, and brought to [-pi/4, pi/4] with pi/2
// in two parts: what is left is off by 2^-52 of itself and, for up to 2^31 quarter turns, 2^-66 or so.  Then Taylor's series,
// whose first term left out is below 2^-53 (of sin r: 2^-54 r; r <= 0.786).  A frequency that is not finite gives NaN.
__device__ __forceinline__ CosSin cos_sin(int position, double freq, double scale) {
  const double p = (double)position, hi = p * freq, lo = fma(p, freq, -hi);
  const double n = rint(hi * 0.63661977236758134308);   // 2 / pi
  double r = fma(-n, 1.57079632679489655800, hi);       // pi / 2 to 53 bits: an exact difference
  r += fma(-n, 6.12323399573676603587e-17, lo);         // the next 53
  const double z = r * r;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;   // 1 / 15!, 1 / 16!
  s = fma(s, z, 1.0 / 6227020800.0);
  c = fma(c, z, -1.0 / 87178291200.0);
  s = fma(s, z, -1.0 / 39916800.0);
  c = fma(c, z, 1.0 / 479001600.0);
  s = fma(s, z, 1.0 / 362880.0);
  c = fma(c, z, -1.0 / 3628800.0);
  s = fma(s, z, -1.0 / 5040.0);
  c = fma(c, z, 1.0 / 40320.0);
  s = fma(s, z, 1.0 / 120.0);
  c = fma(c, z, -1.0 / 720.0);
  s = fma(s, z, -1.0 / 6.0);
  c = fma(c, z, 1.0 / 24.0);
  s = fma(s * z, r, r);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quarter = (int)fma(-4.0, floor(n * 0.25), n);   // 0 .. 3 while n is a whole number below 2^53
  const double c1 = quarter & 1 ? s : c, s1 = quarter & 1 ? c : s;
  return CosSin{scale * ((quarter + 1) & 2 ? -c1 : c1), scale * (quarter & 2 ? -s1 : s1)};
}

// (a, b) turned, in float64 and rounded to float32
__device__ __forceinline__ void turn(float& a, float& b, const CosSin& t) {
  const double x = a, y = b;
  a = (float)fma(x, t.c, -(y * t.s));
  b = (float)fma(x, t.s, y * t.c);
}

}  // namespace ptq
