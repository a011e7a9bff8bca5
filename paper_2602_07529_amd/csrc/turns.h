// Angles of rotary positions.
#pragma once
#include <stdint.h>

#include <hip/hip_runtime.h>

// Cosine and sine of x turns: the nearest quarter is taken off exactly, and what is left, an angle y of at most pi / 4, goes through the
// Taylor series (the terms left out are below 2e-14 there).  A library call for any angle takes three times as long.
template <typename T>
__device__ __forceinline__ void cos_sin_of_turns(double x, T* c, T* s) {
  const double quarter = rint(4. * x), y = fma(-0.25, quarter, x) * 6.283185307179586477, z = y * y;
  double sn = 1. / 6227020800., cs = -1. / 87178291200.;
  sn = fma(sn, z, -1. / 39916800.);
  sn = fma(sn, z, 1. / 362880.);
  sn = fma(sn, z, -1. / 5040.);
  sn = fma(sn, z, 1. / 120.);
  sn = fma(sn, z, -1. / 6.);
  sn = fma(sn * z, y, y);
  cs = fma(cs, z, 1. / 479001600.);
  cs = fma(cs, z, -1. / 3628800.);
  cs = fma(cs, z, 1. / 40320.);
  cs = fma(cs, z, -1. / 720.);
  cs = fma(cs, z, 1. / 24.);
  cs = fma(cs, z, -0.5);
  cs = fma(cs, z, 1.);
  const int k = (int)((int64_t)quarter & 3);
  const T u = (T)(k & 1 ? sn : cs), v = (T)(k & 1 ? cs : sn);
  *c = k == 1 || k == 2 ? -u : u;
  *s = k >= 2 ? -v : v;
}
