// Rotary embedding shared by the cache-write kernels: frequencies, and cosine / sine of an angle at any position.
#pragma once
#include "common.cuh"

namespace mv {

// theta_i = base^(-2i/d) for i < d/2, evaluated once per launch on the host in double precision
struct ThetaTable {
  double theta[64];
};

// cos and sin of pos * theta, for |pos * theta| below 2^31 (the quadrant is counted in an int; positions of tables go up to
// 2^30 and theta is at most 1 for a base of at least 1).  The angle and its reduction to [-pi/4, pi/4] (two-term Cody-Waite with a
// 53-bit and a residual piece of pi/2, by fused multiply-adds) are double precision; the reduced angle is rounded to float and
// its cosine and sine come from the accurate float routine (no fast-math intrinsics).  Up to an angle of 2^25 both agree with the
// double-precision values to within two units in the last place of a float; beyond, what theta and the product lost as doubles shows
// as well: 2^-22 at 2^30 (against 80-bit arithmetic: 2^-23).  Six double-precision instructions per (token, i) instead of a
// double-precision sincos: with the latter the arithmetic, not HBM, bounded the kernel at prefill sizes.
__device__ __forceinline__ void rope_cos_sin(int pos, double theta, float& c, float& s) {
  constexpr double TWO_OVER_PI = 0.63661977236758134308;
  constexpr double PIO2_HI = 1.57079632679489655800e+00;  // pi/2 rounded to double
  constexpr double PIO2_LO = 6.12323399573676603587e-17;  // pi/2 - PIO2_HI
  const double a = double(pos) * theta;
  const double kf = rint(a * TWO_OVER_PI);
  double r = fma(-kf, PIO2_HI, a);
  r = fma(-kf, PIO2_LO, r);
  float sr, cr;
  sincosf(float(r), &sr, &cr);
  const int k = int(kf) & 3;  // quadrant: angle = r + k * pi/2
  const float ss = (k & 1) ? cr : sr, cc = (k & 1) ? sr : cr;
  s = (k & 2) ? -ss : ss;
  c = ((k + 1) & 2) ? -cc : cc;
}

// the table for head_dim d
inline ThetaTable theta_table(double rope_base, int d) {
  ThetaTable tt{};
  const double c = -2.0 * log2(rope_base) / double(d);
  for (int i = 0; i < d / 2; ++i) tt.theta[i] = exp2(double(i) * c);  // base^(-2i/d)
  return tt;
}

}  // namespace mv
