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

// ---- rotary forms (mv_rope_form): which elements of a head make up a pair, and what is left alone
//
// A head is worked on in pieces: two vectors of W elements at lo and hi.  Pieces c = 0, W, 2 W, .. below half (the number of
// pairs) hold the pairs c .. c + W - 1: as halves, element first + i goes with first + half + i; as pairs, first + 2 i goes with its
// neighbour.  The pieces behind hold the elements outside the rotated part.  first and 2 half are multiples of 16, so no piece
// straddles a border for W up to 8.
struct FormTable {
  ThetaTable t;
  float amplitude;
  int first, half, pairs;  // pairs: 1 = neighbours, 0 = halves
};

inline bool form_ok(const mv_rope_form* f, int head_dim) {
  if (!f || (f->layout != MV_ROPE_HALVES && f->layout != MV_ROPE_PAIRS)) return false;
  if (f->first < 0 || f->rotary_dim < 16 || (f->first & 15) || (f->rotary_dim & 15) || f->rotary_dim > head_dim - f->first) return false;
  if (!(f->amplitude > 0.f) || !(f->amplitude <= 1024.f)) return false;
  for (int i = 0; i < f->rotary_dim / 2; ++i)
    if (!(f->theta[i] >= -1.0 && f->theta[i] <= 1.0)) return false;
  return true;
}
inline FormTable form_table(const mv_rope_form& f) {
  FormTable r{};
  for (int i = 0; i < f.rotary_dim / 2; ++i) r.t.theta[i] = f.theta[i];
  r.amplitude = f.amplitude;
  r.first = f.first;
  r.half = f.rotary_dim / 2;
  r.pairs = f.layout == MV_ROPE_PAIRS ? 1 : 0;
  return r;
}

struct Piece {
  int lo, hi;
  bool turns;
};
template <int W>
__device__ __forceinline__ Piece piece_at(const FormTable& f, int c) {
  if (c < f.half) return f.pairs ? Piece{f.first + 2 * c, f.first + 2 * c + W, true} : Piece{f.first + c, f.first + f.half + c, true};
  const int u = 2 * (c - f.half), e = u < f.first ? u : u + 2 * f.half;
  return Piece{e, e + W, false};
}
// One pair turned.  The roundings are spelt out, so that every kernel that turns the same pair gets the same bits.
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
  const float x = a;
  a = __fmaf_rn(x, c, -__fmul_rn(b, s));
  b = __fmaf_rn(b, c, __fmul_rn(x, s));
}
// the pairs of a piece turned; cs, sn: cosines and sines of pair c and those behind it (amplitude included)
template <int W>
__device__ __forceinline__ void turn_piece(bool pairs, float (&lo)[W], float (&hi)[W], const float* cs, const float* sn) {
  if (pairs) {
#pragma unroll
    for (int n = 0; n < W; n += 2) {
      turn_pair(lo[n], lo[n + 1], cs[n / 2], sn[n / 2]);
      turn_pair(hi[n], hi[n + 1], cs[W / 2 + n / 2], sn[W / 2 + n / 2]);
    }
  } else {
#pragma unroll
    for (int n = 0; n < W; ++n) turn_pair(lo[n], hi[n], cs[n], sn[n]);
  }
}

// the table for head_dim d
inline ThetaTable theta_table(double rope_base, int d) {
  ThetaTable tt{};
  const double c = -2.0 * log2(rope_base) / double(d);
  for (int i = 0; i < d / 2; ++i) tt.theta[i] = exp2(double(i) * c);  // base^(-2i/d)
  return tt;
}

}  // namespace mv
