// Sines and cosines of RoPE angles p * base^(-2j/d_h) (App. B.1.1).  The angle is formed and reduced to [-pi/4, pi/4] in
// fp64 (pi/2 in two parts), then comes a Taylor series and the quadrant.  Good for angles up to 2^40: every position at a
// base of 1 or more (rope_angles_small).
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>

namespace gta {

// Frequencies are at most 1.  A smaller base is accepted, but its frequencies grow up to base^-1 and leave the range of
// the reduction: such calls keep to kernels that call the library's sine.
inline bool rope_angles_small(int rope, double base) { return !rope || base >= 1.0; }

// p * f = x + quadrant * pi/2
__device__ __forceinline__ double rope_reduce(int p, double f, int &quadrant) {
  const double ang = (double)p * f, k = rint(ang * 0.6366197723675814);
  quadrant = (int)(k - 4.0 * floor(k * 0.25));   // 0 .. 3
  return fma(-k, 6.123233995736766e-17, fma(-k, 1.5707963267948966, ang));
}

// (cos, sin) rounded once from fp64: the series to degree 11 / 12 (the first terms left out are below 1e-11).  For fp32
// rows and tables.
__device__ __forceinline__ float2 rope_cos_sin(int p, double f) {
  int q;
  const double x = rope_reduce(p, f, q), y = x * x;
  const double s = fma(x * y, fma(y, fma(y, fma(y, fma(y, -1. / 39916800., 1. / 362880.), -1. / 5040.), 1. / 120.), -1. / 6.), x);
  const double c = fma(y, fma(y, fma(y, fma(y, fma(y, fma(y, 1. / 479001600., -1. / 3628800.), 1. / 40320.), -1. / 720.), 1. / 24.), -0.5), 1.);
  const float a = (float)(q & 1 ? c : s), b = (float)(q & 1 ? s : c);
  return make_float2((q + 1) & 2 ? -b : b, q & 2 ? -a : a);
}

// the same for any angle (tables)
__device__ __forceinline__ float2 rope_cos_sin_any(int p, double f) {
  const double ang = (double)p * f;
  if (fabs(ang) < 0x1p40) return rope_cos_sin(p, f);
  double s, c;
  sincos(ang, &s, &c);
  return make_float2((float)c, (float)s);
}

// rope_cos_sin with the series in fp32, to degree 9 / 10 (the first terms left out are below 2e-9 and 2e-10): largest error
// 5.8e-8 against 3.0e-8.  For rows that are rounded to bf16.
__device__ __forceinline__ float2 rope_cos_sin_short(int p, double f) {
  int q;
  const float r = (float)rope_reduce(p, f, q), r2 = r * r;
  const float s = fmaf(r * r2, fmaf(r2, fmaf(r2, fmaf(r2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), r);
  const float c = fmaf(r2, fmaf(r2, fmaf(r2, fmaf(r2, fmaf(r2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  return make_float2((q + 1) & 2 ? -b : b, q & 2 ? -a : a);
}

// base^(-2j/d_h) for the pairs j < n, base at least 1: products in long double, each rounded once to fp64 (its error before that is below
// 2^-56 at n = 128; 0.5 us for 128 of them, a power each takes the host 2).
inline void rope_freqs(double base, int dh, int n, double *freq) {
  const long double ratio = powl((long double)base, -2.0L / dh);
  long double f = 1.0L;
  for (int j = 0; j < n; ++j, f *= ratio) freq[j] = (double)f;
}

// Angles as fractions of a turn in 64 bits: position p times the fraction that one position turns by, modulo 2^64, is exact but
// for the fraction's own error, for any sign of p and any frequency.  Fractions of the pairs j < n, base^(-2j/d_h) / (2 pi): products
// of integers where they fall (each within 2^-57 of a turn at n = 128, 2^-26 of one at the last position there is), in long double
// (10 us for 64 of them) where base is below 1 and they grow past a turn.
inline void rope_turns(double base, int dh, int n, uint64_t *turn) {
  const long double per_radian = 0.15915494309189533576888376337251436203L, two64 = 18446744073709551616.0L;
  const long double ratio = powl((long double)base, -2.0L / dh);
  if (ratio < 1.0L) {
    const uint64_t r = (uint64_t)(ratio * two64);
    turn[0] = (uint64_t)(per_radian * two64);
    for (int j = 1; j < n; ++j) turn[j] = (uint64_t)(((unsigned __int128)turn[j - 1] * r + ((uint64_t)1 << 63)) >> 64);
    return;
  }
  long double t = per_radian;
  for (int j = 0; j < n; ++j, t *= ratio) turn[j] = (uint64_t)((t - floorl(t)) * two64);
}

// (cos, sin) of p positions: the quadrant is in the upper bits, the rest becomes an angle in [-pi/4, pi/4] in fp32 (two roundings)
// for the series of rope_cos_sin_short.  No fp64: 3.6 of 19 us of a norm over 21 600 tokens were the reduction in fp64.  Largest
// error 9.7e-8 against 3.0e-8 of rope_cos_sin: for rows that are rounded to bf16.
__device__ __forceinline__ float2 rope_cos_sin_turn(int p, uint64_t turn) {
  const unsigned f = (unsigned)(((uint64_t)(int64_t)p * turn) >> 32), q = (f + 0x20000000u) >> 30;
  const float r = (float)(int)(f - (q << 30)) * 1.4629180792671596e-9f, r2 = r * r;   // 2 pi / 2^32
  const float s = fmaf(r * r2, fmaf(r2, fmaf(r2, fmaf(r2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), r);
  const float c = fmaf(r2, fmaf(r2, fmaf(r2, fmaf(r2, fmaf(r2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const float a = q & 1 ? c : s, b = q & 1 ? s : c;
  return make_float2((q + 1) & 2 ? -b : b, q & 2 ? -a : a);
}

}  // namespace gta
