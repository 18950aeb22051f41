// cos and sin of the rotary embedding's angles.  Internal to the library; plain arithmetic, so that a host build of it
// can be checked over the whole range.
#pragma once
#include <math.h>
#include <stdint.h>

namespace forge {

// cos and sin of an angle 0 <= a < 2^31 in fp64: quadrant by two-part reduction (both products are
// exact in the fused multiply-add; what pi / 2 still lacks is below 1e-32 per turn), Taylor series up to
// x^15 / x^16 on [-pi/4, pi/4] (truncated below 1e-16).  Rounded to fp32 once, like the library call it stands
// for, which takes three times the registers and twice the instructions (for arguments that no position
// reaches).
__host__ __device__ inline void cos_sin(double a, float& cosine, float& sine) {
  const double n = rint(a * 0.63661977236758134308);                     // 2 / pi
  double x = __builtin_fma(n, -1.5707963267948966192, a);               // pi / 2 rounded to fp64 ...
  x = __builtin_fma(n, -6.123233995736766036e-17, x);                   // ... and what that rounding dropped
  const double z = x * x;
  double s = -1.0 / 1307674368000.0, c = 1.0 / 20922789888000.0;
  s = __builtin_fma(s, z, 1.0 / 6227020800.0);
  s = __builtin_fma(s, z, -1.0 / 39916800.0);
  s = __builtin_fma(s, z, 1.0 / 362880.0);
  s = __builtin_fma(s, z, -1.0 / 5040.0);
  s = __builtin_fma(s, z, 1.0 / 120.0);
  s = __builtin_fma(s, z, -1.0 / 6.0);
  s = __builtin_fma(s * z, x, x);
  c = __builtin_fma(c, z, -1.0 / 87178291200.0);
  c = __builtin_fma(c, z, 1.0 / 479001600.0);
  c = __builtin_fma(c, z, -1.0 / 3628800.0);
  c = __builtin_fma(c, z, 1.0 / 40320.0);
  c = __builtin_fma(c, z, -1.0 / 720.0);
  c = __builtin_fma(c, z, 1.0 / 24.0);
  c = __builtin_fma(c, z, -0.5);
  c = __builtin_fma(c, z, 1.0);
  const int q = (int)n & 3;
  const double co = (q & 1) ? s : c, si = (q & 1) ? c : s;
  cosine = (float)(q == 1 || q == 2 ? -co : co);
  sine = (float)(q >= 2 ? -si : si);
}

// The angle position * increment in units of 2^-64 turns, modulo whole turns: its top 32 bits.
__host__ __device__ inline uint32_t turned(int32_t position, uint64_t increment) {
  const uint32_t p = (uint32_t)position, lo = (uint32_t)increment, hi = (uint32_t)(increment >> 32);
  const uint32_t carry = (uint32_t)((uint64_t)p * lo >> 32);
  return p * hi + carry - (position < 0 ? lo : 0u);        // (a negative position counts 2^32 too many)
}

// cos and sin of `top` 2^-32 parts of a full turn, in fp32: the nearest quarter from the top bits, the rest in
// [-pi/4, pi/4], Taylor series up to x^9 / x^10 (truncated below 2e-9).  Largest error 1.2e-7 with the 2^-32 turns that `turned` drops.
__host__ __device__ inline void turn_cos_sin(uint32_t top, float& cosine, float& sine) {
  const uint32_t quarter = (top + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(top - (quarter << 30)) * 1.4629180792671596e-9f;    // 2 pi / 2^32
  const float z = x * x;
  float s = 2.7557319e-6f, c = -2.7557319e-7f;
  s = __builtin_fmaf(s, z, -1.9841270e-4f);
  s = __builtin_fmaf(s, z, 8.3333333e-3f);
  s = __builtin_fmaf(s, z, -1.6666667e-1f);
  s = __builtin_fmaf(s * z, x, x);
  c = __builtin_fmaf(c, z, 2.4801587e-5f);
  c = __builtin_fmaf(c, z, -1.3888889e-3f);
  c = __builtin_fmaf(c, z, 4.1666667e-2f);
  c = __builtin_fmaf(c, z, -0.5f);
  c = __builtin_fmaf(c, z, 1.0f);
  const float co = (quarter & 1u) ? s : c, si = (quarter & 1u) ? c : s;
  cosine = ((quarter + 1u) & 2u) ? -co : co;       // quarters 1 and 2 of 0 .. 3 (4 is 0)
  sine = (quarter & 2u) ? -si : si;
}

}  // namespace forge
