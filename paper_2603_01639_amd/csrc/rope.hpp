// The cosine and sine of a rotary angle.
#pragma once

#include "ltd_device.hpp"

namespace ltd {
namespace {

// cos and sin of pos * freq, times m.
//
// A float32 angle is off by pos * freq * 2^-24: 0.06 radians a million tokens
// out.  The angle is taken in revolutions in float64 instead, as the unrounded
// product of pos and freq / 2 pi (two parts of it, with the product's rounding
// recovered by an fma), reduced exactly to within an eighth of a revolution of
// a multiple of a quarter, and only then made float32.  There the Taylor sums
// to x^9 and x^10 are off by at most 2e-9.
__device__ __forceinline__ float2 rope_turn(int64_t pos, double freq, float m) {
  constexpr double kInv2Pi = 0.15915494309189535, kInv2PiLow = -9.839338337591243e-18;
  const double c1 = freq * kInv2Pi;
  const double c2 = __builtin_fma(freq, kInv2Pi, -c1) + freq * kInv2PiLow;
  const double p = static_cast<double>(pos);
  const double whole = p * c1;
  const double rest = __builtin_fma(p, c1, -whole) + p * c2;
  const double frac = (whole - __builtin_rint(whole)) + rest;  // revolutions, within about a half
  const double quarter = __builtin_rint(4.0 * frac);
  const float x = static_cast<float>((frac - 0.25 * quarter) * 6.283185307179586);
  const float x2 = x * x;
  float s = __builtin_fmaf(x2, 1.f / 362880, -1.f / 5040);
  s = __builtin_fmaf(x2, s, 1.f / 120);
  s = __builtin_fmaf(x2, s, -1.f / 6);
  s = __builtin_fmaf(x2 * x, s, x);
  float c = __builtin_fmaf(x2, -1.f / 3628800, 1.f / 40320);
  c = __builtin_fmaf(x2, c, -1.f / 720);
  c = __builtin_fmaf(x2, c, 1.f / 24);
  c = __builtin_fmaf(x2, c, -0.5f);
  c = __builtin_fmaf(x2, c, 1.f);
  const int q = static_cast<int>(quarter) & 3;
  const float cq = (q & 1) ? s : c, sq = (q & 1) ? c : s;
  return make_float2(m * ((q == 1 || q == 2) ? -cq : cq), m * ((q & 2) ? -sq : sq));
}

}  // namespace
}  // namespace ltd
