// Angles of the position rotation as integers (host).
#pragma once
#include <cmath>

namespace provip {

// Turns a position as a fraction of 2^64, from radians a position of at most 1e6 either way: f / (2 pi) with a product
// in two doubles (1 / (2 pi) as two as well), of which only the fraction counts at whole positions. Of the magnitude, as the
// fraction of a small negative number is close to one and would be rounded; the other way round is the negative
// integer. Off by one unit at most, so by 2^-33 of a turn at every 32-bit position.
inline unsigned long long turns_of(double f) {
  const double hi = 0x1.45f306dc9c883p-3, lo = -0x1.6b01ec5417056p-57;  // 1 / (2 pi)
  const double x = std::fabs(f), t = x * hi, rest = std::fma(x, hi, -t) + x * lo;
  const double frac = t - std::floor(t);  // exact, below 1
  const unsigned long long n = (unsigned long long)(frac * 0x1p64) + (unsigned long long)(long long)(rest * 0x1p64);
  return f < 0. ? 0ull - n : n;
}

}  // namespace provip
