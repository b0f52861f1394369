// How far each pair of a rotary embedding turns per position (host code; include/eagle3.h: eagle3_rope_turns).
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>

// false: sizes or parameters without a meaning; nothing is written then.
inline bool rope_turns(int rot, double theta, int scaling, double factor, double low, double high, double original_len, double* out) {
  if (rot < 2 || rot % 2 || !(theta > 0) || !std::isfinite(theta) || scaling < 0 || scaling > 2) return false;
  if (scaling >= 1 && (!(factor > 0) || !std::isfinite(factor))) return false;
  if (scaling == 2 && (!(original_len > 0) || !std::isfinite(original_len) || !(low < high) || !std::isfinite(high - low))) return false;
  const double two_pi = 6.283185307179586476925286766559;
  auto turns = [&](int i) {
    double f = std::pow(theta, -2.0 * i / rot) / two_pi;
    if (scaling == 1) f /= factor;
    if (scaling == 2) {
      const double w = std::min(1.0, std::max(0.0, (original_len * f - low) / (high - low)));
      f *= w + (1 - w) / factor;
    }
    return f;
  };
  for (int i = 0; i < rot / 2; ++i)
    if (!(turns(i) < 0x1p992)) return false;                // position times turns has to be a number, for any int32 position
  for (int i = 0; i < rot / 2; ++i) out[i] = turns(i);
  return true;
}
