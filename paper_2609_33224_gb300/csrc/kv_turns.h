// Frequencies of rotary positions as fractions of a turn: host code without CUDA, so that it can be tested alone.
#pragma once

#include <stdint.h>

#include <cmath>

namespace pskv {

// A frequency as turns per position, in 2^-64 of a turn.  The fraction is that of the magnitude, which loses nothing by it;
// a small negative number's distance to the whole turn below would be rounded.
inline uint64_t turns_of(double frequency) {
  double t = std::fabs(frequency) / 6.283185307179586476925;
  t -= std::floor(t);  // [0, 1)
  const double hi = std::floor(t * 0x1p32), lo = (t * 0x1p32 - hi) * 0x1p32;
  // a low part that rounds up to 2^32 carries, and a whole turn is none
  const uint64_t turns = ((uint64_t)hi << 32) + (uint64_t)std::nearbyint(lo);
  return frequency < 0.0 ? 0 - turns : turns;
}

}  // namespace pskv
