// Rotary positions, device side: a pair (a, b) of a head's dims turns by an angle that
// grows with the row's position,
//   (a, b) -> (a cos - b sin, b cos + a sin),  angle = 2 pi position turns[pair].
//
// The angle is a fraction of a turn, in 64 bits: at position 10^6 the fastest pair has
// made 160,000 turns, of which 32 bits would leave 0.016 (0.1 radian). A (row, pair) is
// one of these for all heads.
#pragma once

#include "q4_internal.h"

namespace oasis {
namespace {

__device__ __forceinline__ double2 rotary_cos_sin(const RotaryArgs& rot, long long position, int pair) {
  const double t = (double)position * rot.turns[pair];
  double s, c;
  sincospi(2.0 * (t - floor(t)), &s, &c);
  return make_double2(c * rot.cos_amplitude, s * rot.sin_amplitude);
}

}  // namespace
}  // namespace oasis
