// Scales of the delta rule's operands (delta_rule.hip): powers of two, found in the exponent fields of floats, apart from
// device code so that a CPU can go through all of them.
#pragma once

#include <stdint.h>

#include "lstm_int_math.h"

namespace lstm_int {

// 2^e, -126 <= e <= 127
LSTM_HD float power_of_two(int e) {
  union { uint32_t u; float f; } v;
  v.u = (uint32_t)(e + 127) << 23;
  return v.f;
}
// exponent of a number by its bits (without sign); -126 below the normal range
LSTM_HD int exponent_of(uint32_t bits) {
  const int e = (int)(bits >> 23);
  return (e > 1 ? e : 1) - 127;
}

// What the largest of an operand's row or column is brought to: just below what fp16 holds, so that the floor of its numbers,
// 2^-24, is as far below the largest as it can be; less for keys, whose scale is lost to the other operand of K' u.
constexpr int kTop = 14, kKeyTop = 2;

// scale and 1 / scale, powers of two, that bring numbers whose largest has these bits (without sign) to 2^top .. 2^(top + 1);
// those below 2^(top - 126) not all the way
struct Scale {
  float up, down;
};
template <int top>
LSTM_HD Scale scale_of(uint32_t bits) {
  const uint32_t low = (uint32_t)(top + 1) << 23, high = 254u << 23, e = bits & 0x7f800000u;
  union { uint32_t u; float f; } up, down;
  down.u = e < low ? low : e > high ? high : e;
  up.u = ((uint32_t)(254 + top) << 23) - down.u;
  down.u -= (uint32_t)top << 23;
  return {up.f, down.f};
}

// A column of the state is kept times 2^e: the largest that is kept of it, in that scale, and the largest factor of the keys in
// what is added to it, as it is, by their bits (0: nothing), neither infinite.  What e becomes: the larger one of what is kept
// and added comes to 2^11 .. 2^12, as far as e stays within -kUp .. kUp.  2^e and 2^-e are floats, and so is whatever a float
// of the column is in that scale.
constexpr int kUp = 120;
LSTM_HD int next_exponent(int e, uint32_t kept, uint32_t added) {
  const int k = kept ? exponent_of(kept) : -1000, a = added ? exponent_of(added) + e + kKeyTop : -1000;
  const int next = e + 11 - (k > a ? k : a);
  return next > kUp ? kUp : next < -kUp ? -kUp : next;
}

// whole * 2^d for |d| <= 2 kUp, at most 2^127: what is kept of a column, at a new scale.  A column of nothing may have any.
LSTM_HD float scaled_whole(float whole, int d) {
  const float v = whole * power_of_two(d / 2) * power_of_two(d - d / 2);
  return v < 0x1p127f ? v : 0x1p127f;
}

}  // namespace lstm_int
