// Angles as fractions of a turn in units of 2^-64.  Host code only.
#pragma once

#include <stdint.h>
#include <string.h>

namespace fsx {

// freq / 2 pi turns, modulo a turn, in units of 2^-64, rounded to nearest; |freq| <= 2^20.
// freq is m 2^e with a whole m of 53 bits.  1 / 2 pi is floor(2^128 / 2 pi) units of 2^-128 here, off by less than one, so of at most
// 2^84 units of 2^-64 the product is off by less than 2^-44: what is left is the rounding, 2^-65 of a turn.  (A product of 64 bits is off
// by 2^20 times as much where freq is 2^20, and that again by the position.)
inline uint64_t turn_per_step(double freq) {
  constexpr uint64_t HIGH = 0x28be60db9391054aull, LOW = 0x7f09d5f47d4d3770ull;
  uint64_t u;
  memcpy(&u, &freq, 8);
  const uint64_t m = (u & ((1ull << 52) - 1)) | 1ull << 52;
  const int e = (int)((u >> 52) & 0x7FF) - 1075;
  // m / 2 pi in units of 2^-128: three words
  const unsigned __int128 a = (unsigned __int128)m * LOW, b = (unsigned __int128)m * HIGH + (uint64_t)(a >> 64);
  const uint64_t word[3] = {(uint64_t)a, (uint64_t)b, (uint64_t)(b >> 64)};
  const int shift = 64 - e;  // 2^e of it in units of 2^-64: bits from `shift` on, 96 at least
  if (shift > 182) return 0;  // less than a half (zero and subnormal frequencies too)
  const auto bits = [&](int at) {  // the 64 bits from `at` on
    const int i = at / 64, r = at % 64;
    const uint64_t low = i < 3 ? word[i] : 0, high = i < 2 ? word[i + 1] : 0;
    return r ? (low >> r) | (high << (64 - r)) : low;
  };
  const uint64_t turn = bits(shift) + (bits(shift - 1) & 1);
  return freq < 0 ? -turn : turn;
}

}  // namespace fsx
