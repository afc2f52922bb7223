// Frequencies as turns: host code of the rotary handles.
#pragma once

#include <cmath>
#include <cstdint>

namespace libra {

// theta / 2 pi mod 1 in units of 2^-64 (nearest), for |theta| < 2^20.  The quotient's whole
// turns, up to 18 bits, come before the fraction's 64, so that a floating-point quotient would
// lose as many of them; here the 64-bit mantissa is multiplied by 2^192 / 2 pi as integers.
inline uint64_t rotary_turns(long double theta) {
  constexpr uint64_t kInvTwoPi[3] = {0x36d8a5664f10e410, 0x7f09d5f47d4d3770, 0x28be60db9391054a};
  int e = 0;
  const uint64_t n = uint64_t(std::ldexp(std::frexp(std::fabs(theta), &e), 64));
  // |theta| = n 2^(e - 64); p = n 2^192 / 2 pi, and the turns are p 2^(e - 256).
  unsigned __int128 carry = 0;
  uint64_t p[4];
  for (int i = 0; i < 3; ++i) {
    carry += static_cast<unsigned __int128>(n) * kInvTwoPi[i];
    p[i] = uint64_t(carry);
    carry >>= 64;
  }
  p[3] = uint64_t(carry);
  // In units of 2^-64 that is p / 2^shift with shift = 192 - e > 128: the upper half has it all.
  const int shift = 192 - e;
  if (shift > 256) return 0;
  const unsigned __int128 upper = static_cast<unsigned __int128>(p[3]) << 64 | p[2];
  const uint64_t t = uint64_t(((upper >> (shift - 129)) + 1) >> 1);
  return theta < 0 ? 0 - t : t;
}

}  // namespace libra
