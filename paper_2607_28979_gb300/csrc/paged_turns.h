// An angle in radians as a fraction of a turn, in units of 2^-64, by integers alone: a rate gives the same on every host.
#pragma once

#include <cmath>
#include <cstdint>

namespace mot {

// 1 / (2 pi) in units of 2^-192, the upper word first, from its decimal digits: (d1 + (d2 + ..) / 10) / 10 in long
// division. 63 digits are good to 2^-206; every step cuts off below a unit, which the tenths behind it make 1.2 in all.
struct InverseTwoPi {
  uint64_t w[3];
  constexpr InverseTwoPi() : w{0, 0, 0} {
    constexpr char digits[] = "159154943091895335768883763372514362034459645740456448747667344";
    for (int i = int(sizeof(digits)) - 2; i >= 0; --i) {
      unsigned __int128 rest = digits[i] - '0';
      for (uint64_t& x : w) {
        rest = rest << 64 | x;
        x = uint64_t(rest / 10);
        rest %= 10;
      }
    }
  }
};

// r / (2 pi) without its whole turns, in units of 2^-128, cut off (r finite, at most 2^16 either way): |r| = m 2^e with m
// a whole number below 2^53, so the product with the words above is exact, off by 2^(17 - 192) of a turn as they are.
inline unsigned __int128 turn128_of(double r) {
  constexpr InverseTwoPi inv;
  int e;
  const uint64_t m = uint64_t(std::ldexp(std::frexp(std::fabs(r), &e), 53));
  const int shift = 192 - 128 - (e - 53);   // of m inv, in units of 2^(e - 53 - 192), to units of 2^-128: 100 or more
  if (shift >= 246) return 0;               // m inv is below 2^246
  uint64_t p[6] = {0, 0, 0, 0, 0, 0}, carry = 0;   // m inv, the lowest word first
  for (int i = 0; i < 3; ++i) {
    const unsigned __int128 x = (unsigned __int128)(m) * inv.w[2 - i] + carry;
    p[i] = uint64_t(x);
    carry = uint64_t(x >> 64);
  }
  p[3] = carry;
  const int at = shift / 64, bit = shift % 64;
  auto word = [&](int i) { return bit ? p[i] >> bit | p[i + 1] << (64 - bit) : p[i]; };
  const unsigned __int128 turn = (unsigned __int128)(word(at + 1)) << 64 | word(at);
  return r < 0 ? 0 - turn : turn;
}

inline uint64_t rounded(unsigned __int128 turn) { return uint64_t((turn + (uint64_t(1) << 63)) >> 64); }
inline uint64_t turn_of(double r) { return rounded(turn128_of(r)); }
// A rate base^(-2 i / rot), 1 at most, in the host's widest type: two parts of 53 bits.
inline uint64_t turn_of(long double r) {
  const double hi = double(r);
  return rounded(turn128_of(hi) + turn128_of(double(r - hi)));
}

}  // namespace mot
