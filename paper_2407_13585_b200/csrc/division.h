// What the host works out for unsigned division by a constant of a run, without a divider and without a branch (Granlund and
// Montgomery's round-up multiplier, 33 bits with the add-and-shift fix-up): l = ceil(log2 d), m = floor(2^32 (2^l - d) / d) + 1,
// v / d = (t + ((v - t) >> min(l, 1))) >> max(l - 1, 0) with t = umulhi(v, m); d = 1 gives v.
#pragma once
#include <cstdint>

namespace acc {

struct Divisor {
  uint32_t d, mul, sh1, sh2;
};

inline Divisor divisor(uint32_t d) {
  uint32_t l = 0;
  while (l < 32 && (1ull << l) < d) ++l;
  const uint32_t sh1 = l < 1 ? l : 1;
  return {d, (uint32_t)((((1ull << l) - d) << 32) / d + 1), sh1, l - sh1};
}

}  // namespace acc
