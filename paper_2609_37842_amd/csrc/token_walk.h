// How a worker of the rotation kernels goes through its tokens.
#pragma once
#include <stdint.h>

namespace eogp {

// Tokens first, first + step, ... below n, 64 of them at a time. The last group's successor lies up to 64 steps past the
// end: beyond 31 bits for n near 2^31, so the place is 64 bits wide.
struct TokenWalk {
  int64_t first;
  int step, n;
  constexpr TokenWalk(int from, int by, int tokens) : first(from - 64 * (int64_t)by), step(by), n(tokens) {}
  // The next group; false at the end.
  constexpr bool next() {
    first += 64 * (int64_t)step;
    return first < n;
  }
  // Token k of the group, and whether it is one.
  constexpr int64_t at(int k) const { return first + (int64_t)k * step; }
  constexpr bool has(int k) const { return at(k) < n; }
};

}  // namespace eogp
