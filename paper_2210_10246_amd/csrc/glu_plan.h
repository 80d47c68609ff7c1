// Host arithmetic of the gated unit's products (no HIP in here).
#pragma once

#include <stdint.h>

namespace tempo {

// An operand that lies by k, rows of `n` elements, each a value of k's: pieces of 8 elements are loaded whole also where a row ends
// inside one.  The last piece of a row then ends in a later row, and that of the last rows would end behind the tensor: so many values
// of k, the last ones, are loaded element by element.  1 from 4 elements a row on, up to 7 of rows of one.
constexpr int ends_later(int n) { return n % 8 == 0 ? 0 : (8 - n % 8 + n - 1) / n; }
// Steps of `step` values of k that are loaded in whole pieces, of two operands that lie by k (n: elements of a row) or do not (n: 0).
constexpr int whole_steps(int k, int step, int a, int b) {
  const int of_a = a > 0 ? ends_later(a) : 0, of_b = b > 0 ? ends_later(b) : 0, left = k - (of_a > of_b ? of_a : of_b);
  return left > 0 ? left / step : 0;
}

}  // namespace tempo
