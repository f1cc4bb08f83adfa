// Index arithmetic of the generation kernels that has to hold up to the largest sizes that are accepted.  Plain functions of
// integers, without a device type: a host program evaluates them at those sizes.
#pragma once

namespace ac {

// A ring's first entry, taken modulo its n entries (n up to 2^31 - 1).
constexpr int ring_first(int first, int n) {
  const int f = first % n;
  return f < 0 ? f + n : f;
}

}  // namespace ac
