// Index arithmetic of the generation kernels that has to hold up to the largest sizes that are accepted.  Plain functions of
// integers, without a device type: a host program evaluates them at those sizes.
#pragma once

namespace ac {

// A ring's first entry, taken modulo its n entries (n up to 2^31 - 1).
constexpr int ring_first(int first, int n) {
  const int f = first % n;
  return f < 0 ? f + n : f;
}

// Blocks of a run where `waves` waves share `total` of them (below 2^31 - 65536).  Runs of one block as long as every second wave has
// none: more partial results cost the join more than the runs save (one request of 8,000 tokens of 8 heads of 128, 2,016 blocks
// for 2,048 waves: 18.6 us, runs of two 16.9; of 2,000 tokens 11.7 / 13.2).
constexpr int run_length(int total, int waves) {
  if (total <= waves / 2) return 1;
  const int even = (total + waves - 1) / waves;
  return even > 2 ? even : 2;
}

// The partial result in which wave w leaves its part of the unit whose first block is `from`: the second of its two if its
// run begins no later than the unit.  (Of a wave that has a part: the number of its run's first block is below 2^31 then.)
constexpr int partial_of(int w, int per, int from) {
  return 2 * w + (w * per <= from);
}

// Consecutive rows of a wave where at most `most` waves share `rows` of them (below 2^31 - 65536).
constexpr int rows_of_a_wave(int rows, int most) {
  return rows > most ? (rows - 1) / most + 1 : 1;
}

// Rows of a workgroup of the page plan, B requests of S slots: some 1,024 slots (256 x 1,024 5.3 us, 2,048 6.2; 2,000 x 500 24.6, 512
// 27.0), but no more than 16,384 workgroups, since each sums all requests before its own: of 2^22 requests a row each had 10^13 to look at.
// (rows * S stays below 2^31.  More than kPlanSlots slots a row: several workgroups share it if it is the only one.)
constexpr int kPlanSlots = 1024, kPlanRowsMost = 256, kPlanWgsMost = 16384;
constexpr int plan_rows(int B, int S) {
  const int few = S >= kPlanSlots ? 1 : S * kPlanRowsMost <= kPlanSlots ? kPlanRowsMost : kPlanSlots / S;
  const int share = (B - 1) / kPlanWgsMost + 1;
  return share > few && (long long)share * S < (1 << 30) ? share : few;
}

}  // namespace ac
