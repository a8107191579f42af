// The search for a number that enough of a wave's numbers reach (log probabilities' alternatives).
#pragma once

#include <cstdint>

#include <hip/hip_runtime.h>

namespace spp {

// A number that at least c of some numbers reach, and no more than c + c / 4 + 1 of them unless equal ones leave no
// choice.  count(m): how many reach m; lo is the least of them, hi the largest, below 2^32 - 1, at least c there are.
//
// Seven halvings of what lies between lo and hi do it for most rows, with no branch; where many octaves lie between
// them (a few values of both signs behind a mask) it is halved to 2^17 numbers, a 64th of an octave; then by how many
// reach the number alone.  How close two logits are would not do: a row's common offset and its spread change
// nothing in its probabilities, and at 300 all of a row's largest may lie within 2^17 numbers.
// (A row of 128256 with 20 alternatives 8.8 us at any offset, of 4096 with 8 6.0; by 2^17 numbers alone 8.7 and 6.1, and at
// an offset of 300 41 and 7.8, of 1000 41 and 223.)
template <typename Count>
__device__ inline uint32_t narrow_floor(uint32_t lo, uint32_t hi, int c, Count count) {
  ++hi;  // (the least number that too few reach, so far)
#pragma unroll
  for (int k = 0; k < 7; ++k) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const bool enough = count(mid) >= c;
    lo = enough ? mid : lo;
    hi = enough ? hi : mid;
  }
  const int most = c + c / 4 + 1;
  int n = count(lo);
  while (hi - lo > 0x20000 || (n > most && hi - lo > 1)) {
    const uint32_t mid = lo + (hi - lo) / 2;
    const int reach = count(mid);
    if (reach >= c) {
      lo = mid;
      n = reach;
    } else {
      hi = mid;
    }
  }
  return lo;
}

}  // namespace spp
