// What the operators of a training step's computation share on the host: limits, alignment, the join of split sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ccld.h"

namespace ccld {

constexpr int DEPTH = 64;              // contractions are divided in whole multiples of it
constexpr uint64_t COMPUTE_UNITS = 256;
constexpr uint64_t MAX_GROUPS = (uint64_t)1 << 22;      // workgroups of up to 1,024 threads in a launch
constexpr int64_t MAX_ROWS = (int64_t)1 << 31, MAX_EXPERTS = (int64_t)1 << 20, MAX_WIDTH = (int64_t)1 << 22;
// a tile's last row starts below 2^31 bytes from its first: 256 rows (or DEPTH of them) of this many 16-bit elements, and a row
constexpr int64_t MAX_LD = ((int64_t)1 << 22) - ((int64_t)1 << 14);

// How a product is cut: tiles of 256 x 256, one to a compute unit, or of 128 x 128, two to one, and the contraction in `splits` parts whose
// sums are joined.  A step of 32 of the contraction takes 0.77 us in the former (8192^3: 1,390 TFLOP/s) and 0.5 us in the latter (1,084), a tile's
// start and end 10 and 6 us, and sums of parts move at 4.5 TB/s.  The smaller tiles win where the larger ones would leave
// compute units idle: the weights of 12 experts, 1,000 x 1,336 each, are 288 tiles of 256 (48 us) or 1,056 of 128 (38 us); those of 64
// experts, 1,024 x 2,048 each and 128 rows on average, 98 us and 123.  counted: the numbers of tiles are what they will be, not what ragged rows are expected to give.
struct Cut { bool large; uint32_t splits; };
inline Cut choose_cut(double tiles_256, double tiles_128, uint64_t steps, double results, bool counted, uint32_t most_splits = 16) {
  Cut best{true, 1};
  double least = 1e300;
  for (int large = 1; large >= 0; --large)
    for (uint32_t s = 1; s <= most_splits && (s == 1 || steps / s >= 16); s *= 2) {
      double rounds = (large ? tiles_256 : tiles_128) * s / (double)(large ? COMPUTE_UNITS : 2 * COMPUTE_UNITS);
      if (rounds < 0.7) rounds = 1;
      else if (rounds < 4) rounds = counted ? (double)(int64_t)(rounds + 0.999) : rounds + 0.35;
      const double us = rounds * ((large ? 10 : 6) + (double)((steps + s - 1) / s) * (large ? 0.77 : 0.5)) + (s > 1 ? 4 + results * (8.0 * s + 2) / 4.5e6 : 0);
      if (us < least) { least = us; best = Cut{large != 0, s}; }
    }
  return best;
}

// Where the number of tiles is known on the device only, the parts of their contraction are chosen there (tiles.h).
constexpr uint32_t MOST_SPLITS = 64, MOST_PIECES = 2 * (uint32_t)COMPUTE_UNITS;

inline bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline ccld_status launched() { return hipGetLastError() == hipSuccess ? CCLD_OK : CCLD_E_HIP; }

// out[r][c] = sum over the splits, in their order, of part[s][r][c] (join.hip)
void launch_join(const float* part, uint32_t splits, uint64_t rows, uint64_t cols, void* out, int64_t ldo, int32_t dtype,
                 hipStream_t stream);

}  // namespace ccld
