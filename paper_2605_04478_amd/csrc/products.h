// What the operators of a training step's computation share on the host: limits, alignment, the join of split sums.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ccld.h"

namespace ccld {

constexpr int DEPTH = 64;              // contractions are divided in whole multiples of it
constexpr uint64_t COMPUTE_UNITS = 256;
constexpr int64_t MAX_ROWS = (int64_t)1 << 31, MAX_EXPERTS = (int64_t)1 << 20, MAX_WIDTH = (int64_t)1 << 22;
// a tile's last row starts below 2^31 bytes from its first: 256 rows (or DEPTH of them) of this many 16-bit elements, and a row
constexpr int64_t MAX_LD = ((int64_t)1 << 22) - ((int64_t)1 << 14);

// How a product is cut: the tiles (tiles.h) and the parts of the contraction, whose sums are joined.
//
// Tiles of 256 x 256, one to a compute unit, or of 128 x 128, two to one.  A step of 32 of the contraction takes 0.77 us in the former (8192^3: 1,390
// TFLOP/s) and 0.5 us in the latter (1,084), a tile's start and end 10 and 6 us, and sums of parts move at 4.5 TB/s.  The smaller tiles win
// where the larger ones would leave compute units idle: the weights of 12 experts, 1,000 x 1,336 each, are 288 tiles of 256 (48 us) or 1,056 of
// 128 (38 us).  (Tiles of 256 x 128, two to a compute unit, were between the two in every case but one, by less than a tenth.)  Operands that pass through
// registers need too many of them beside the sums of 256 x 256 (dx and dw of 43 experts of 600 x 3,728, 504 rows each, not aligned, 398 and 413 us in the larger
// tiles and 311 and 296 in the smaller ones; 4 of 4,096 x 4,096, 4,096 rows each, y, dx and dw 1,090, 1,379 and 1,278, and 1,079, 1,012 and 988).  counted: the numbers of tiles are what they will be, not what ragged rows are expected to give.
enum Tile { LARGE, MEDIUM, SHORT, FEW, NARROW };
inline uint32_t tile_m(Tile t) { return t == LARGE ? 256 : t == MEDIUM || t == SHORT ? 128 : 32; }
inline uint32_t tile_n(Tile t) { return t == LARGE ? 256 : t == NARROW ? 32 : 128; }
// a launch has less than 2^32 threads
inline int64_t most_groups(int threads) { return ((int64_t)1 << 32) / threads - 1; }
inline bool launches(Tile t, uint64_t groups) { return groups <= (uint64_t)most_groups(t == LARGE || t == MEDIUM ? 512 : t == NARROW ? 128 : 256); }
struct Cut { Tile tile; uint32_t splits; };
inline Cut choose_cut(double tiles_256, double tiles_128, uint64_t steps, double results, bool counted, bool direct, uint32_t most_splits = 16) {
  const struct { Tile tile; double tiles, at_once, start, step; } forms[] = {{MEDIUM, tiles_128, 2 * COMPUTE_UNITS, 6, 0.5},
                                                                             {LARGE, tiles_256, COMPUTE_UNITS, 10, 0.77}};
  Cut best{MEDIUM, 1};
  double least = 1e300;
  for (const auto& f : forms) {
    if (f.tile == LARGE && !direct) continue;
    for (uint32_t s = 1; s <= most_splits && (s == 1 || steps / s >= 16); s *= 2) {
      double rounds = f.tiles * s / f.at_once;
      if (rounds < 0.7) rounds = 1;
      else if (rounds < 4) rounds = counted ? (double)(int64_t)(rounds + 0.999) : rounds + 0.35;
      const double us = rounds * (f.start + (double)((steps + s - 1) / s) * f.step) + (s > 1 ? 4 + results * (8.0 * s + 2) / 4.5e6 : 0);
      if (us < least) { least = us; best = Cut{f.tile, s}; }
    }
  }
  return best;
}
inline uint64_t parts_of(uint64_t n, uint64_t by) { return (n + by - 1) / by; }
// rows x cols of results, of as many products
inline Cut choose_cut(uint64_t rows, uint64_t cols, uint64_t depth, bool direct, uint32_t most_splits = 16, uint64_t products = 1) {
  return choose_cut((double)products * parts_of(rows, 256) * parts_of(cols, 256), (double)products * parts_of(rows, 128) * parts_of(cols, 128),
                    parts_of(depth, 32), (double)products * rows * cols, true, direct, most_splits);
}
// Gradients of weights, n x k of them from so many rows.  Few steps are bound by writing the results: three small workgroups to a compute unit, so
// that some write while others load (64 experts of 1,024 x 2,048: 2 rows each 47 us, 53 in the larger tiles and 58 in those of 128 x 128; 64 rows 57, 65
// and 72).  With more steps that holds for ragged rows, as routing leaves them, where there are neither many results nor so few that the contraction
// is better taken in parts.  dw alone in small workgroups and else, rows spread like exp(0.7 N): 16 experts of 1,024 x 1,024 at 8 steps on average 22 and 25 us, at 20
// 46 and 50, at 32 64 and 72; 16 of 1,024 x 2,048 at 13 48 and 57; 43 of 224 x 888 at 8 20 and 29, at 20 47 and 60; 12 of 1,336 x 1,000 at 13 34 and 34.  Beyond 20 steps
// more results lose: 32 of 1,024 x 1,024 at 20 74 and 71, at 32 112 and 99; so do equal rows at any number: 16 of 1,024 x 1,024 at 8 20 and 18, at 20 35 and 28.  (The
// host does not know the rows.)
inline Cut choose_weight_cut(uint64_t n, uint64_t k, uint64_t rows, bool direct, uint64_t products = 1) {
  const uint64_t tiles = products * parts_of(n, 128) * parts_of(k, 128), steps = parts_of(rows, 32);
  const bool few = steps <= 4 || (steps <= 20 && tiles >= 2 * COMPUTE_UNITS);
  if (direct && (steps <= 2 || (few && tiles <= 12 * COMPUTE_UNITS))) return Cut{SHORT, 1};
  return choose_cut(n, k, rows, direct, 16, products);
}

// Where the number of tiles is known on the device only, the parts of their contraction are chosen there (tiles.h).
constexpr uint32_t MOST_SPLITS = 64, MOST_PIECES = 2 * (uint32_t)COMPUTE_UNITS;

inline bool aligned(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
inline ccld_status launched() { return hipGetLastError() == hipSuccess ? CCLD_OK : CCLD_E_HIP; }

// out[r][c] = sum over the splits, in their order, of part[s][r][c] (join.hip)
void launch_join(const float* part, uint32_t splits, uint64_t rows, uint64_t cols, void* out, int64_t ldo, int32_t dtype,
                 hipStream_t stream);

}  // namespace ccld
