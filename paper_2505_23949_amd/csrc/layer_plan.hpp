// How tsenor_product divides a product between its kernels: host code that needs no GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace tsenor_dev {

constexpr int kCus = 256;

// How the rows of a and b from m0 and n0 on are multiplied.
enum Kind { kNoColumns, kFewRows, kSmallTile, kTile, kTilePairs, kWideTile, kLargeTile };
struct Part {
  Kind kind;
  int64_t m0, n0, m, n;
  int tiles_m, tiles_n, splits;
  double us;  // estimated
};
struct Plan {
  int count;
  Part parts[2];
  size_t workspace;
};
struct Cost {
  Kind kind;
  int rows_m, rows_n;
  double step, around;
  int at_once;  // workgroups that run at a time, a whole number of rounds of them unless `fluid`
  bool fluid;
};
// The kind that takes least by measured us of a step (a block of 128 columns) and of what is around the steps of a tile (first loads,
// results).  Whole calls, us (rows of a x rows of b x columns), by tiles of
//   64 x 128 / 128 x 128 / the same, two workgroups to a CU / 256 x 128 / 256 x 256:
//     48 x 14336 x 4096        13 / 16 / - / 26 / -          512 x 4096 x 4096       14 / 16 / - / 24 / 37
//     1024 x 4096 x 8192       47 / 33 / 43 / 43 / 68        1999 x 4096 x 14336     170 / 120 / 115 / 106 / 145
//     2327 x 6544 x 1413       40 / 39 / 33 / 47 / 48        2048 x 4096 x 512       13 / 13 / 11 / 11 / 14
//     4096 x 4096 x 4096       101 / 72 / 62 / 63 / 54       8192 x 8192 x 128       54 / 59 / 39 / 46 / 36
//     7569 x 8229 x 920        147 / 127 / 96 / 102 / 88     14336 x 4096 x 8192     733 / 485 / 475 / 393 / 357
// Where the small tiles leave CUs idle, workgroups share the columns of a tile; what they leave costs 0.025 us each to write and add,
// and a launch: 48 x 4096 x 14336 alone 35, two 22, four 16.5, six (its choice) 16.1-16.6, eight 17.5; 128 x 4096 x 14336 35, 23, 19.
// Up to 16 rows of a need no tiles: 1, 8 and 16 x 4096 x 14336 12.7, 14.0 and 15.7 (shared tiles 16); 16 x 4096 x 4096 8 (11); but 16 x
// 14336 x 4096 18 where unshared tiles take 13, and 16 x 28672 x 8192 58 (51).  (Weights that no cache holds: 1, 8 and
// 16 x 14336 x 4096 15, 16.6 and 19, tiles 17.)
//
// What does not fill a round of large or wide tiles can go to a launch of its own, with the kind that takes least for it (us, one
// launch and two): 4096 x 14336 x 4096 222, 207 (large tiles, then wide ones); 5000 x 5000 x 5000 143, 134 (then 128 x 128); 14336 x
// 4096 x 8192 413, 407 (power is what counts there); but 5000 x 5000 x 2000 59.8, 65.3.
constexpr double kSecond = 5.0;  // us that a second launch has to save
inline Part part_of(const Cost& c, int64_t m0, int64_t n0, int64_t m, int64_t n, int64_t blocks) {
  const int64_t tiles_m = (m + c.rows_m - 1) / c.rows_m, tiles_n = (n + c.rows_n - 1) / c.rows_n, tiles = tiles_m * tiles_n;
  const double steps = (double)blocks * c.step;
  double us;
  if (c.fluid) {
    const double share = (double)tiles / c.at_once;
    us = std::max(0.5 + 0.5 * share, share) * (steps + c.around);
  } else {
    // (large tiles on fewer CUs have more of the L2 and of the power each: 128 of 256 x 256 take 1.15 us a step)
    const int64_t rest = tiles % c.at_once;
    const double fill = c.kind == kSmallTile ? 1.0 : 0.6 + 0.4 * (double)rest / c.at_once;
    us = (double)(tiles / c.at_once) * (steps + c.around) + (rest ? steps * fill + c.around : 0.0);
  }
  int64_t splits = 1;
  if (c.kind == kSmallTile)
    for (int64_t k = 2; k <= blocks && k * tiles <= kCus; ++k) {
      const double shared = (double)((blocks + k - 1) / k) * c.step + c.around + 1.0 + 0.025 * (double)(k * tiles);
      if (shared < us) us = shared, splits = k;
    }
  return {c.kind, m0, n0, m, n, (int)tiles_m, (int)tiles_n, (int)splits, us};
}

constexpr Cost kWide = {kWideTile, 256, 128, 0.85, 4.0, kCus, false}, kLarge = {kLargeTile, 256, 256, 1.45, 6.0, kCus, false};

// the kind that takes least for all rows from m0 and n0 on
inline Part part_of(int64_t m0, int64_t n0, int64_t m, int64_t n, int64_t blocks) {
  const bool few = (m + 63) / 64 * ((n + 127) / 128) <= kCus, pairs = (m + 127) / 128 * ((n + 127) / 128) > kCus;
  Part best = part_of({kSmallTile, 64, 128, few ? 0.25 : 0.36, 1.5, kCus, false}, m0, n0, m, n, blocks);
  if (m <= 8 || (m <= 16 && best.splits > 1)) {
    best.kind = kFewRows, best.splits = 1;
    return best;
  }
  for (const Cost& c : {pairs ? Cost{kTilePairs, 128, 128, 0.91, 3.0, 2 * kCus, true} : Cost{kTile, 128, 128, 0.41, 2.8, kCus, false}, kWide, kLarge}) {
    const Part part = part_of(c, m0, n0, m, n, blocks);
    if (part.us < best.us) best = part;
  }
  return best;
}

// rows of a and of b, blocks of 128 columns
inline Plan plan_of(int64_t m, int64_t n, int64_t blocks) {
  if (m == 0 || n == 0) return {};
  if (blocks == 0) return {1, {{kNoColumns, 0, 0, m, n, 0, 0, 1, 0.0}}, 0};
  Plan best = {1, {part_of(0, 0, m, n, blocks)}, 0};
  double least = best.parts[0].us;
  for (const Cost& c : {kWide, kLarge}) {
    const int64_t tiles_m = (m + c.rows_m - 1) / c.rows_m, tiles_n = (n + c.rows_n - 1) / c.rows_n;
    const int64_t whole = tiles_m * tiles_n / kCus * kCus;  // tiles of the whole rounds
    for (int of_b = 0; of_b < 2; ++of_b) {
      const int64_t m1 = of_b ? m : whole / tiles_n * c.rows_m, n1 = of_b ? whole / tiles_m * c.rows_n : n;
      if (m1 <= 0 || n1 <= 0 || m1 > m || n1 > n || (m1 == m && n1 == n)) continue;
      const Part first = part_of(c, 0, 0, m1, n1, blocks);
      const Part rest = of_b ? part_of(0, n1, m, n - n1, blocks) : part_of(m1, 0, m - m1, n, blocks);
      if (first.us + rest.us + kSecond < least) best = {2, {first, rest}, 0}, least = first.us + rest.us + kSecond;
    }
  }
  for (int k = 0; k < best.count; ++k)
    if (best.parts[k].splits > 1)
      best.workspace = (size_t)best.parts[k].splits * best.parts[k].tiles_m * best.parts[k].tiles_n * 64 * 128 * sizeof(float);
  return best;
}

}  // namespace tsenor_dev
