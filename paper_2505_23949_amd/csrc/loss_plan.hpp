// Which tiles the products of the losses are made in, and how many workgroups share the sum of a tile: host code that needs no GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "layer_plan.hpp"

namespace tsenor_dev {

constexpr int kMaxSplits = 128;
struct ProductPlan {
  Kind kind;  // kSmallTile (64 rows of a x 128 of b), kTile and kTilePairs (128 x 128), kWideTile (256 x 128), kLargeTile (256 x 256)
  int tiles_m, tiles_n, splits;
  double us;  // estimated
  size_t workspace;
};

// m rows of a, n of b, `blocks` of 64 columns of the sum; `logits`: they need whole sums, so that parts are joined by one workgroup to a tile
inline ProductPlan product_plan(int64_t m, int64_t n, int64_t blocks, bool logits, Kind only = kNoColumns) {
  ProductPlan best = {kSmallTile, 0, 0, 1, 0.0, 0};
  if (m == 0 || n == 0) return best;
  for (const Cost& c : {Cost{kSmallTile, 64, 128, 0.42, 3.0, kCus, false}, Cost{kTile, 128, 128, 0.585, 4.0, kCus, false},
                        Cost{kTilePairs, 128, 128, 1.085, 4.5, 2 * kCus, true}, Cost{kWideTile, 256, 128, 0.86, 6.0, kCus, false},
                        Cost{kLargeTile, 256, 256, 1.556, 9.0, kCus, false}}) {
    if (only != kNoColumns && c.kind != only) continue;
    const int64_t tiles_m = (m + c.rows_m - 1) / c.rows_m, tiles_n = (n + c.rows_n - 1) / c.rows_n, tiles = tiles_m * tiles_n;
    const int64_t most = logits ? (c.rows_m * c.rows_n <= 128 * 128 ? 16 : 1) : kMaxSplits;
    for (int64_t splits = 1; splits <= std::min<int64_t>(most, std::max<int64_t>(blocks / 4, 1)); ++splits) {
      if (splits > 1 && (splits - 1) * tiles >= c.at_once) break;
      const double steps = (double)((blocks + splits - 1) / splits) * c.step;
      const int64_t groups = tiles * splits, rounds = groups / c.at_once, rest = groups % c.at_once;
      // (the last round: fewer workgroups have more of the memory and of the power each; of two on a CU, one alone takes 0.7 of the time)
      const double fill = c.fluid ? (rest <= kCus ? 0.7 : 1.0) : 0.75 + 0.25 * (double)rest / c.at_once;
      double us = (double)rounds * (steps + c.around) + (rest ? steps * fill + c.around : 0.0);
      const double parts = splits > 1 ? (double)groups * c.rows_m * c.rows_n * 4.0 : 0.0;
      if (splits > 1) us += 4.0 + 2.0 * parts / 5.0e6 + (logits ? 0.5 : 0.1) * (double)splits;
      if (best.us == 0.0 || us < best.us) best = {c.kind, (int)tiles_m, (int)tiles_n, (int)splits, us, (size_t)parts};
    }
  }
  return best;
}

// The head's gradient: what does not fill a round of large or wide tiles can go to a launch of its own (us of the kernels, one launch and two:
// 50257 x 1024 x 1433 175, XXX).
struct HeadPlan {
  int count;
  int64_t rows[2];
  ProductPlan parts[2];
};
inline HeadPlan head_plan(int64_t m, int64_t n, int64_t blocks) {
  const ProductPlan whole = product_plan(m, n, blocks, false);
  HeadPlan best = {1, {m, 0}, {whole, {}}};
  double least = whole.us;
  for (int rows_n : {128, 256}) {
    const int64_t tiles_m = (m + 255) / 256, tiles_n = (n + rows_n - 1) / rows_n, rounds = tiles_m * tiles_n / kCus;
    const int64_t m1 = tiles_n ? rounds * kCus / tiles_n * 256 : 0;
    if (m1 <= 0 || m1 >= m) continue;
    const ProductPlan first = product_plan(m1, n, blocks, false), rest = product_plan(m - m1, n, blocks, false);
    if (first.us + rest.us + 4.0 < least) best = {2, {m1, m - m1}, {first, rest}}, least = first.us + rest.us + 4.0;
  }
  return best;
}

// Both gradients in one launch, with tiles of one kind: a launch less, and the one fills the CUs that the other leaves idle.  (us of the
// call: fp32 645 x 401 x 320 69, 58 so, 84 x 1856 x 711 44, 40.)
struct BothPlan {
  bool use;
  ProductPlan dh, dweight;
};
inline BothPlan both_plan(int64_t tokens, int64_t vocab, int64_t width, int64_t blocks_dh, int64_t blocks_dweight, double apart) {
  BothPlan best = {};
  double least = apart;
  for (Kind kind : {kSmallTile, kTile}) {
    const ProductPlan a = product_plan(tokens, width, blocks_dh, false, kind), b = product_plan(vocab, width, blocks_dweight, false, kind);
    const double groups_a = (double)a.tiles_m * a.tiles_n * a.splits, groups_b = (double)b.tiles_m * b.tiles_n * b.splits;
    const double us = groups_a + groups_b <= kCus ? std::max(a.us, b.us) : a.us + b.us;
    if (us < least) best = {true, a, b}, least = us;
  }
  return best;
}

}  // namespace tsenor_dev
