// How a call of the losses is made: pieces, tiles of the products, workgroups that share the sum of a tile, and which way where there are
// several: host code that needs no GPU.
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

// The kind of tiles, and how many workgroups share a tile's sum, that take least by measured us of a step (64 columns) and of what is around the
// steps of a tile.  us of the kernels of tokens x vocab x width (bf16), no sum shared, by 64 x 128 / 128 x 128 / the same, two to a CU /
// 256 x 128 / 256 x 256:
//   logits  512 x 32000 x 4096  240 / 177 / 162 / 129 / 120      1433 x 50257 x 1024  302 / 212 / 184 / 183 / 166
//           1024 x 8192 x 512    25 /  20 /  18 /  16 /  23      4096 x 32768 x 4096  1867 / 1276 / 1103 / 988 / 856
//           128 x 16384 x 1024   11 /  11 /  16 /  16 /  28      4096 x 32000 x 256    298 / 201 / 151 / 161 / 132
//   dh      300 x 5003 x 4096    32 /  36 /  51 /  50 /  86      4096 x 32768 x 4096  1726 / 1204 / 1118 / 909 / 813
//   dW      300 x 5003 x 4096    50 /  30 /  25 /  26 /  27      1433 x 50257 x 1024   315 / 204 / 169 / 169 / 157
// Shared sums, and what adds them: dh of 1433 x 50257 x 1024 with 256 x 256 787 alone, 2 workgroups to a tile 393 + 6, 4 207 + 8, 8 139 + 12;
// logits of 71 x 768 x 6645 with 64 x 128 33 alone, 7 to a tile 8 + 11 (logits in larger tiles have no CUs left to share with).
// m rows of a, n of b, `blocks` of 64 columns of the sum; `logits`: they need whole sums, so that parts are joined by one workgroup to a tile
inline ProductPlan product_plan(int64_t m, int64_t n, int64_t blocks, bool logits, Kind only = kNoColumns) {
  ProductPlan best = {kSmallTile, 0, 0, 1, 0.0, 0};
  if (m == 0 || n == 0) return best;
  for (const Cost& c : {Cost{kSmallTile, 64, 128, 0.42, 3.0, kCus, false}, Cost{kTile, 128, 128, 0.585, 4.0, kCus, false},
                        Cost{kTilePairs, 128, 128, 1.085, 4.5, 2 * kCus, true}, Cost{kWideTile, 256, 128, 0.88, 5.5, kCus, false},
                        Cost{kLargeTile, 256, 256, 1.556, 8.0, kCus, false}}) {
    if (only != kNoColumns && c.kind != only) continue;
    const int64_t tiles_m = (m + c.rows_m - 1) / c.rows_m, tiles_n = (n + c.rows_n - 1) / c.rows_n, tiles = tiles_m * tiles_n;
    const int64_t most = logits ? (c.kind == kSmallTile ? 16 : 1) : kMaxSplits;
    for (int64_t splits = 1; splits <= std::min<int64_t>(most, std::max<int64_t>(blocks / 4, 1)); ++splits) {
      if (splits > 1 && (splits - 1) * tiles >= c.at_once) break;
      const double steps = (double)((blocks + splits - 1) / splits) * c.step;
      const int64_t groups = tiles * splits, rounds = groups / c.at_once, rest = groups % c.at_once;
      // (the last round: fewer workgroups have more of the memory and of the power each; of two on a CU, one alone takes 0.7 of the time)
      const double fill = c.fluid ? (rest <= kCus ? 0.7 : 1.0) : 0.75 + 0.25 * (double)rest / c.at_once;
      double us = (double)rounds * (steps + c.around) + (rest ? steps * fill + c.around : 0.0);
      const double parts = splits > 1 ? (double)groups * c.rows_m * c.rows_n * 4.0 : 0.0;
      if (splits > 1) us += 4.0 + parts / 4.0e6 + (logits ? 0.5 : 0.1) * (double)splits;  // (written and added up)
      if (best.us == 0.0 || us < best.us) best = {c.kind, (int)tiles_m, (int)tiles_n, (int)splits, us, (size_t)parts};
    }
  }
  return best;
}

// The head's gradient: what does not fill a round of large or wide tiles can go to a launch of its own (us of the kernels, one launch and two:
// 1433 x 50257 x 1024 157, 138 + 15; fp32 1000 x 5003 x 769 with both gradients 245, 231 in all).
struct HeadPlan {
  int count;
  int64_t rows[2];
  ProductPlan parts[2];
};
inline HeadPlan head_plan(int64_t m, int64_t n, int64_t blocks) {
  const ProductPlan whole = product_plan(m, n, blocks, false);
  HeadPlan best = {1, {m, 0}, {whole, {}}};
  double least = whole.us;
  for (int kind = 0; kind < 3; ++kind) {  // by tiles of 256 x 256, 256 x 128 and 128 x 128
    const int rows_m = kind == 2 ? 128 : 256, rows_n = kind == 0 ? 256 : 128;
    const int64_t tiles_m = (m + rows_m - 1) / rows_m, tiles_n = (n + rows_n - 1) / rows_n, rounds = tiles_m * tiles_n / kCus;
    const int64_t m1 = tiles_n ? rounds * kCus / tiles_n * rows_m : 0;
    if (m1 <= 0 || m1 >= m) continue;
    const ProductPlan first = product_plan(m1, n, blocks, false), rest = product_plan(m - m1, n, blocks, false);
    if (first.us + rest.us + 4.0 < least) best = {2, {m1, m - m1}, {first, rest}}, least = first.us + rest.us + 4.0;
  }
  return best;
}

// Both gradients in one launch, with tiles of one kind: a launch less, and the one fills the CUs that the other leaves idle.  (us of the
// call: fp32 645 x 401 x 320 69, 58-61 so, 84 x 1856 x 711 44, 40.)
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

// ---- a call ------------------------------------------------------------------------------------------------------------------
// Of dz (or, without gradients, 10 times the sums of the parts of tiles), of the hidden states, and of sums and entries: each.
constexpr int64_t kPieceBytes = (int64_t)1 << 31;
constexpr int kPieceRows = 256;                    // pieces are a multiple of this
constexpr int64_t kMostRows = (int64_t)1 << 22;    // (a grid has fewer than 2^32 threads; a row takes 256 of them)
constexpr int kPairs = 6;                          // of planes, that a product in single precision takes
constexpr int kFewTokens = 16, kFewWords = 16;     // of the kernel for few tokens: words of a workgroup
constexpr int kTileTokens = 64;                    // of the smallest tile
// Logits from which on dh alone is made without the pass that makes dz of the exponentials (4 bytes a logit at 4.8 TB/s, and a launch and the looks at
// c.refs for it): us of the call with the pass and without 512 x 32000 x 4096 (16 million) 273, 271, 4096 x 4096 x 4096 (17) 259, 267, 700 x 32000 x 2048
// (22) 223, 222, 1024 x 32000 x 1024 (33) 200, 184, 2048 x 32000 x 2048 with 8 entries (66) 525, 495, 2048 x 50257 x 1024 (103) 508, 446, 8192 x 16384 x
// 4096 (134) 1785, 1774, 4096 x 50264 x 2048 with 32 (206) 1603, 1485, 8192 x 32000 x 512 (262) 845, 670, 4096 x 128256 x 1024 (525) 2464, 2115.
constexpr int64_t kWithoutPass = 20000000;

// dh of up to kFewTokens from the head as it stands, in blocks of columns; `words` (whole lines of 64) to a workgroup, four workgroups to a CU
constexpr int kFewDhWords = 512, kFewDhColumns = 128;  // kFewDhWords: whose dz a workgroup holds at a time
struct FewDhPlan {
  int blocks, words, splits;  // splits: workgroups that share a block's words
  size_t workspace;
};
inline FewDhPlan few_dh_plan(int64_t tokens, int64_t vocab, int64_t width) {
  FewDhPlan plan = {1, 64, 1, 0};
  if (tokens == 0 || vocab == 0 || width == 0) return plan;
  plan.blocks = (int)((width + kFewDhColumns - 1) / kFewDhColumns);
  const int64_t most = std::max<int64_t>(4 * kCus / plan.blocks, 1), lines = (vocab + 63) / 64;
  plan.words = (int)((lines + most - 1) / most) * 64;
  plan.splits = (int)((vocab + plan.words - 1) / plan.words);
  plan.workspace = plan.splits > 1 ? (size_t)plan.splits * tokens * width * sizeof(float) : 0;
  return plan;
}

struct LossShape {
  int64_t tokens, vocab, width;
  bool bf16, dh, dweight;
  int k;            // entries of a token
  bool teacher;     // whether they have a teacher's logits
  bool in_place;    // whether products can read the head where it is
  bool states_too;  // and the hidden states, in whole lines
};
struct LossPlan {
  int64_t rows;  // of a piece
  ProductPlan logits, dh;
  HeadPlan dweight;
  BothPlan both;
  bool few;      // logits by the kernel for few tokens
  bool few_dh;   // and dh
  FewDhPlan dh_of_few;
  bool direct;   // no gather: rows are the tokens in their order
  bool counted;  // exponentials counted from a number for a row
  bool picked;   // several entries to a token, put in order for the tiles that they are in
  int row_threads;  // of the workgroup that goes through a token's sums and exponentials
  int tile_n, tiles;  // words of a part of a row's sums, such parts
};

inline LossPlan loss_plan(const LossShape& p) {
  LossPlan plan = {};
  const auto round_up = [](int64_t n, int64_t to) { return (n + to - 1) / to * to; };
  const bool gradients = p.dh || p.dweight;
  const int64_t parts = (p.vocab + 63) / 64, of_states = round_up(std::max<int64_t>(p.width, 1), 64) * (p.bf16 ? 2 : 6);
  const int64_t row_bytes = std::max({gradients ? parts * 64 * (p.bf16 ? 2 : 10) : parts * 8 * 10, of_states, parts * 10 + 8 * (int64_t)p.k + 8});
  const int64_t most = std::min(std::max<int64_t>(kPieceBytes / row_bytes / kPieceRows * kPieceRows, kPieceRows), kMostRows);
  const int64_t pieces = std::max<int64_t>((p.tokens + most - 1) / most, 1);
  plan.rows = std::min(round_up((p.tokens + pieces - 1) / pieces, kPieceRows), round_up(p.tokens, 16));

  const int64_t tokens = std::min(plan.rows, p.tokens), pairs = p.bf16 ? 1 : kPairs;
  const auto blocks = [&](int64_t n) { return (n + 63) / 64 * pairs; };
  plan.logits = product_plan(tokens, p.vocab, blocks(std::max<int64_t>(p.width, 1)), true);
  if (p.dh) plan.dh = product_plan(tokens, p.width, blocks(p.vocab), false);
  if (p.dweight) plan.dweight = head_plan(p.vocab, p.width, blocks(tokens));
  if (p.dh && p.dweight) {
    const double apart = plan.dh.us + plan.dweight.parts[0].us + plan.dweight.parts[1].us + 4.0 * plan.dweight.count;
    plan.both = both_plan(tokens, p.vocab, p.width, blocks(p.vocab), blocks(tokens), apart);
  }
  // Up to 16 tokens: straight from memory in fp32, where tiles would need a copy of the head that nothing else needs, or are few (us of the call:
  // 3 x 1216 x 2326 27.4, 10.4 so, 4 x 1650 x 6912 with dh 58.3, 39.6).  In whole lines, scores of 1 token and of 16 with 8 entries, tiles and so:
  //   4096 x 512  11.0, 8.6 and 12.5, 9.4     x 4096  18.9, 11.8 and 21.0, 15.2
  //   8192 x 512  10.9, 8.7 and 12.4, 10.2    x 4096  22.8, 18.9 and 24.8, 22.7
  //  12288 x 512  10.6, 9.6 and 12.5, 11.0    x 4096  25.8, 24.4 and 28.0, 29.5
  //  16384 x 512  11.1, 10.6 and 12.7, 12.1   x 4096  30.8, 29.7 and 32.5, 36.5
  //  32000 x 512  11.5, 12.8 and 13.1, 16.0   x 4096  44.4, 48.8 and 46.0, 64.6
  // 128256 x 512  34.8, 31.2 and 37.0, 40.1   x 4096  175, 186 and 177, 288
  plan.few = p.tokens <= kFewTokens && (!p.bf16 || p.vocab < 64 * kCus || !p.in_place);
  // dh likewise, where tiles would need that copy (us of the call, with copy and tiles and so: fp32 1 x 116621 x 5083 2553, 1096, 16 x 1000 x 513 31.8,
  // 25.3, bf16 2 x 4484 x 897 40.0, 30.6, 16 x 30001 x 1027 75.3, 77.2; without a need for the copy as well as tiles: bf16 3 x 4096 x 1024 24.0,
  // 20.9, 16 x 16000 x 4096 75.5, 79.2).
  plan.few_dh = plan.few && p.dh && !p.in_place;
  if (plan.few_dh) plan.dh_of_few = few_dh_plan(tokens, p.vocab, p.width), plan.dh = {}, plan.both = {};
  // A tile has 64 rows at the least: up to there, rows of tokens that are left out cost nothing, and the states are read where they are (48 x
  // 32000 x 4096 69 us, 57 so).
  plan.direct = !gradients && (plan.few || (p.in_place && p.states_too && p.tokens <= kTileTokens && plan.logits.kind == kSmallTile));
  // (few tokens and direct tiles look through all entries)
  plan.picked = p.teacher && p.k > 1 && !plan.few && !plan.direct;
  plan.tile_n = plan.few ? kFewWords : plan.logits.kind == kLargeTile ? 128 : 64;
  plan.tiles = (int)((p.vocab + plan.tile_n - 1) / plan.tile_n);
  // 1024 threads where there are few tokens with many words or several entries, a wave where a token has little to do, so that more of them wait at a time.
  // us of the call so and with 256 threads: 126 x 116032 x 128 with both gradients 83, 102, 100 x 32000 x 1024 with 8 entries 84, 89 (but scores, 1 x
  // 32000 x 2048 with 8, 26.2, 25.5); 7744 x 512 x 1216 91, 100, 4000 x 1500 x 256 with 64 entries 67, 74.
  plan.row_threads = tokens <= 2 * kCus && (p.k > 4 || plan.tiles > 1024) ? 1024 : tokens > 4 * kCus && p.vocab <= 2048 && p.k <= 64 ? 64 : 256;
  plan.counted = p.bf16 && p.dh && !p.dweight && !plan.few && plan.logits.kind == kLargeTile && plan.rows * p.vocab >= kWithoutPass;
  return plan;
}

}  // namespace tsenor_dev
