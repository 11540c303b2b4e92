// What the kernels of the losses (tsenor_loss.h) share.
//
// A call goes through its tokens in pieces:
//   order     (once) the tokens that count in front, those left out behind them: the products then have no rows for nothing
//   gather    the piece's hidden states, one behind the other; outputs of those left out are cleared
//   logits    z = h W^T in tiles: of each tile's rows the largest logit and the sum of exponentials, and, where gradients are wanted,
//             the exponentials; the logits of entries, and of a token's only one not its exponential in the sum
//   rows      for each token: the sums of its tiles joined, its loss; the exponentials become dz
//   products  dh = dz W, dW = dz^T h
// How many tokens count is known on the GPU only.  Grids are made for all of them, and workgroups without work end at once.
//
// The exponential of a target (or of a teacher's only entry) stays apart from the sum of all others, `rest`, until the end: loss = log(1 + rest / own),
// and the gradient of its logit is -rest / (rest + own).  Of a word that a model has learned both are small, and as lse - z and p - 1 they would be what is
// left of numbers thousands of times as large; and its logit is the one that the sum would have had, from the same product.  (Losses of 1e-6 to
// 0.1, 8192 words of width 512 to 37543 of 64: from a second product and lse - z up to 4.6e-6 off, which can be more than all of one, and some below 0; at
// most 3.9e-6 of itself off so, none below 0.  Scores of many tokens pay for the look at their words, 4096 x 32000 x 64 78 us, 84.6, x 256 106, 112.)
#pragma once
#include "layer.hpp"
#include "loss_plan.hpp"
#include "tile_loads.hpp"
#include "tsenor_loss.h"

namespace tsenor_dev {

struct LossCall {
  const void *h, *weight;
  int64_t h_ld, weight_ld;
  const int64_t* ids;
  const void* teacher;     // logits of the entries; NULL: one entry to a token, of weight 1
  int64_t ids_ld, teacher_ld;
  int teacher_bf16, k;
  float inverse_temperature, scale;  // scale: 1 / (temperature ln 2), logits to exponents of 2
  const float* dloss;
  float *loss, *lse;
  void *dh, *dweight;
  int tokens, vocab, width;
  // workspace
  int* count;              // tokens that count; NULL: the rows are the tokens in their order, those left out among them
  float* largest_weight;   // largest |dloss| of them (of the finite ones), and that over the temperature
  int* order;              // tokens that count, in order; the last ones left out
  uint8_t* counts;         // of a token, where that takes more than a look at its target
  // Rows of the operands of the products are whole lines of 128 bytes: one plane in bf16, or three for single precision (see loss_tile.hpp)
  void* states;            // hidden states of the piece, states_ld to a row and plane, zeros behind the width and the last row
  const void* head;        // the head (its own memory, where its rows begin at multiples of 16 bytes and end there), head_ld to a row
  float2* sums;            // of each row and tile: a logit c, the sum of 2^((z - c) scale + bits) (bits: exp_bits)
  // the logits of the entries, by the workgroups that make them
  float* dots;             // of each row and entry
  int* words;              // of each row: its only entry (NULL: they are read where they are, or there are several)
  uint32_t* sorted;        // of each row: its k entries by word, word << 8 | entry, those that take no part behind (NULL likewise, or k is 1)
  uint16_t* begins;        // of each row and part of a tile, and once more: how many entries stand before it
  // Exponentials counted from one number for a row (bf16, dh alone): they are dz but for a factor of the row, which dh takes at the end, and
  // its entries.  The number comes from the logits of some of the row's entries before all others are known.
  float* refs;             // of each row; NULL: counted from the largest logit of each part of a tile
  int* again;              // not 0: a row has exponentials too far above its number, and all are made again the other way
  float2* row_scale;       // of each row: what dh is multiplied with, in two factors
  void* exps;              // exponentials of the piece, dz_ld to a row: fp16 in the memory of dz (bf16), or fp32
  void* dz;                // of the piece, dz_ld to a row and plane, zeros behind the vocabulary
  float* dweight_sum;      // the head's gradient of the pieces so far (bf16 and more than one piece)
  floatx4* parts;          // of tiles whose sums workgroups share
  int groups;              // workgroups that share the tiles of a product
  int64_t head_ld, states_row;  // states_row: elements from row to row of the states
  int states_ld, dz_ld, head_bytes;  // head_bytes: of a row of a plane of the head
  int tile_n, tiles;       // words of a wave's part of a tile of logits, such parts of a row
  // of the piece
  int first, rows;         // of `order`
  bool last;
  int head_first, head_rows;  // words whose gradient a launch makes
};

// rows of the piece that there are
__device__ __forceinline__ int rows_of(const LossCall& c) { return c.count ? min(max(*c.count - c.first, 0), c.rows) : c.rows; }

// An exponential is 2^exp_bits for the largest of its row and tile: kept in fp16 (bf16 matrices, not counted from c.refs) they then have 11 bits down
// to 2^-29 of that one, and steps of 2^-39 of it below.
__host__ __device__ constexpr float exp_bits(bool bf16, bool counted) { return bf16 && !counted ? 15.0f : 0.0f; }
// The difference is taken before the scaling, so that the largest is 2^bits whatever the scale is.
__device__ __forceinline__ float exp_from(float z, float from, float scale, float bits) { return __builtin_amdgcn_exp2f(fmaf(z - from, scale, bits)); }

// the only entry of a row, -1 for none
__device__ __forceinline__ int word_of(const LossCall& c, int row) {
  if (c.words) return c.words[row];
  const int64_t id = c.ids[(int64_t)(c.first + row) * c.ids_ld];
  return id >= 0 && id < c.vocab ? (int)id : -1;
}

// logits of up to kFewTokens
void launch_few_logits(const LossCall& c, bool bf16, hipStream_t s);
void launch_few_dh(const LossCall& c, const FewDhPlan& plan, bool bf16, hipStream_t s);  // dh of up to kFewTokens
void launch_logits(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s);
void launch_dh(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s);
void launch_both(const LossCall& c, const BothPlan& plan, bool bf16, hipStream_t s);  // dh and dW
void launch_dweight(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s);

}  // namespace tsenor_dev
