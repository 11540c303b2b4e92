/*
 * tsenor_loss.h - C ABI of the losses that a masked model is retrained with, on MI355X (gfx950): from the final hidden states of its
 * tokens through the product with the head (a matrix with a row for each word of the vocabulary) to a loss for each token and the
 * gradients of both.
 *
 *   tsenor_cross_entropy   softmax cross entropy: the model learns the next word of a text
 *   tsenor_distill         divergence from a teacher's top logits: the pruned model learns what the dense one answers
 *
 * Conventions are those of tsenor.h and tsenor_layer.h (device pointers of the caller, problem structs in HOST memory, work enqueued on
 * `stream`, nothing allocated, everything checked before the first launch, calls that overlap in time do not share a workspace, calls
 * can be captured in a HIP graph, sums have a fixed order and there are no atomics; counts may be zero, and pointers to arrays without
 * elements NULL).  Besides:
 *   - The logits of a call are never all kept.  They are made and used in tiles; a call that wants gradients keeps what becomes their
 *     gradients, 2 bytes a logit (bf16) or 10 (fp32), for as many tokens as 2 GiB hold but 256 at the least (5 GiB at 2^21 words in fp32), and goes
 *     on to the next ones then (with a sum of dweight in fp32 beside it, for bf16).  Copies of the tokens' hidden states take up to as much, and
 *     so do sums with entries.
 *   - Loss and gradients are one call: nothing but a weight for each token comes between the loss and its gradients, and the product
 *     with the head is made once for both.
 *   - Logits, sums of exponentials and losses are in single precision, and a cross entropy near 0 is right to its own digits and never below 0.
 *     Gradients are summed in single precision and rounded to `dtype` once.  Of bf16 matrices, the gradient of a logit is rounded to bf16
 *     before it is multiplied, by at most 2^-8 of itself to either side (and its exponential, in calls with dweight_out or of few logits, to fp16
 *     before that, by 2^-11).
 *   - Gradients are made relative to the largest finite weight (dloss) of the call's tokens: of a token whose weight is less than 2^-90 of it they
 *     lose digits, and may be 0.
 *   - Tokens that are left out (no target, no entries) have loss, logarithm and gradients 0, whatever their hidden state is.
 *   - A logit that is NaN or infinite makes the loss of its token NaN, and with it the gradients it takes part in; but a word whose logit is
 *     minus infinity has probability 0: the loss is infinite if the word is the target (or an entry with a share of q), and what it is without the
 *     word if not.  (Of fp32 matrices a product beyond single precision may be NaN.)  An infinite or NaN entry of the head may make NaN of all tokens.
 */
#ifndef TSENOR_LOSS_H
#define TSENOR_LOSS_H

#include "tsenor.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { TSENOR_LOSS_MAX_ENTRIES = 256 };

/* What both losses have in common: z[t][j] = sum_c h[t][c] weight[j][c]. */
typedef struct tsenor_head {
  const void* h;          /* tokens x width of `dtype`, leading dimension h_ld */
  const void* weight;     /* vocab x width of `dtype`, leading dimension weight_ld */
  int32_t dtype;          /* TSENOR_F32 or TSENOR_BF16 */
  int64_t tokens, vocab, width, h_ld, weight_ld; /* tokens at most 2^24, vocab 2^21, width 2^16; leading dimensions 2^40 */
  const float* dloss;     /* optional, tokens floats: the gradient of each token's loss (1 if NULL) */
  float* loss_out;        /* tokens floats */
  float* lse_out;         /* optional, tokens floats: log sum_j exp(z[t][j]) (of z / temperature) */
  void* dh_out;           /* optional, tokens x width of `dtype`, leading dimension width */
  void* dweight_out;      /* optional, vocab x width of `dtype`, leading dimension width: written, not added to */
} tsenor_head;            /* outputs overlap no other argument */

/* loss[t] = lse[t] - z[t][target];  dz[t][j] = dloss[t] (exp(z[t][j] - lse[t]) - (j == target))
 * dh = dz weight;  dweight = dz^T h */
typedef struct tsenor_cross_entropy_problem {
  tsenor_head head;
  const int64_t* targets; /* tokens; one that is not in 0 .. vocab - 1 leaves its token out */
} tsenor_cross_entropy_problem;
size_t tsenor_cross_entropy_workspace_bytes(const tsenor_cross_entropy_problem* p); /* 0 on invalid arguments */
int tsenor_cross_entropy(const tsenor_cross_entropy_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream);

/* The teacher's distribution over k words of each token, q = softmax(logits / temperature), against the model's over all of them:
 *   loss[t] = sum_i q[t][i] (log q[t][i] - z[t][id] / temperature + lse[t])          (0 log 0 = 0)
 *   dz[t][j] = dloss[t] / temperature (exp(z[t][j] / temperature - lse[t]) - sum_i q[t][i] (j == id))
 * Entries whose id is not in 0 .. vocab - 1 take no part, and a token with none that does, or with nothing but logits of minus
 * infinity, is left out.  An id may stand more than once: each is an entry of its own.  A caller that wants gradients independent of the temperature
 * puts its square into dloss. */
typedef struct tsenor_distill_problem {
  tsenor_head head;
  const int64_t* ids;     /* tokens x k, leading dimension ids_ld */
  const void* logits;     /* tokens x k of `logits_dtype`, leading dimension logits_ld */
  int32_t logits_dtype;   /* TSENOR_F32 or TSENOR_BF16 */
  int32_t k;              /* 0 .. TSENOR_LOSS_MAX_ENTRIES */
  int64_t ids_ld, logits_ld;
  double temperature;     /* 2^-20 .. 2^20 */
} tsenor_distill_problem;
size_t tsenor_distill_workspace_bytes(const tsenor_distill_problem* p); /* 0 on invalid arguments */
int tsenor_distill(const tsenor_distill_problem* p, void* workspace, size_t workspace_bytes, tsenor_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* TSENOR_LOSS_H */
