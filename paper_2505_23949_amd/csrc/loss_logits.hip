#include "loss_tile.hpp"

void tsenor_dev::launch_logits(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s) {
  if (!bf16)
    launch_tiles<false, kLogits>(c, plan, s);
  else if (c.head_bytes % 128)
    launch_tiles<true, kLogitsInPlace>(c, plan, s);
  else
    launch_tiles<true, kLogits>(c, plan, s);
}
