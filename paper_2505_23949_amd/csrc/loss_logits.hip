#include "loss_tile.hpp"

void tsenor_dev::launch_logits(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s) {
  bf16 ? launch_tiles<true, kLogits>(c, plan, s) : launch_tiles<false, kLogits>(c, plan, s);
}
