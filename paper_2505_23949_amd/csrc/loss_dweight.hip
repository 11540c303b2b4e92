#include "loss_tile.hpp"

void tsenor_dev::launch_dweight(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s) {
  bf16 ? launch_tiles<true, kHead>(c, plan, s) : launch_tiles<false, kHead>(c, plan, s);
}
