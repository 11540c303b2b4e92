#include "loss_tile.hpp"

void tsenor_dev::launch_dh(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s) {
  bf16 ? launch_tiles<true, kStates>(c, plan, s) : launch_tiles<false, kStates>(c, plan, s);
}
