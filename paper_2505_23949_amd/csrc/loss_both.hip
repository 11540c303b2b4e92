#include "loss_tile.hpp"

void tsenor_dev::launch_both(const LossCall& c, const BothPlan& plan, bool bf16, hipStream_t s) {
  if (plan.dh.kind == kTile)
    bf16 ? launch_both<true, 2, 1, 4, 4>(c, plan, s) : launch_both<false, 2, 1, 4, 4>(c, plan, s);
  else
    bf16 ? launch_both<true, 2, 1, 2, 6>(c, plan, s) : launch_both<false, 2, 1, 2, 6>(c, plan, s);
}
