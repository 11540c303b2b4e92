#include "loss_tile.hpp"

void tsenor_dev::launch_logits(const LossCall& c, bool bf16, hipStream_t s) { bf16 ? launch_tiles<true, kLogits>(c, s) : launch_tiles<false, kLogits>(c, s); }
