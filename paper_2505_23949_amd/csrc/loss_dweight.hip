#include "loss_tile.hpp"

void tsenor_dev::launch_dweight(const LossCall& c, bool bf16, hipStream_t s) { bf16 ? launch_tiles<true, kHead>(c, s) : launch_tiles<false, kHead>(c, s); }
