#include "loss_tile.hpp"

void tsenor_dev::launch_dh(const LossCall& c, bool bf16, hipStream_t s) { bf16 ? launch_tiles<true, kStates>(c, s) : launch_tiles<false, kStates>(c, s); }
