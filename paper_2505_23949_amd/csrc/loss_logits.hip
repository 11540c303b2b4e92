#include "loss_tile.hpp"

namespace {
using namespace tsenor_dev;

// counted from c.refs, and the other way should that not do
template <int COUNTED, int PLAIN>
void launch_counted(const LossCall& c, unsigned tiles, hipStream_t s) {
  tile_kernel<true, COUNTED, 4, 2, 4, 2, kNever><<<tiles, TileShape<4, 2, 4>::kThreads, 0, s>>>(c);
  logits_again_kernel<PLAIN><<<std::min<unsigned>(tiles, kCus), TileShape<4, 2, 4>::kThreads, 0, s>>>(c, (int)tiles);
}
}  // namespace

void tsenor_dev::launch_logits(const LossCall& c, const ProductPlan& plan, bool bf16, hipStream_t s) {
  const bool in_place = c.head_bytes % 128 != 0;
  const unsigned tiles = (unsigned)(plan.tiles_m * plan.tiles_n);
  if (!bf16)
    launch_tiles<false, kLogits>(c, plan, s);
  else if (c.refs)
    in_place ? launch_counted<kLogitsInPlaceCounted, kLogitsInPlace>(c, tiles, s) : launch_counted<kLogitsCounted, kLogits>(c, tiles, s);
  else
    in_place ? launch_tiles<true, kLogitsInPlace>(c, plan, s) : launch_tiles<true, kLogits>(c, plan, s);
}
