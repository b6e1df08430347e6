// The loss's products on 128 x 128 tiles of fp32 operands.
#include "mm_tile.h"

namespace muon {
namespace layers {

hipError_t launch_loss128_f32(int step, int form, const Product& p, const LossArgs& a, hipStream_t st) {
  return launch_loss_step<float, 128, 128, 5>(step, form, p, a, st);
}

}  // namespace layers
}  // namespace muon
