// The loss's products on 64 x 64 tiles of bf16 operands.
#include "mm_tile.h"

namespace muon {
namespace layers {

hipError_t launch_loss64_bf16(int step, int form, const Product& p, const LossArgs& a, hipStream_t st) {
  return launch_loss_step<__bf16, 64, 64, 10>(step, form, p, a, st);
}

}  // namespace layers
}  // namespace muon
