// The 128 x 128 tile kernels on fp32 operands.
#include "mm_tile.h"

namespace muon {
namespace layers {

hipError_t launch_tile128_f32(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  return launch_form<float, 128, 128, 5>(form, group, p, t, st);
}

}  // namespace layers
}  // namespace muon
