// The 64 x 64 tile kernels on fp32 operands.
#include "mm_tile.h"

namespace muon {
namespace layers {

hipError_t launch_tile64_f32(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  return launch_form<float, 64, 64, 10>(form, group, p, t, st);
}

}  // namespace layers
}  // namespace muon
