// The 256 x 256 tile kernels on bf16 operands.
#include "mm_tile.h"

namespace muon {
namespace layers {

hipError_t launch_tile256_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  return launch_form<__bf16, 256, 256, 5>(form, group, p, t, st);
}

}  // namespace layers
}  // namespace muon
