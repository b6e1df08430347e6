// The 128 x 128 tile kernels on bf16 operands.
#include "mm_tile.h"

namespace muon {
namespace layers {

hipError_t launch_tile128_bf16(int form, int group, const Product& p, const Table* t, hipStream_t st) {
  return launch_form<__bf16, 128, 128, 5>(form, group, p, t, st);
}

}  // namespace layers
}  // namespace muon
